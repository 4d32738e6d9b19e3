"""kvx_attend where seen slots hold values that are not finite: what comes out, and at what cost."""
import pytest
import torch

from test_gpu_decode import Problem, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("d,new", [(64, 300), (128, 300), (256, 300), (128, 1)])
def test_rows_that_cannot_come_out_finite_cost_no_more(d, new, bad, dtype):
    """One key in a slot that every row of a sequence sees: scores of NaN or infinities, so sums and outputs of NaN, in about the
    time of finite ones.  (Summed again slot by slot each row costs thousands of reads, one after the other.)"""
    p = Problem(2, 4, d, [6000, 500], [new, new], dtype, 16, seed=81)
    good_k, k, v = p.cache(p.K), p.K.clone(), p.cache(p.V)
    k[0, :, 17] = bad
    k = p.cache(k)
    q, off, n = p.q.cuda(), i32(p.off), i32(p.L)
    out, lse = torch.zeros_like(q), torch.zeros((p.T, 8), device="cuda")
    base = torch.zeros_like(q)

    def call(keys, to):
        p.dec.attend(q, off, n, keys, v, to, lse=lse, **p.paged())

    def us(keys, to):
        best = float("inf")
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            call(keys, to)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b) * 1e3)
        return best

    clean, dirty = us(good_k, base), us(k, out)
    scores = q[:new].double().abs().sum(-1) > 0
    assert bool(scores.all())
    assert bool(out[:new].isnan().all()) and bool(lse[:new].isnan().all() if bad != bad else ~lse[:new].isfinite().any())
    assert torch.equal(out[new:], base[new:])       # the other sequence's rows
    assert p.dec.device_status() == 0
    assert dirty < 3 * clean + 50, (dirty, clean)
