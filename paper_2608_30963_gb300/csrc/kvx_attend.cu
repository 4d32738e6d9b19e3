// kvx_attend.cu -- attention of new tokens over an fp32 cache on the CUDA cores (kvx_attend_simt.cuh), its weight sums, and
// the choice of the attention kernels.
#include "kvx_attend_simt.cuh"
#include "kvx_kernels.h"
#include "kvx_tc_common.cuh"

namespace kvx {
namespace {

// key_weight[b, h, j] += sum over the rows i of (b, h) of exp(x_ij - lse_i): the scores are formed again, now
// that every row's sum is known, one CTA to a tile of 32 slots, which no other CTA adds to.
template <int D> constexpr int weight_smem()
{
    return ((64 + kBN) * (D + 4) + 64 + kTR * kBN) * 4 + (kMaxAttendBatch + 2) * 8;
}
template <int D, bool CAP>
__global__ void __launch_bounds__(kThreads) key_weight_simt_kernel(const __grid_constant__ AttendParams P)
{
    constexpr int BM = 64, RM = BM / kTR;
    extern __shared__ __align__(16) float sm[];
    float* sQ = sm;
    float* sK = sQ + BM * (D + 4);
    float* sL = sK + kBN * (D + 4);             // the rows' lse in log2 units, +infinity past the end
    float* sW = sL + BM;                        // [kTR][kBN]
    long long* first = reinterpret_cast<long long*>(sW + kTR * kBN);   // slot tiles before each sequence's
    const int tid = threadIdx.x, tc = tid & 7, tr = tid >> 3;
    const float inv_cap = P.cap > 0.0f ? 1.0f / P.cap : 0.0f;
    for (int b = tid; b < P.batch; b += kThreads) first[b + 1] = (load_seq(P, b).L + kBN - 1) / kBN;
    if (tid == 0) first[0] = 0;
    __syncthreads();
    if (tid == 0)
        for (int b = 0; b < P.batch; ++b) first[b + 1] += first[b];
    __syncthreads();
    const long long units = first[P.batch] * P.H;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const long long ut = u / P.H;
        const int h = (int)(u - ut * P.H);
        int lo = 0, hi = P.batch - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (first[mid] <= ut) lo = mid; else hi = mid - 1;
        }
        const int b = lo, j0 = (int)(ut - first[b]) * kBN;
        const Seq s = load_seq(P, b);
        // rows of tokens before the first that sees the tile need not be formed
        const int t_first = j0 < s.pre ? 0 : max(0, j0 - (s.L - s.n));
        const int t_end = (j0 < s.pre || P.window == 0) ? s.n : (int)min((long long)s.n, (long long)j0 + kBN - 1 + P.window - (s.L - s.n));
        if (t_end <= t_first) continue;         // no token sees the tile (the whole CTA): no copy is begun that nothing waits for
        __syncthreads();
        load_tile<D, kBN, kThreads>(sK, (const float*)P.ck, [&](int r) {
            const long long at = j0 + r < s.L ? cache_row(P.cache, b, j0 + r) : -1;
            return at < 0 ? -1ll : at + cache_head(P.cache) * h;
        });
        float w[kKN];
#pragma unroll
        for (int j = 0; j < kKN; ++j) w[j] = 0.0f;
        for (int r0 = t_first * P.G; r0 < t_end * P.G; r0 += BM) {
            const int rows = min(BM, t_end * P.G - r0);
            load_tile<D, BM, kThreads>(sQ, (const float*)P.q, [&](int r) {
                if (r >= rows) return -1ll;
                const RowId id = row_id(P, s, h, r0 + r);
                return (long long)(s.t0 + id.t) * P.q_t + (long long)id.head * P.q_h;
            });
            async_commit();
            for (int r = tid; r < BM; r += kThreads) {
                float z = INFINITY;
                if (r < rows) {
                    const RowId id = row_id(P, s, h, r0 + r);
                    z = P.lse[(long long)(s.t0 + id.t) * P.Hq + id.head] * kLog2e;
                }
                sL[r] = z;
            }
            async_wait<0>();
            __syncthreads();
            float x[RM][kKN];
            scores<D, RM>(sQ, sK, tr, tc, x);
#pragma unroll
            for (int i = 0; i < RM; ++i) {
                const int r = tr + kTR * i;
                const int own = s.slot((r0 + r) / P.G);
#pragma unroll
                for (int j = 0; j < kKN; ++j)
                    if (r < rows && sees(P, s, own, j0 + tc + kTC * j)) w[j] += exp2_hw(score2<CAP>(P, x[i][j], inv_cap) - sL[r]);
            }
            __syncthreads();
        }
#pragma unroll
        for (int j = 0; j < kKN; ++j) sW[tr * kBN + tc + kTC * j] = w[j];
        __syncthreads();
        if (tid < kBN && j0 + tid < s.L && j0 + tid < P.weight_stride) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < kTR; ++i) sum += sW[i * kBN + tid];
            P.key_weight[((long long)b * P.H + h) * P.weight_stride + j0 + tid] += sum;
        }
        __syncthreads();
    }
}

template <int D, bool CAP> cudaError_t run_weight_simt(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    constexpr int smem = weight_smem<D>();
    if (cudaError_t e = smem_opt_in<key_weight_simt_kernel<D, CAP>>(smem); e != cudaSuccess) return e;
    const int grid = num_sms * ctas_per_sm<key_weight_simt_kernel<D, CAP>>(smem, kThreads);
    key_weight_simt_kernel<D, CAP><<<grid, kThreads, smem, stream>>>(P);
    return cudaGetLastError();
}

template <int D, bool CAP> cudaError_t run_fp32(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    // Few rows for each sequence and head: 16-row tiles waste less of the arithmetic (eight sequences of 4096 slots, heads of
    // 128: 12 rows 79.5 us in tiles of 16 and 89.8 of 64, 18 rows 96.9 and 90.8; heads of 256: 93.9 and 99.0, 162 and 102)
    const bool few = (long long)P.T * P.G <= 16ll * P.batch;
    return few ? run_simt<D, 16, CAP, false>(P, num_sms, stream) : run_simt<D, D == 256 ? 32 : 64, CAP, false>(P, num_sms, stream);
}
template <bool CAP> cudaError_t attend_fp32(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    return P.d == 64 ? run_fp32<64, CAP>(P, num_sms, stream) : P.d == 128 ? run_fp32<128, CAP>(P, num_sms, stream) : run_fp32<256, CAP>(P, num_sms, stream);
}
template <bool CAP> cudaError_t weigh_fp32(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    return P.d == 64 ? run_weight_simt<64, CAP>(P, num_sms, stream) : P.d == 128 ? run_weight_simt<128, CAP>(P, num_sms, stream)
                                                                             : run_weight_simt<256, CAP>(P, num_sms, stream);
}

}  // namespace

cudaError_t launch_attend(const AttendParams& call, int dtype, int num_sms, cudaStream_t stream, int* launches)
{
    *launches = 0;
    if (call.T == 0) return cudaSuccess;
    AttendParams P = call;
    const bool bf16 = dtype == KVX_BF16;
    // Weight sums add up the scores that the attention leaves, where they fit the workspace and cost less than to be formed
    // again: always in fp32 (8 bytes of traffic against 2 d operations on the CUDA cores: 512 tokens of 12 heads over
    // 512 slots 209 us, 48 so), for few rows in bf16 (16 a sequence and KV head: less than a slot's K; four sequences of 16000
    // slots, 14 rows 83.6 us kept and 91.8 formed again, 28 rows 97.9 and 98.9; one sequence, 28 rows 50.8 and 46.8).
    // (weight_stride is the caller's, up to 2^63: divided by, not multiplied)
    const long long most = kAttendScores / ((long long)P.T * P.Hq) / 64 * 64;   // slots a row of the workspace may have
    const bool keep = P.key_weight && (!bf16 || (long long)P.T * P.G <= 16ll * P.batch) && P.weight_stride <= most;
    P.scores_stride = keep ? (P.weight_stride + 63) / 64 * 64 : 0;
    if (!keep) P.scores = nullptr;
    const bool cap = P.cap > 0.0f;
    cudaError_t e = bf16 ? launch_attend_tc(P, num_sms, stream) : cap ? attend_fp32<true>(P, num_sms, stream) : attend_fp32<false>(P, num_sms, stream);
    *launches = 2;
    if (e != cudaSuccess || !P.key_weight) return e;
    *launches = 3;
    if (keep) return launch_sum_scores(P, stream);
    if (bf16) return launch_key_weight(P, num_sms, stream);
    return cap ? weigh_fp32<true>(P, num_sms, stream) : weigh_fp32<false>(P, num_sms, stream);
}

}  // namespace kvx
