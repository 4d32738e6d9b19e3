// kvx_attend_codes.cu -- attention of new tokens over an 8-bit cache: the choice of the kernels.
#include "kvx_attend_simt.cuh"

namespace kvx {
namespace {

// fp32 queries: on the CUDA cores
template <int D, bool CAP> cudaError_t run_fp32(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    // few rows: 16-row tiles, as over fp32 caches
    const bool few = (long long)P.T * P.G <= 16ll * P.batch;
    return few ? run_simt<D, 16, CAP, true>(P, num_sms, stream) : run_simt<D, D == 256 ? 32 : 64, CAP, true>(P, num_sms, stream);
}
template <bool CAP> cudaError_t attend_fp32(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    return P.d == 64 ? run_fp32<64, CAP>(P, num_sms, stream) : P.d == 128 ? run_fp32<128, CAP>(P, num_sms, stream) : run_fp32<256, CAP>(P, num_sms, stream);
}

// Prompts: every row tile of a (sequence, KV head) reads its slots again, so from some rows on the slots become bf16
// once, in the workspace (64 MiB, where the call's cache may fit it), and the kernels of bf16 caches take them from there.
// (One sequence, us so and with the codes converted by each row tile: 7 query heads on each of 4 KV heads of 128 over 16384
// slots, 896 rows 58 and 55, 1344 rows 72 and 71, 1792 rows 80 and 82, 7168 rows 207 and 247; heads of 256, whose tiles have 128
// rows, over 8192 slots, 384 rows 50 and 48, 512 rows 52 and 54, 768 rows 56 and 64, over 2000 slots 768 rows 37 and 36, 1024 rows 39
// and 39; heads of 64, 4096 rows 36 and 35, 8192 rows 46 and 47; 4096 tokens over 32768 slots 1166 and 1568.
// Capped scores: heads of 128, 1792 rows 382 and 221, 7168 rows 1040 and 677, so not there; heads of 256, 1024 rows 75 and 86.)
bool expands(const AttendParams& P)
{
    const int rows = P.d == 256 ? 512 : 1536;
    if (P.cap > 0.0f && P.d == 128) return false;
    // (batch <= 1024, capacity <= 2^30: no product wraps)
    return (long long)P.T * P.G > (long long)rows * P.batch && (long long)P.batch * P.cache.capacity <= kAttendScores / ((long long)P.H * P.d);
}
// Few rows: the rows of a tile (8, 16 or 32) that hold the call's mean a sequence and KV head, in whole tokens, or 0.  (Four
// sequences of 16384 slots, us so and with the codes converted: 7 rows on each of 4 KV heads of 128 23 and 48, 28 rows 46 and 56, on 8
// KV heads 32 rows 63 and 84; heads of 256 over 8192 slots, 2 rows 22 and 40, 32 rows 45 and 50; one sequence of 2000 slots, 32
// rows 18.5 and 18.0.  A head of 64 fills half of a 128-byte block: not taken.)
int few_rows(const AttendParams& P)
{
    if (P.d == 64) return 0;
    for (int r = 8; r <= 32; r *= 2)
        if (P.G <= r && (long long)P.T * P.G <= (long long)(r / P.G * P.G) * P.batch) return r;
    return 0;
}
cudaError_t attend_expanded(const AttendParams& call, int num_sms, cudaStream_t stream)
{
    AttendParams P = call;
    __nv_bfloat16* k = reinterpret_cast<__nv_bfloat16*>(call.scores);
    __nv_bfloat16* v = k + (long long)P.batch * P.H * P.cache.capacity * P.d;
    if (cudaError_t e = launch_expand(call, k, v, num_sms, stream); e != cudaSuccess) return e;
    P.ck = k;
    P.cv = v;
    P.k_scale = P.v_scale = nullptr;
    P.scores = nullptr;
    P.cache.paged = 0;
    P.cache.page_table = nullptr;
    P.cache.st = P.d;
    P.cache.sh = (long long)P.cache.capacity * P.d;
    P.cache.sb = P.cache.sh * P.H;
    return launch_attend_tc(P, num_sms, stream);
}

}  // namespace

cudaError_t launch_attend_codes(const AttendParams& call, int dtype, int num_sms, cudaStream_t stream, int* launches)
{
    *launches = 0;
    if (call.T == 0) return cudaSuccess;
    AttendParams P = call;
    P.scores = nullptr;                          // no weight sums
    const bool cap = P.cap > 0.0f;
    *launches = 2;
    if (dtype != KVX_BF16) return cap ? attend_fp32<true>(P, num_sms, stream) : attend_fp32<false>(P, num_sms, stream);
    if (const int rows = few_rows(P)) return cap ? launch_attend_few_capped(P, rows, num_sms, stream) : launch_attend_few(P, rows, num_sms, stream);
    if (!expands(P)) return cap ? launch_attend_tc_codes_capped(P, num_sms, stream) : launch_attend_tc_codes(P, num_sms, stream);
    *launches = 3;
    return attend_expanded(call, num_sms, stream);
}

}  // namespace kvx
