// kvx_attend.cu -- attention of new tokens over an fp32 cache on the CUDA cores, and the choice of the
// attention kernels.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(x_ij - m_i),  x_ij = cap(scale q_i . k_j)
// in one pass over the slots j with the running maximum m_i and sum (kept in units of log2).
//
// Bound by the fp32 FMA pipe where rows are many: a thread takes 4 rows by 4 slots (packed products, 8 16-byte reads of
// shared memory for 32 of them), 64 rows a CTA of 128 threads; 512 tokens of 12 heads of 128 over 1024 slots take 92 us, 26
// TFLOP/s of what the masks leave.  Few rows (16 a tile): by the copies of K and V, whose next tile is only begun when this
// one's is used up: a token of each of eight sequences over up to 16384 slots, 209 MB, 123 us, 1.7 TB/s; short ones by the
// fixed cost of a call.
#include <atomic>

#include "kvx_attend_rows.cuh"
#include "kvx_kernels.h"
#include "kvx_tc_common.cuh"

namespace kvx {
namespace {

// Two packed fp32 products added to a packed sum.
__device__ __forceinline__ float2 ffma2(float2 a, float2 b, float2 c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(r)
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)),
          "l"(reinterpret_cast<unsigned long long&>(c)));
    return reinterpret_cast<float2&>(r);
}

// A tile of R rows (BM queries or kBN slots) of D channels in shared memory, rows D + 4 floats apart (float4 reads of
// neighbouring rows fall into different banks), copied asynchronously.  off(r) gives a row's element offset, or -1
// for a row of zeros.
template <int D, int R, int THREADS, typename Off> __device__ __forceinline__ void load_tile(float* dst, const float* src, Off off)
{
    // a warp has R / 4 consecutive rows; lane l finds row l's place, so that lookups run side by side
    static_assert(THREADS == 128);
    constexpr int PER = D / 4, ROWS = R / 4, RPI = PER < 32 ? 32 / PER : 1;   // 16-byte chunks of a row; rows of one instruction
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long mine = lane < ROWS ? off(warp * ROWS + lane) : -1;
#pragma unroll 4
    for (int k = 0; k < ROWS; k += RPI) {
        const int r = k + lane / PER % RPI;
        const long long at = __shfl_sync(0xffffffffu, mine, r);
        float* d = dst + (warp * ROWS + r) * (D + 4);
#pragma unroll
        for (int c = lane % PER * 4; c < D; c += 128) {
            if (at < 0) *reinterpret_cast<float4*>(d + c) = make_float4(0.f, 0.f, 0.f, 0.f);
            else cp_async16(smem_u32(d + c), src + at + c);
        }
    }
}
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

constexpr int kBN = 32;          // slots a tile
constexpr int kThreads = 128;    // 16 row groups (tr) x 8 slot groups (tc)
constexpr int kTR = 16, kTC = 8, kKN = kBN / kTC;

// Scores of rows tr + 16 i and slots tc + 8 j of the tile: each thread RM x kKN of them.
template <int D, int RM>
__device__ __forceinline__ void scores(const float* sQ, const float* sK, int tr, int tc, float (&x)[RM][kKN])
{
    float2 acc[RM][kKN];
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int j = 0; j < kKN; ++j) acc[i][j] = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
        float4 q[RM], k[kKN];
#pragma unroll
        for (int i = 0; i < RM; ++i) q[i] = *reinterpret_cast<const float4*>(sQ + (tr + kTR * i) * (D + 4) + c);
#pragma unroll
        for (int j = 0; j < kKN; ++j) k[j] = *reinterpret_cast<const float4*>(sK + (tc + kTC * j) * (D + 4) + c);
#pragma unroll
        for (int i = 0; i < RM; ++i)
#pragma unroll
            for (int j = 0; j < kKN; ++j) {
                acc[i][j] = ffma2(make_float2(q[i].x, q[i].y), make_float2(k[j].x, k[j].y), acc[i][j]);
                acc[i][j] = ffma2(make_float2(q[i].z, q[i].w), make_float2(k[j].z, k[j].w), acc[i][j]);
            }
    }
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int j = 0; j < kKN; ++j) x[i][j] = acc[i][j].x + acc[i][j].y;
}

// A raw score in log2 units, capped (the capped scores' code in kernels of its own: inlined for each score, it
// would be most of a kernel's).
template <bool CAP> __device__ __forceinline__ float score2(const AttendParams& P, float dot, float inv_cap)
{
    float v = dot * P.scale;
    if constexpr (CAP) v = capped(v, P.cap, inv_cap);
    return v * kLog2e;
}

template <int D, int BM> constexpr int simt_smem()
{
    return ((BM + 2 * kBN) * (D + 4) + BM * (kBN + 4)) * 4 + (kMaxAttendBatch + 2) * 8;
}

// 128 threads on a tile of BM rows and 32 slots; K of the next tile is copied while V is multiplied, V
// while the scores are.
template <int D, int BM, bool CAP>
__global__ void __launch_bounds__(kThreads) attend_simt_kernel(const __grid_constant__ AttendParams P)
{
    constexpr int RM = BM / kTR, CN = D / 32;   // rows of a thread; its float4 column groups 4 tc + 32 n
    extern __shared__ __align__(16) float sm[];
    float* sQ = sm;
    float* sK = sQ + BM * (D + 4);
    float* sV = sK + kBN * (D + 4);
    float* sP = sV + kBN * (D + 4);             // [BM][kBN + 4]
    long long* sums = reinterpret_cast<long long*>(sP + BM * (kBN + 4));
    const int tid = threadIdx.x, tc = tid & 7, tr = tid >> 3, lane = tid & 31, warp = tid >> 5;
    const float inv_cap = P.cap > 0.0f ? 1.0f / P.cap : 0.0f;
    const Plan plan = make_plan<kBN, kThreads>(P, sums);
    WalkState state;
    SegmentWalk<kBN> walk(P, &plan, &state);
    Segment g;
    bool have = false;
    while (walk.next(g)) {
        have = true;
        const int rows = min(BM, g.s.n * P.G - g.rt * BM);
        const long long head = cache_head(P.cache) * g.h;
        auto slot_row = [&](int tile, int r) {
            const int j = tile * kBN + r;
            long long at = -1;
            if (j < g.s.L) {
                at = cache_row(P.cache, g.b, j);
                if (at < 0) set_status(P.status, KVX_DEV_PAGE_INVALID);
                else at += head;
            }
            return at;
        };
        auto load_slots = [&](float* dst, const void* src, int tile) {
            load_tile<D, kBN, kThreads>(dst, (const float*)src, [&](int r) { return slot_row(tile, r); });
            async_commit();
        };
        load_tile<D, BM, kThreads>(sQ, (const float*)P.q, [&](int r) {
            if (r >= rows) return -1ll;
            const RowId id = row_id(P, g.s, g.h, g.rt * BM + r);
            return (long long)(g.s.t0 + id.t) * P.q_t + (long long)id.head * P.q_h;
        });
        load_slots(sK, P.ck, g.kv.at(g.i0));
        int slot_i[RM];                          // the rows' own slots
        float m[RM], l[RM];
        float2 o[RM][2 * CN];
#pragma unroll
        for (int i = 0; i < RM; ++i) {
            slot_i[i] = g.s.slot((g.rt * BM + tr + kTR * i) / P.G);
            m[i] = -INFINITY;
            l[i] = 0.0f;
#pragma unroll
            for (int c = 0; c < 2 * CN; ++c) o[i][c] = make_float2(0.f, 0.f);
        }
        for (int it = 0; it < g.n; ++it) {
            const int tile = g.kv.at(g.i0 + it);
            load_slots(sV, P.cv, tile);
            async_wait<1>();
            __syncthreads();
            float x[RM][kKN];
            scores<D, RM>(sQ, sK, tr, tc, x);
            __syncthreads();
            if (it + 1 < g.n) load_slots(sK, P.ck, g.kv.at(g.i0 + it + 1));
            else async_commit();
#pragma unroll
            for (int i = 0; i < RM; ++i) {
                float top = -INFINITY;
                const int j0 = tile * kBN, lo = window_lo(P, slot_i[i]);
                const bool all = (j0 >= lo && j0 + kBN - 1 <= slot_i[i] && j0 + kBN <= g.s.L) || j0 + kBN <= g.s.pre;
#pragma unroll
                for (int j = 0; j < kKN; ++j) x[i][j] = score2<CAP>(P, x[i][j], inv_cap);
                if (!all)
#pragma unroll
                    for (int j = 0; j < kKN; ++j)
                        if (!sees(P, g.s, slot_i[i], j0 + tc + kTC * j)) x[i][j] = -INFINITY;
                if (P.scores && tr + kTR * i < rows && j0 < P.scores_stride) {   // for the weight sums
                    const RowId id = row_id(P, g.s, g.h, g.rt * BM + tr + kTR * i);
                    float* to = P.scores + ((long long)(g.s.t0 + id.t) * P.Hq + id.head) * P.scores_stride + j0 + tc;
#pragma unroll
                    for (int j = 0; j < kKN; ++j) __stcg(to + kTC * j, x[i][j]);
                }
#pragma unroll
                for (int j = 0; j < kKN; ++j) top = fmaxf(top, x[i][j]);
#pragma unroll
                for (int k = 4; k; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
                const float next = fmaxf(m[i], top), base = next == -INFINITY ? 0.0f : next;
                const float w = exp2_hw(m[i] - base);
                m[i] = next;
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < kKN; ++j) {
                    const float p = exp2_hw(x[i][j] - base);
                    sum += p;
                    sP[(tr + kTR * i) * (kBN + 4) + tc + kTC * j] = p;
                }
#pragma unroll
                for (int k = 4; k; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
                l[i] = fmaf(l[i], w, sum);
#pragma unroll
                for (int c = 0; c < 2 * CN; ++c) {
                    o[i][c].x *= w;
                    o[i][c].y *= w;
                }
            }
            async_wait<1>();
            __syncthreads();
#pragma unroll 2
            for (int j = 0; j < kBN; j += 4) {
                float4 p[RM];
#pragma unroll
                for (int i = 0; i < RM; ++i) p[i] = *reinterpret_cast<const float4*>(sP + (tr + kTR * i) * (kBN + 4) + j);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c = 0; c < CN; ++c) {
                        const float4 v = *reinterpret_cast<const float4*>(sV + (j + e) * (D + 4) + 4 * tc + 32 * c);
#pragma unroll
                        for (int i = 0; i < RM; ++i) {
                            const float pe = e == 0 ? p[i].x : e == 1 ? p[i].y : e == 2 ? p[i].z : p[i].w;
                            o[i][2 * c] = ffma2(make_float2(pe, pe), make_float2(v.x, v.y), o[i][2 * c]);
                            o[i][2 * c + 1] = ffma2(make_float2(pe, pe), make_float2(v.z, v.w), o[i][2 * c + 1]);
                        }
                    }
            }
            __syncthreads();
        }
        async_wait<0>();
        if (g.whole()) {
            // through shared memory (the queries' place), so that a warp has a whole row
#pragma unroll
            for (int i = 0; i < RM; ++i) {
                const int r = tr + kTR * i;
#pragma unroll
                for (int c = 0; c < CN; ++c)
                    *reinterpret_cast<float4*>(sQ + r * (D + 4) + 4 * tc + 32 * c) =
                        make_float4(o[i][2 * c].x, o[i][2 * c].y, o[i][2 * c + 1].x, o[i][2 * c + 1].y);
                if (tc == 0) {
                    sP[r * (kBN + 4)] = m[i];
                    sP[r * (kBN + 4) + 1] = l[i];
                }
            }
            __syncthreads();
            for (int r = warp; r < rows; r += kThreads / 32) {
                float y[D / 32];
#pragma unroll
                for (int c = 0; c < D / 32; ++c) y[c] = sQ[r * (D + 4) + lane * (D / 32) + c];
                const RowId id = row_id(P, g.s, g.h, g.rt * BM + r);
                finish_row<float, D>(P, g.b, g.h, g.rt * BM + r, g.s.t0 + id.t, id.head, sP[r * (kBN + 4)], sP[r * (kBN + 4) + 1], y);
            }
        } else {
            const size_t at = (size_t)(2 * blockIdx.x + (g.first ? 0 : 1)) * BM;
#pragma unroll
            for (int i = 0; i < RM; ++i) {
                const int r = tr + kTR * i;
                if (r >= rows) continue;
#pragma unroll
                for (int c = 0; c < CN; ++c)
                    __stcg(reinterpret_cast<float4*>(P.part_o + (at + r) * D + 4 * tc + 32 * c),
                           make_float4(o[i][2 * c].x, o[i][2 * c].y, o[i][2 * c + 1].x, o[i][2 * c + 1].y));
                if (tc == 0) __stcg(P.part_ml + at + r, make_float2(m[i], l[i]));
            }
        }
        __syncthreads();
    }
    if (tid == 0) leave_split(P, plan, g, have);
}

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

template <auto Kernel> int ctas_per_sm(int smem, int threads)
{
    static std::atomic<int> known{0};
    int n = known.load();
    if (n == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, Kernel, threads, smem) != cudaSuccess || n < 1) n = 1;
        known.store(n);
    }
    return n;
}

template <int D, int BM, bool CAP> cudaError_t run_simt(const AttendParams& call, int num_sms, cudaStream_t stream)
{
    AttendParams P = call;
    P.tile_rows = BM;
    constexpr int smem = simt_smem<D, BM>();
    if (cudaError_t e = smem_opt_in<attend_simt_kernel<D, BM, CAP>>(smem); e != cudaSuccess) return e;
    const int grid = min(num_sms * ctas_per_sm<attend_simt_kernel<D, BM, CAP>>(smem, kThreads), kAttendMaxRows / BM / 2);
    attend_simt_kernel<D, BM, CAP><<<grid, kThreads, smem, stream>>>(P);
    if (cudaError_t e = cudaGetLastError(); e != cudaSuccess) return e;
    return run_join<float, D, BM>(P, grid, stream);
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
    return few ? run_simt<D, 16, CAP>(P, num_sms, stream) : run_simt<D, D == 256 ? 32 : 64, CAP>(P, num_sms, stream);
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
