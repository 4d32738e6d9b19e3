// kvx_attend_simt.cuh -- attention of new tokens on the CUDA cores, over fp32 caches and over 8-bit ones (library-internal).
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(x_ij - m_i),  x_ij = cap(scale q_i . k_j)
// in one pass over the slots j with the running maximum m_i and sum (kept in units of log2).
//
// Bound by the fp32 FMA pipe where rows are many: a thread takes 4 rows by 4 slots (packed products, 8 16-byte reads of
// shared memory for 32 of them), 64 rows a CTA of 128 threads; 512 tokens of 12 heads of 128 over 1024 slots take 92 us, 26
// TFLOP/s of what the masks leave.  Few rows (16 a tile): by the copies of K and V, whose next tile is only begun when this
// one's is used up: a token of each of eight sequences over up to 16384 slots, 209 MB, 123 us, 1.7 TB/s; short ones by the
// fixed cost of a call.
// Over 8-bit caches tiles come through registers, a phase ahead, and lie in shared memory as fp32.
#pragma once

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

// Codes of an 8-bit tile of kBN slots on their way: 16 of a row to a thread at a time, loaded a phase ahead into registers
// (the copies of a tile of the type that it is multiplied in go straight to shared memory).
template <int D> struct CodeTile {
    static constexpr int PER = D / 16, N = kBN * PER / kThreads;    // 16-code chunks of a row; of a thread
    uint4 w[N];
    float scale[N];
    template <typename Place> __device__ __forceinline__ void fetch(const uint8_t* src, const uint8_t* scales, Place place)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int x = i * kThreads + threadIdx.x;
            const CodePlace at = place(x / PER);
            scale[i] = 0.0f;
            w[i] = make_uint4(0u, 0u, 0u, 0u);
            if (at.row >= 0) {
                w[i] = __ldg(reinterpret_cast<const uint4*>(src + at.row) + x % PER);
                scale[i] = scale_of(__ldg(scales + at.scale));
            }
        }
    }
    __device__ __forceinline__ void put(float* dst) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int x = i * kThreads + threadIdx.x;
            float* d = dst + x / PER * (D + 4) + x % PER * 16;
            const uint32_t in[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 lo = codes_f32((unsigned short)in[e]), hi = codes_f32((unsigned short)(in[e] >> 16));
                *reinterpret_cast<float4*>(d + 4 * e) = make_float4(lo.x * scale[i], lo.y * scale[i], hi.x * scale[i], hi.y * scale[i]);
            }
        }
    }
};

template <int D, int BM> constexpr int simt_smem()
{
    return ((BM + 2 * kBN) * (D + 4) + BM * (kBN + 4)) * 4 + (kMaxAttendBatch + 2) * 8;
}

// 128 threads on a tile of BM rows and 32 slots; K of the next tile is copied while V is multiplied, V
// while the scores are.
template <int D, int BM, bool CAP, bool CODES>
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
        auto query = [&](int r) {
            if (r >= rows) return -1ll;
            const RowId id = row_id(P, g.s, g.h, g.rt * BM + r);
            return (long long)(g.s.t0 + id.t) * P.q_t + (long long)id.head * P.q_h;
        };
        load_tile<D, BM, kThreads>(sQ, (const float*)P.q, query);
        // (8 bits: a tile is fetched where its copies would begin, and put where they would be waited for)
        CodeTile<D> codes;
        auto begin = [&](float* dst, const void* src, const unsigned char* scales, int tile) {
            if constexpr (CODES)
                codes.fetch((const uint8_t*)src + head, scales + scale_head(P.cache, P.scales) * g.h, [&](int r) {
                    const int j = tile * kBN + r;
                    if (j >= g.s.L) return CodePlace{-1, -1};
                    const CodePlace at = code_place(P.cache, P.scales, g.b, j);
                    if (at.row < 0) set_status(P.status, KVX_DEV_PAGE_INVALID);
                    return at;
                });
            else load_slots(dst, src, tile);
        };
        begin(sK, P.ck, P.k_scale, g.kv.at(g.i0));
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
            if constexpr (CODES) codes.put(sK);
            begin(sV, P.cv, P.v_scale, tile);
            if constexpr (CODES) cp_async_wait_all();      // the queries: the only copies here, and in no group yet
            else async_wait<1>();
            __syncthreads();
            float x[RM][kKN];
            scores<D, RM>(sQ, sK, tr, tc, x);
            __syncthreads();
            if constexpr (CODES) codes.put(sV);
            if (it + 1 < g.n) begin(sK, P.ck, P.k_scale, g.kv.at(g.i0 + it + 1));
            else if (!CODES) async_commit();
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
            if constexpr (!CODES) async_wait<1>();
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
        if constexpr (!CODES) async_wait<0>();
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

template <int D, int BM, bool CAP, bool CODES> cudaError_t run_simt(const AttendParams& call, int num_sms, cudaStream_t stream)
{
    AttendParams P = call;
    P.tile_rows = BM;
    constexpr int smem = simt_smem<D, BM>();
    if (cudaError_t e = smem_opt_in<attend_simt_kernel<D, BM, CAP, CODES>>(smem); e != cudaSuccess) return e;
    const int grid = min(num_sms * ctas_per_sm<attend_simt_kernel<D, BM, CAP, CODES>>(smem, kThreads), kAttendMaxRows / BM / 2);
    attend_simt_kernel<D, BM, CAP, CODES><<<grid, kThreads, smem, stream>>>(P);
    if (cudaError_t e = cudaGetLastError(); e != cudaSuccess) return e;
    return run_join<float, D, BM>(P, grid, stream);
}

}  // namespace
}  // namespace kvx
