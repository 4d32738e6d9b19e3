// kvx_attend_rows.cuh -- the end of an attention row, shared by the attention kernels (library-internal):
// joining the partial results of split rows, normalising, and the rows whose sums met a value
// that is not finite.
#pragma once

#include "kvx_codes.cuh"
#include "kvx_decode.cuh"
#include "kvx_tc_common.cuh"

namespace kvx {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// C consecutive elements of T (C * sizeof(T) a multiple of 4, at most 32 bytes) as floats.
template <typename T, int C> __device__ __forceinline__ void load_f32(const T* p, float (&x)[C])
{
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] = to_f32<T>(p[i]);
}

template <typename T, int C> __device__ __forceinline__ void store_f32(T* p, const float (&x)[C])
{
    constexpr int B = C * (int)sizeof(T) < 16 ? C * (int)sizeof(T) : 16, N = B / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < C; i += N) {
        alignas(16) T v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = from_f32<T>(x[i + e]);
        if constexpr (B == 16) *reinterpret_cast<uint4*>(p + i) = *reinterpret_cast<const uint4*>(v);
        else if constexpr (B == 8) *reinterpret_cast<uint2*>(p + i) = *reinterpret_cast<const uint2*>(v);
        else *reinterpret_cast<uint32_t*>(p + i) = *reinterpret_cast<const uint32_t*>(v);
    }
}

// C consecutive codes of an 8-bit row (C a multiple of 2) as floats.
template <int C> __device__ __forceinline__ void load_codes(const uint8_t* p, float scale, float (&x)[C])
{
#pragma unroll
    for (int i = 0; i < C; i += 2) {
        const float2 f = codes_f32(*reinterpret_cast<const unsigned short*>(p + i));
        x[i] = f.x * scale;
        x[i + 1] = f.y * scale;
    }
}

// One row of a tile: its token and query head.
struct RowId {
    int t, head;
};
__device__ __forceinline__ RowId row_id(const AttendParams& P, const Seq& s, int h, int row)
{
    RowId r;
    r.t = row / P.G;
    r.head = h * P.G + (row - r.t * P.G);
    return r;
}

// The output of one row taken again slot by slot, by one warp, lane holding channels [lane * C, lane * C + C).
// The tiled sums multiply hidden slots' rows by a weight of zero; where such a row holds an infinity
// or a NaN that gives a NaN, so a row that did not come out finite is summed over the slots it sees only.  (Not where
// its sum of weights is NaN: hidden scores never enter that, so a score that is seen is not finite, and every output is NaN.)
template <typename T, int D>
__device__ __noinline__ void resum_row(const AttendParams& P, const Seq& s, int b, int h, int row, float lse2,
                                       float (&o)[D / 32], volatile int* beat = nullptr)
{
    constexpr int C = D / 32;
    const int lane = threadIdx.x & 31;
    const RowId id = row_id(P, s, h, row);
    float q[C], acc[C], x[C];
    load_f32<T, C>((const T*)P.q + (long long)(s.t0 + id.t) * P.q_t + (long long)id.head * P.q_h + lane * C, q);
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] = 0.0f;
    const int i = s.slot(id.t), hi = min(i + 1, s.L), lo = max(window_lo(P, i), 0);
    const float inv_cap = P.cap > 0.0f ? 1.0f / P.cap : 0.0f;
    for (int j = s.pre > 0 ? 0 : lo; j < max(hi, s.pre); ++j) {
        if (beat && (j & 4095) == 0 && lane == 0) *beat = *beat + 1;   // waits elsewhere in the CTA go on
        if (!sees(P, s, i, j)) continue;
        const CodePlace at = P.k_scale ? code_place(P.cache, P.scales, b, j) : CodePlace{cache_row(P.cache, b, j), 0};
        if (at.row < 0) continue;
        const long long off = at.row + cache_head(P.cache) * h + lane * C;
        const long long scale = at.scale + scale_head(P.cache, P.scales) * h;
        if (P.k_scale) load_codes<C>((const uint8_t*)P.ck + off, scale_of(P.k_scale[scale]), x);
        else load_f32<T, C>((const T*)P.ck + off, x);
        float dot = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) dot = fmaf(q[c], x[c], dot);
#pragma unroll
        for (int m = 16; m; m >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, m);
        float v = dot * P.scale;
        if (P.cap > 0.0f) v = capped(v, P.cap, inv_cap);
        const float p = exp2_hw(v * kLog2e - lse2);
        if (P.k_scale) load_codes<C>((const uint8_t*)P.cv + off, scale_of(P.v_scale[scale]), x);
        else load_f32<T, C>((const T*)P.cv + off, x);
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] = fmaf(p, x[c], acc[c]);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] = acc[c];
}

// Write one row from its unnormalised sums (lane holds C channels), its running maximum m (log2 units) and sum l; the
// row is row `row` of (sequence b, KV head h), its output that of packed token `token` and query head `head`.  Whole
// warps call it.
template <typename T, int D>
__device__ __forceinline__ void finish_row(const AttendParams& P, int b, int h, int row, int token, int head, float m, float l,
                                           float (&o)[D / 32])
{
    constexpr int C = D / 32;
    const int lane = threadIdx.x & 31;
    const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);   // nothing seen: zeros; NaN stays
    bool fine = true;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        o[c] *= inv;
        fine = fine && fabsf(o[c]) <= 3.0e38f;
    }
    const float lse2 = l == 0.0f ? -INFINITY : m + log2f(l);
    if (!__all_sync(0xffffffffu, fine)) {
        if (l == 0.0f) {
#pragma unroll
            for (int c = 0; c < C; ++c) o[c] = 0.0f;
        } else if (l == l) {
            resum_row<T, D>(P, load_seq(P, b), b, h, row, lse2, o);
        }
    }
    store_f32<T, C>((T*)P.out + (long long)token * P.o_t + (long long)head * P.o_h + lane * C, o);
    if (P.lse && lane == 0) P.lse[(long long)token * P.Hq + head] = lse2 * kLn2;
}

// C floats of a partial result.
template <int C> __device__ __forceinline__ void load_part(const float* src, float (&v)[C])
{
    if constexpr (C == 2) {
        const float2 x = __ldcg((const float2*)src);
        v[0] = x.x;
        v[1] = x.y;
    } else {
#pragma unroll
        for (int c = 0; c < C; c += 4) {
            const float4 x = __ldcg((const float4*)(src + c));
            v[c] = x.x;
            v[c + 1] = x.y;
            v[c + 2] = x.z;
            v[c + 3] = x.w;
        }
    }
}

// The last segment of a CTA's range: where an item begins that other CTAs go on with, this CTA leaves its
// description for the join, else an empty one.
__device__ __forceinline__ void leave_split(const AttendParams& P, const Plan& plan, const Segment& g, bool have)
{
    SplitItem it = {};
    if (have && g.i0 == 0 && !g.whole()) {
        const Parts parts = item_parts(plan, g);
        it = {g.b, g.rt, g.h, min(P.tile_rows, g.s.n * P.G - g.rt * P.tile_rows), g.s.t0 + g.rt * P.tile_rows / P.G,
              parts.parts, parts.slot0, parts.lines};
    }
    P.split[blockIdx.x] = it;
}

// Joins the partial results of split items: CTA (c, y) takes rows [y * RPC, ...) of the item that CTA c of the
// attention kernel left.  Bound by the latency of two reads from L2, the item's and the parts', so many of the
// latter are in flight at once: a warp takes RW rows and two parts of each at a time; where rows are few (and
// parts may be many), WPR warps a row, each with every WPR-th part, eight at a time, their sums added in order.
template <typename T, int D, int BM, int WPR>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ AttendParams P)
{
    constexpr int C = D / 32, RW = WPR > 1 ? 1 : C == 8 ? 2 : 4, RPC = 8 / WPR * RW, U = WPR > 1 ? (C == 8 ? 4 : 8) : 2;
    __shared__ float sh[8][D + 2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_launch_dependents();
    grid_dependency_wait();
    const SplitItem it = P.split[blockIdx.x];
    const int r0 = blockIdx.y * RPC + warp / WPR * RW, w0 = warp % WPR;
    if (r0 - warp / WPR * RW >= it.rows || it.parts == 0) return;      // the whole CTA
    const Parts parts = {(int)blockIdx.x, it.lines, it.parts, it.slot0};
    // running maximum, sum and channels of the rows over the parts so far
    float m[RW], l[RW], o[RW][C];
#pragma unroll
    for (int k = 0; k < RW; ++k) {
        m[k] = -INFINITY;
        l[k] = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) o[k][c] = 0.0f;
    }
    for (int i0 = w0; i0 < it.parts; i0 += U * WPR) {
        float2 ml[U][RW];
        float v[U][RW][C];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < RW; ++k) {
                ml[u][k] = make_float2(-INFINITY, 0.0f);
                if (i0 + u * WPR < it.parts && r0 + k < it.rows) {
                    const size_t at = (size_t)parts.slot(i0 + u * WPR) * BM + r0 + k;
                    ml[u][k] = __ldcg(&P.part_ml[at]);
                    load_part<C>(P.part_o + at * D + lane * C, v[u][k]);
                }
            }
#pragma unroll
        for (int k = 0; k < RW; ++k) {
            float top = m[k];
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, ml[u][k].x);
            const float base = top == -INFINITY ? 0.0f : top, w = exp2_hw(m[k] - base);
            m[k] = top;
            l[k] *= w;
#pragma unroll
            for (int c = 0; c < C; ++c) o[k][c] *= w;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u * WPR < it.parts && r0 + k < it.rows) {
                    const float e = exp2_hw(ml[u][k].x - base);
                    l[k] = fmaf(ml[u][k].y, e, l[k]);
#pragma unroll
                    for (int c = 0; c < C; ++c) o[k][c] = fmaf(v[u][k][c], e, o[k][c]);
                }
        }
    }
    if constexpr (WPR > 1) {
#pragma unroll
        for (int c = 0; c < C; ++c) sh[warp][lane * C + c] = o[0][c];
        if (lane == 0) {
            sh[warp][D] = m[0];
            sh[warp][D + 1] = l[0];
        }
        __syncthreads();
        if (w0 != 0) return;
        float top = m[0];
#pragma unroll
        for (int k = 1; k < WPR; ++k) top = fmaxf(top, sh[warp + k][D]);
        const float base = top == -INFINITY ? 0.0f : top, w = exp2_hw(m[0] - base);
        m[0] = top;
        l[0] *= w;
#pragma unroll
        for (int c = 0; c < C; ++c) o[0][c] *= w;
#pragma unroll
        for (int k = 1; k < WPR; ++k) {
            const float e = exp2_hw(sh[warp + k][D] - base);
            l[0] = fmaf(sh[warp + k][D + 1], e, l[0]);
#pragma unroll
            for (int c = 0; c < C; ++c) o[0][c] = fmaf(sh[warp + k][lane * C + c], e, o[0][c]);
        }
    }
#pragma unroll
    for (int k = 0; k < RW; ++k)
        if (r0 + k < it.rows) {
            // (a tile that begins inside a token has its first row's head in it)
            const int row = it.rt * P.tile_rows + r0 + k, t = row / P.G, t_first = it.rt * P.tile_rows / P.G;
            finish_row<T, D>(P, it.b, it.h, row, it.token + t - t_first, it.h * P.G + (row - t * P.G), m[k], l[k], o[k]);
        }
}
template <typename T, int D, int BM> cudaError_t run_join(const AttendParams& P, int grid, cudaStream_t stream)
{
    // An item has at most min(tile_rows, T G) rows; few in the whole call: four warps a row, as it may have many parts (16384
    // slots, 7 rows a KV head 29 us so and 54 with one warp, 63 rows 35 and 54; 16 sequences of 8192 slots, 112 rows in all
    // 82.6 and 76.5)
    const long long rows = min((long long)P.tile_rows, (long long)P.T * P.G);
    const bool few = (long long)P.T * P.G <= 64;
    const int rpc = few ? 2 : 8 * (D == 256 ? 2 : 4);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid, (unsigned)((rows + rpc - 1) / rpc));
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return few ? cudaLaunchKernelEx(&cfg, join_kernel<T, D, BM, 4>, P) : cudaLaunchKernelEx(&cfg, join_kernel<T, D, BM, 1>, P);
}

}  // namespace
}  // namespace kvx
