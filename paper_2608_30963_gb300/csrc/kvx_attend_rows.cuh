// kvx_attend_rows.cuh -- the end of an attention row, shared by the attention kernels (library-internal):
// joining the partial results of split rows, normalising, and the rows whose sums met a value
// that is not finite.
#pragma once

#include "kvx_decode.cuh"

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
// or a NaN that gives a NaN, so a row that did not come out finite is summed over the slots it sees only.
template <typename T, int D>
__device__ __noinline__ void resum_row(const AttendParams& P, const Seq& s, int b, int h, int row, float lse2,
                                       float (&o)[D / 32])
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
        if (!sees(P, s, i, j)) continue;
        const long long at = cache_row(P.cache, b, j);
        if (at < 0) continue;
        const long long off = at + cache_head(P.cache) * h + lane * C;
        load_f32<T, C>((const T*)P.ck + off, x);
        float dot = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) dot = fmaf(q[c], x[c], dot);
#pragma unroll
        for (int m = 16; m; m >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, m);
        float v = dot * P.scale;
        if (P.cap > 0.0f) v = capped(v, P.cap, inv_cap);
        const float p = exp2_hw(v * kLog2e - lse2);
        load_f32<T, C>((const T*)P.cv + off, x);
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] = fmaf(p, x[c], acc[c]);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] = acc[c];
}

// Write one row from its unnormalised sums (lane holds C channels), its running maximum m (log2 units) and sum l.
// Whole warps call it.
template <typename T, int D>
__device__ __forceinline__ void finish_row(const AttendParams& P, const Seq& s, int b, int h, int row, float m, float l,
                                           float (&o)[D / 32])
{
    constexpr int C = D / 32;
    const int lane = threadIdx.x & 31;
    const RowId id = row_id(P, s, h, row);
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
        } else {
            resum_row<T, D>(P, s, b, h, row, lse2, o);
        }
    }
    T* out = (T*)P.out + (long long)(s.t0 + id.t) * P.o_t + (long long)id.head * P.o_h + lane * C;
    store_f32<T, C>(out, o);
    if (P.lse && lane == 0) P.lse[(long long)(s.t0 + id.t) * P.Hq + id.head] = lse2 * kLn2;
}

// Join the partial results of a split item, rows [0, rows) of its tile; WARPS warps call it, numbered from 0.
template <typename T, int D, int BM, int WARPS>
__device__ __forceinline__ void join_parts(const AttendParams& P, const Segment& g, const Parts& parts, int rows, int warp)
{
    constexpr int C = D / 32;
    const int lane = threadIdx.x & 31;
    for (int r = warp; r < rows; r += WARPS) {
        float m = -INFINITY;
        for (int i = lane; i < parts.parts; i += 32) m = fmaxf(m, __ldcg(&P.part_ml[(size_t)parts.slot(i) * BM + r]).x);
#pragma unroll
        for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
        const float base = m == -INFINITY ? 0.0f : m;
        float l = 0.0f, o[C];
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] = 0.0f;
#pragma unroll 4
        for (int i = 0; i < parts.parts; ++i) {
            const size_t at = (size_t)parts.slot(i) * BM + r;
            const float2 ml = __ldcg(&P.part_ml[at]);
            const float w = exp2_hw(ml.x - base);
            l = fmaf(ml.y, w, l);
            const float* src = P.part_o + at * D + lane * C;
            if constexpr (C == 2) {
                const float2 v = __ldcg((const float2*)src);
                o[0] = fmaf(v.x, w, o[0]);
                o[1] = fmaf(v.y, w, o[1]);
            } else {
#pragma unroll
                for (int c = 0; c < C; c += 4) {
                    const float4 v = __ldcg((const float4*)(src + c));
                    o[c] = fmaf(v.x, w, o[c]);
                    o[c + 1] = fmaf(v.y, w, o[c + 1]);
                    o[c + 2] = fmaf(v.z, w, o[c + 2]);
                    o[c + 3] = fmaf(v.w, w, o[c + 3]);
                }
            }
        }
        finish_row<T, D>(P, g.s, g.b, g.h, g.rt * BM + r, m, l, o);
    }
}

// After a CTA has written its partial result: whether it is the last of the item's CTAs (all threads get the
// answer).  The counter goes back to zero for the next launch.
__device__ __forceinline__ bool last_to_arrive(const AttendParams& P, const Parts& parts, int* flag)
{
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        const unsigned before = atomicAdd(&P.arrived[parts.c0], 1u);
        *flag = before == (unsigned)parts.parts - 1;
        if (*flag) P.arrived[parts.c0] = 0;
        __threadfence();
    }
    __syncthreads();
    return *flag;
}

}  // namespace
}  // namespace kvx
