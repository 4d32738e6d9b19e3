// kvx_append.cu -- new tokens' queries and keys rotated, their keys and values written into the cache.
//
//   q'_i = R(p_i) q_i,  K[s_i] = R(p_i) k_i,  V[s_i] = v_i
// Every element is read once and written once: the bound is memory (171 MB in 32.8 us: 5.2 TB/s, 77% of a copy's
// rate).  A thread takes one 16-byte chunk
// of a token's head and the chunk it is paired with, for several heads: the angles of the pairs are
// the same in every head, so their sines are taken once.
#include "kvx_decode.cuh"

namespace kvx {
namespace {

constexpr int kAppendThreads = 128;

template <typename T> struct Chunk {
    static constexpr int N = 16 / (int)sizeof(T);
    float x[N];
};
template <typename T> __device__ __forceinline__ Chunk<T> load_chunk(const T* p)
{
    Chunk<T> c;
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
    for (int i = 0; i < Chunk<T>::N; ++i) c.x[i] = to_f32<T>(e[i]);
    return c;
}
template <typename T> __device__ __forceinline__ void store_chunk(T* p, const Chunk<T>& c)
{
    uint4 w;
    T* e = reinterpret_cast<T*>(&w);
#pragma unroll
    for (int i = 0; i < Chunk<T>::N; ++i) e[i] = from_f32<T>(c.x[i]);
    *reinterpret_cast<uint4*>(p) = w;
}

// heads: query heads, then K heads, then V heads; blockIdx.y takes `per` of them.
template <typename T>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const __grid_constant__ AppendParams P, int per)
{
    constexpr int N = Chunk<T>::N;
    const int chunks = P.d / 2 / N;
    const long long item = (long long)blockIdx.x * kAppendThreads + threadIdx.x;
    const int t = (int)(item / chunks);
    if (t >= P.T) return;
    const int slot = (int)(item - (long long)t * chunks) * N;   // first pair slot of the chunk
    const int b = find_seq(P.seq_off, P.batch, t);
    const int n = __ldg(&P.seq_off[b + 1]), L = __ldg(&P.kv_len[b]);
    const int s = L - (n - t);                                  // the token's slot
    const int all = P.Hq + 2 * P.H, h0 = blockIdx.y * per, h1 = min(all, h0 + per);
    long long row = -1;
    if (h1 > P.Hq) {
        if (s < 0 || s >= P.cache.capacity) {
            set_status(P.status, KVX_DEV_SEQ_CLAMPED);
        } else {
            row = cache_row(P.cache, b, s);
            if (row < 0) set_status(P.status, KVX_DEV_PAGE_INVALID);
        }
    }
    int lo, hi;
    pair_channels(slot, P.d / 2, P.rhalf, lo, hi);
    const bool turns = P.rope && slot < P.rhalf;
    float2 cs[N];
    if (turns && h0 < P.Hq + P.H) {
        const int p = clamp_pos(P.pos ? __ldg(&P.pos[t]) : s, P.max_position, P.status);
#pragma unroll
        for (int i = 0; i < N; ++i) cs[i] = turn_cs(__ldg(&P.turns[slot + i]), p);
    }
#pragma unroll 4
    for (int h = h0; h < h1; ++h) {
        const T* src;
        T* dst;
        if (h < P.Hq) {
            src = (const T*)P.q + (long long)t * P.q_t + (long long)h * P.q_h;
            dst = (T*)P.q_out + (long long)t * P.o_t + (long long)h * P.o_h;
        } else {
            if (row < 0) break;
            const int g = h - P.Hq < P.H ? h - P.Hq : h - P.Hq - P.H;
            const bool key = h - P.Hq < P.H;
            src = key ? (const T*)P.k + (long long)t * P.k_t + (long long)g * P.k_h
                      : (const T*)P.v + (long long)t * P.v_t + (long long)g * P.v_h;
            dst = (T*)(key ? P.ck : P.cv) + row + cache_head(P.cache) * g;
        }
        if (h < P.Hq + P.H && turns) {
            const Chunk<T> a = load_chunk<T>(src + lo), c = load_chunk<T>(src + hi);
            Chunk<T> x, y;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x.x[i] = fmaf(a.x[i], cs[i].x, -c.x[i] * cs[i].y);
                y.x[i] = fmaf(c.x[i], cs[i].x, a.x[i] * cs[i].y);
            }
            store_chunk<T>(dst + lo, x);
            store_chunk<T>(dst + hi, y);
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(src + lo), c = *reinterpret_cast<const uint4*>(src + hi);
            *reinterpret_cast<uint4*>(dst + lo) = a;
            *reinterpret_cast<uint4*>(dst + hi) = c;
        }
    }
}

}  // namespace

cudaError_t launch_append(const AppendParams& P, int dtype, cudaStream_t stream)
{
    if (P.T == 0) return cudaSuccess;
    const int chunks = P.d / 2 / (dtype == KVX_BF16 ? 8 : 4), all = P.Hq + 2 * P.H;
    const long long items = (long long)P.T * chunks;
    // a block's heads: they share the sines, so several, while that keeps the device full of blocks (10797 tokens of 36
    // heads of 128: 34.8, 32.8 and 34.9 us with up to 2, 4 and 12 heads a block)
    const long long blocks = (items + kAppendThreads - 1) / kAppendThreads;
    int per = (int)(blocks * all / 2048);
    per = per < 1 ? 1 : per > 4 ? 4 : per;
    const dim3 grid((unsigned)blocks, (unsigned)((all + per - 1) / per));
    if (dtype == KVX_BF16) append_kernel<__nv_bfloat16><<<grid, kAppendThreads, 0, stream>>>(P, per);
    else append_kernel<float><<<grid, kAppendThreads, 0, stream>>>(P, per);
    return cudaGetLastError();
}

}  // namespace kvx
