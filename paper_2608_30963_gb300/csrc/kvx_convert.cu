// kvx_convert.cu -- caches into 8 bits and back, and new tokens quantised as they are written.
//
//   quantise:    s = smallest scale with max |x| <= 448 * 2^(s - 127),  code = e4m3(x / 2^(s - 127))
//   dequantise:  x = code * 2^(s - 127)
//   append:      q' = R(p) q,  K[slot] = Q(R(p) k),  V[slot] = Q(v)
// Every element is read once and written once: the bound is memory.  A row's lanes hold 8 consecutive values of its first
// half and the 8 that lie half a head further on (append: the channels paired with them), so that every 16-byte load of
// neighbouring lanes is contiguous and the row's largest magnitude takes 2 to 4 exchanges.
#include "kvx_codes.cuh"
#include "kvx_tc_common.cuh"

namespace kvx {
namespace {

constexpr int kConvertThreads = 256, kAppendThreads = 128;

// Each warp takes 32 rows of one (layer, K or V, sequence) at a time: its lanes find a row each, then all of them convert
// the rows, U at a time for each of the warp's 32 / LANES places.
template <typename T, int D, bool TO_CODES>
__global__ void __launch_bounds__(kConvertThreads) convert_kernel(const __grid_constant__ ConvertParams P)
{
    constexpr int LANES = D / 16, ROWS = 32 / LANES, U = sizeof(T) == 2 ? 4 : 2;
    extern __shared__ long long first[];             // groups of 32 rows before each sequence's
    const int tid = threadIdx.x, lane = tid & 31, sub = lane / LANES, c = lane % LANES * 8;
    for (int b = tid; b < P.batch; b += kConvertThreads) {
        const int most = min(P.full.capacity, P.codes.capacity), n = seq_slots(P.kv_len, most, b, P.status);
        first[b + 1] = ((long long)n * P.H + 31) / 32;
    }
    if (tid == 0) first[0] = 0;
    __syncthreads();
    if (tid == 0)
        for (int b = 0; b < P.batch; ++b) first[b + 1] += first[b];
    __syncthreads();
    const long long groups = first[P.batch], total = groups * 2 * P.L, warps = (long long)gridDim.x * (kConvertThreads / 32);
    for (long long i = (long long)blockIdx.x * (kConvertThreads / 32) + (tid >> 5); i < total; i += warps) {
        const long long unit = i / groups, g = i - unit * groups;
        const int l = (int)(unit >> 1);
        const bool key = !(unit & 1);
        int lo = 0, hi = P.batch - 1;                // the sequence of group g
        while (lo < hi) {
            const int m = (lo + hi + 1) >> 1;
            if (first[m] <= g) lo = m; else hi = m - 1;
        }
        const int b = lo, n = min(max(P.kv_len[b], 0), min(P.full.capacity, P.codes.capacity));
        // rows in the order that the wider cache has them in
        const long long r = (g - first[b]) * 32 + lane;
        long long full = -1, code = -1, scale = 0;
        if (r < (long long)n * P.H) {
            const int s = P.full.paged ? (int)(r / P.H) : (int)(r % n), h = P.full.paged ? (int)(r % P.H) : (int)(r / n);
            full = cache_row(P.full, b, s);
            const CodePlace at = code_place(P.codes, P.scales, b, s);
            code = at.row;
            if (full < 0 || code < 0) {
                set_status(P.status, KVX_DEV_PAGE_INVALID);
                full = code = -1;
            } else {
                full += cache_head(P.full) * h;
                code += cache_head(P.codes) * h;
                scale = at.scale + scale_head(P.codes, P.scales) * h;
            }
        }
        T* fp = (T*)(key ? P.full_k[l] : P.full_v[l]);
        uint8_t* cp = (uint8_t*)(key ? P.code_k[l] : P.code_v[l]);
        uint8_t* sp = key ? P.k_scale[l] : P.v_scale[l];
#pragma unroll 1
        for (int k0 = 0; k0 < 32; k0 += U * ROWS) {
            long long f[U], w[U], z[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                f[u] = __shfl_sync(0xffffffffu, full, k0 + u * ROWS + sub);
                w[u] = __shfl_sync(0xffffffffu, code, k0 + u * ROWS + sub);
                z[u] = __shfl_sync(0xffffffffu, scale, k0 + u * ROWS + sub);
            }
            if constexpr (TO_CODES) {
                float a[U][8], e[U][8];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (f[u] >= 0) {
                        load8<T>(fp + f[u] + c, a[u]);
                        load8<T>(fp + f[u] + D / 2 + c, e[u]);
                    } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k) a[u][k] = e[u][k] = 0.0f;
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    uint2 x, y;
                    const unsigned s = quantise_row<LANES>(a[u], e[u], x, y);
                    if (w[u] >= 0) {
                        __stcs(reinterpret_cast<uint2*>(cp + w[u] + c), x);
                        __stcs(reinterpret_cast<uint2*>(cp + w[u] + D / 2 + c), y);
                        if (c == 0) sp[z[u]] = (uint8_t)s;
                    }
                }
            } else {
                uint2 x[U], y[U];
                unsigned s[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (w[u] >= 0) {
                        x[u] = __ldcs(reinterpret_cast<const uint2*>(cp + w[u] + c));
                        y[u] = __ldcs(reinterpret_cast<const uint2*>(cp + w[u] + D / 2 + c));
                        s[u] = sp[z[u]];
                    }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (f[u] >= 0) {
                        float a[8], e[8];
                        unpack_codes(x[u], scale_of(s[u]), a);
                        unpack_codes(y[u], scale_of(s[u]), e);
                        store8<T>(fp + f[u] + c, a);
                        store8<T>(fp + f[u] + D / 2 + c, e);
                    }
            }
        }
    }
}

// The slots of an 8-bit layer that a call's tokens see, as bf16 rows [batch][H][capacity][D] in the workspace: whole tiles of
// 128 slots, so that no tile of the attention that reads them holds what an earlier call left there.  Rows of pages that are
// not in the pool are zeros.
template <int D>
__global__ void __launch_bounds__(kConvertThreads) expand_kernel(const __grid_constant__ AttendParams P, __nv_bfloat16* to_k, __nv_bfloat16* to_v)
{
    constexpr int LANES = D / 16, ROWS = 32 / LANES, U = 4;
    extern __shared__ long long first[];             // groups of 32 slots before each sequence's
    const int tid = threadIdx.x, lane = tid & 31, sub = lane / LANES, c = lane % LANES * 8;
    grid_dependency_wait();
    grid_launch_dependents();
    // slots [0, a) and [z, L) of a sequence, in tiles
    auto range = [&](int b, int& a, int& z, int& L) {
        const Seq s = load_seq(P, b);
        L = s.L;
        a = min((s.pre + 127) / 128 * 128, L);
        z = max(max(window_lo(P, s.slot(0)), 0) / 128 * 128, a);
        if (s.n == 0) a = z = L = 0;
    };
    for (int b = tid; b < P.batch; b += kConvertThreads) {
        int a, z, L;
        range(b, a, z, L);
        first[b + 1] = (a + 31) / 32 + (max(L - z, 0) + 31) / 32;
    }
    if (tid == 0) first[0] = 0;
    __syncthreads();
    if (tid == 0)
        for (int b = 0; b < P.batch; ++b) first[b + 1] += first[b];
    __syncthreads();
    const long long groups = first[P.batch], total = groups * 2 * P.H, warps = (long long)gridDim.x * (kConvertThreads / 32);
    for (long long i = (long long)blockIdx.x * (kConvertThreads / 32) + (tid >> 5); i < total; i += warps) {
        // heads one after the other: a token's lie side by side in a pool
        const long long g = i / (2 * P.H);
        const int hk = (int)(i - g * (2 * P.H)), h = hk >> 1;
        const bool key = !(hk & 1);
        int lo = 0, hi = P.batch - 1;                // the sequence of group g
        while (lo < hi) {
            const int m = (lo + hi + 1) >> 1;
            if (first[m] <= g) lo = m; else hi = m - 1;
        }
        const int b = lo;
        int a, z, L;
        range(b, a, z, L);
        const int k = (int)(g - first[b]), s0 = k < (a + 31) / 32 ? k * 32 : z + (k - (a + 31) / 32) * 32, s = s0 + lane;
        long long code = -1;
        float scale = 0.0f;
        if (s < L) {
            const CodePlace at = code_place(P.cache, P.scales, b, s);
            if (at.row < 0) {
                set_status(P.status, KVX_DEV_PAGE_INVALID);
            } else {
                code = at.row + cache_head(P.cache) * h;
                scale = scale_of((key ? P.k_scale : P.v_scale)[at.scale + scale_head(P.cache, P.scales) * h]);
            }
        }
        const uint8_t* cp = (const uint8_t*)(key ? P.ck : P.cv);
        __nv_bfloat16* out = (key ? to_k : to_v) + (((long long)b * P.H + h) * P.cache.capacity + s0) * D;
#pragma unroll 1
        for (int k0 = 0; k0 < 32; k0 += U * ROWS) {
            uint2 x[U], y[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long long w = __shfl_sync(0xffffffffu, code, k0 + u * ROWS + sub);
                x[u] = y[u] = make_uint2(0u, 0u);
                if (w >= 0) {
                    x[u] = *reinterpret_cast<const uint2*>(cp + w + c);
                    y[u] = *reinterpret_cast<const uint2*>(cp + w + D / 2 + c);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int r = k0 + u * ROWS + sub;
                const float f = __shfl_sync(0xffffffffu, scale, r);
                if (s0 + r < L) {
                    float p[8], q[8];
                    unpack_codes(x[u], f, p);
                    unpack_codes(y[u], f, q);
                    uint4 v;
                    v = make_uint4(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7]));
                    *reinterpret_cast<uint4*>(out + (long long)r * D + c) = v;
                    v = make_uint4(pack_bf16(q[0], q[1]), pack_bf16(q[2], q[3]), pack_bf16(q[4], q[5]), pack_bf16(q[6], q[7]));
                    *reinterpret_cast<uint4*>(out + (long long)r * D + D / 2 + c) = v;
                }
            }
        }
    }
}

// heads: query heads, then K heads, then V heads; blockIdx.y takes `per` of them.  A thread has one chunk of 8 channels of a
// token's heads and the chunk paired with it, whose sines are taken once.
template <typename T, int D>
__global__ void __launch_bounds__(kAppendThreads) append_codes_kernel(const __grid_constant__ AppendParams P, int per)
{
    constexpr int LANES = D / 16;
    const long long item = (long long)blockIdx.x * kAppendThreads + threadIdx.x;
    const bool live = item / LANES < P.T;                       // (rows past the last go on, so that whole warps exchange)
    const int t = live ? (int)(item / LANES) : P.T - 1, slot = (int)(item % LANES) * 8;
    const int b = find_seq(P.seq_off, P.batch, t);
    const int s = P.kv_len[b] - (P.seq_off[b + 1] - t);         // the token's slot
    const int all = P.Hq + 2 * P.H, h0 = blockIdx.y * per, h1 = min(all, h0 + per);
    CodePlace at = {-1, -1};
    if (h1 > P.Hq) {
        if (s < 0 || s >= P.cache.capacity) {
            set_status(P.status, KVX_DEV_SEQ_CLAMPED);
        } else {
            at = code_place(P.cache, P.scales, b, s);
            if (at.row < 0) set_status(P.status, KVX_DEV_PAGE_INVALID);
        }
    }
    int lo, hi;
    pair_channels(slot, D / 2, P.rhalf, lo, hi);
    const bool turns = P.rope && slot < P.rhalf;
    float2 cs[8];
    if (turns && h0 < P.Hq + P.H) {
        const int p = clamp_pos(P.pos ? P.pos[t] : s, P.max_position, P.status);
#pragma unroll
        for (int i = 0; i < 8; ++i) cs[i] = turn_cs(__ldg(&P.turns[slot + i]), p);
    }
#pragma unroll 2
    for (int h = h0; h < h1; ++h) {
        const int g = h < P.Hq ? h : h - P.Hq < P.H ? h - P.Hq : h - P.Hq - P.H;
        const bool key = h < P.Hq + P.H;
        const T* src = h < P.Hq ? (const T*)P.q + (long long)t * P.q_t + (long long)g * P.q_h
                       : key    ? (const T*)P.k + (long long)t * P.k_t + (long long)g * P.k_h
                                : (const T*)P.v + (long long)t * P.v_t + (long long)g * P.v_h;
        float a[8], c[8];
        load8<T>(src + lo, a);
        load8<T>(src + hi, c);
        if (key && turns) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = fmaf(a[i], cs[i].x, -c[i] * cs[i].y);
                c[i] = fmaf(c[i], cs[i].x, a[i] * cs[i].y);
                a[i] = x;
            }
        }
        if (h < P.Hq) {
            if (!live) continue;
            T* dst = (T*)P.q_out + (long long)t * P.o_t + (long long)g * P.o_h;
            store8<T>(dst + lo, a);
            store8<T>(dst + hi, c);
        } else {
            uint2 x, y;
            const unsigned z = quantise_row<LANES>(a, c, x, y);
            if (!live || at.row < 0) continue;
            uint8_t* dst = (uint8_t*)(key ? P.ck : P.cv) + at.row + cache_head(P.cache) * g;
            *reinterpret_cast<uint2*>(dst + lo) = x;
            *reinterpret_cast<uint2*>(dst + hi) = y;
            if (slot == 0) (key ? P.k_scale : P.v_scale)[at.scale + scale_head(P.cache, P.scales) * g] = (uint8_t)z;
        }
    }
}

template <typename T, int D, bool TO_CODES> cudaError_t run_convert(const ConvertParams& P, int num_sms, cudaStream_t stream)
{
    const long long groups = ((long long)min(P.full.capacity, P.codes.capacity) * P.H + 31) / 32 * P.batch * P.L * 2;
    const int grid = (int)min((groups + kConvertThreads / 32 - 1) / (kConvertThreads / 32), (long long)num_sms * 8);
    if (grid == 0) return cudaSuccess;
    convert_kernel<T, D, TO_CODES><<<grid, kConvertThreads, (P.batch + 1) * sizeof(long long), stream>>>(P);
    return cudaGetLastError();
}
template <typename T, bool TO_CODES> cudaError_t run_convert(const ConvertParams& P, int num_sms, cudaStream_t stream)
{
    return P.d == 64 ? run_convert<T, 64, TO_CODES>(P, num_sms, stream) : P.d == 128 ? run_convert<T, 128, TO_CODES>(P, num_sms, stream)
                                                                                     : run_convert<T, 256, TO_CODES>(P, num_sms, stream);
}
template <int D> cudaError_t run_expand(const AttendParams& P, void* to_k, void* to_v, int num_sms, cudaStream_t stream)
{
    const long long groups = ((long long)P.cache.capacity + 63) / 32 * P.batch * P.H * 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)min((groups + kConvertThreads / 32 - 1) / (kConvertThreads / 32), (long long)num_sms * 8));
    cfg.blockDim = dim3(kConvertThreads);
    cfg.dynamicSmemBytes = (P.batch + 1) * sizeof(long long);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, expand_kernel<D>, P, (__nv_bfloat16*)to_k, (__nv_bfloat16*)to_v);
}
template <typename T> cudaError_t run_append(const AppendParams& P, dim3 grid, int per, cudaStream_t stream)
{
    if (P.d == 64) append_codes_kernel<T, 64><<<grid, kAppendThreads, 0, stream>>>(P, per);
    else if (P.d == 128) append_codes_kernel<T, 128><<<grid, kAppendThreads, 0, stream>>>(P, per);
    else append_codes_kernel<T, 256><<<grid, kAppendThreads, 0, stream>>>(P, per);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_convert(const ConvertParams& P, bool to_codes, int dtype, int num_sms, cudaStream_t stream)
{
    if (dtype == KVX_BF16) return to_codes ? run_convert<__nv_bfloat16, true>(P, num_sms, stream) : run_convert<__nv_bfloat16, false>(P, num_sms, stream);
    return to_codes ? run_convert<float, true>(P, num_sms, stream) : run_convert<float, false>(P, num_sms, stream);
}

cudaError_t launch_expand(const AttendParams& P, void* to_k, void* to_v, int num_sms, cudaStream_t stream)
{
    return P.d == 64 ? run_expand<64>(P, to_k, to_v, num_sms, stream) : P.d == 128 ? run_expand<128>(P, to_k, to_v, num_sms, stream)
                                                                               : run_expand<256>(P, to_k, to_v, num_sms, stream);
}

cudaError_t launch_append_codes(const AppendParams& P, int dtype, cudaStream_t stream)
{
    const int all = P.Hq + 2 * P.H;
    const long long blocks = ((long long)P.T * (P.d / 16) + kAppendThreads - 1) / kAppendThreads;
    // a block's heads share the sines: several, while that keeps the device full of blocks
    int per = (int)(blocks * all / 2048);
    per = per < 1 ? 1 : per > 4 ? 4 : per;
    const dim3 grid((unsigned)blocks, (unsigned)((all + per - 1) / per));
    return dtype == KVX_BF16 ? run_append<__nv_bfloat16>(P, grid, per, stream) : run_append<float>(P, grid, per, stream);
}

}  // namespace kvx
