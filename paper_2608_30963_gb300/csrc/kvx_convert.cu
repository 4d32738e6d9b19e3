// kvx_convert.cu -- caches into 8 bits and back, and new tokens quantised as they are written.
//
//   quantise:    s = smallest scale with max |x| <= 448 * 2^(s - 127),  code = e4m3(x / 2^(s - 127))
//   dequantise:  x = code * 2^(s - 127)
//   append:      q' = R(p) q,  K[slot] = Q(R(p) k),  V[slot] = Q(v)
// Every element is read once and written once: the bound is memory (quantise 28 layers of 53385 slots of 2 heads of 128, 2.3 GB, in
// 348 us and read them back in 355: 6.6 and 6.5 TB/s, 97% of a copy's rate; append 9456 tokens of 36 heads of 128, 165 MB, in
// 30.6 us: 5.4 TB/s; short calls by their latency, 2.5 to 4 us).  A row's lanes hold 8 consecutive values of its first
// half and the 8 that lie half a head further on (append: the channels paired with them), so that every 16-byte load of
// neighbouring lanes is contiguous and the row's largest magnitude takes 2 to 4 exchanges.
#include "kvx_codes.cuh"
#include "kvx_tc_common.cuh"

namespace kvx {
namespace {

constexpr int kConvertThreads = 256, kAppendThreads = 128;

// Sixteen of a row's values as they came from memory: eight of its first half, eight of its second.
template <typename T> struct RowPart {
    uint4 w[sizeof(T)];                              // 16 bytes each
    __device__ __forceinline__ void load(const T* p, int half)
    {
        constexpr int N = 16 / (int)sizeof(T), M = (int)sizeof(T) / 2;
#pragma unroll
        for (int i = 0; i < M; ++i) {
            w[i] = __ldcs(reinterpret_cast<const uint4*>(p + i * N));
            w[M + i] = __ldcs(reinterpret_cast<const uint4*>(p + half + i * N));
        }
    }
    // values 8 half .. 8 half + 7
    __device__ __forceinline__ void get(int half, float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint4 v = sizeof(T) == 2 ? w[half] : w[half * 2 + i / 4];
            const int e = sizeof(T) == 2 ? i / 2 : i % 4;
            const uint32_t u = e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w;
            x[i] = sizeof(T) == 4 ? __uint_as_float(u) : __uint_as_float(i & 1 ? u & 0xffff0000u : u << 16);
        }
    }
};

// Each warp takes 32 rows of one (layer, K or V, sequence) at a time: its lanes find a row each, then all of them convert
// the rows, U at a time for each of the warp's 32 / LANES places.  The next 32 rows' pages are read before.  What is loaded stays
// packed until it is used: 64 registers, 32 warps an SM (with floats 115 registers and 604 us for 28 layers of 53385 slots of 2
// heads of 128).
template <typename T, int D, bool TO_CODES>
__global__ void __launch_bounds__(kConvertThreads, TO_CODES ? 4 : 3) convert_kernel(const __grid_constant__ ConvertParams P)
{
    constexpr int LANES = D / 16, ROWS = 32 / LANES, U = !TO_CODES ? 4 : sizeof(T) == 2 ? 2 : 1;
    extern __shared__ long long first[];             // groups of 32 rows before each sequence's
    const int tid = threadIdx.x, lane = tid & 31, sub = lane / LANES, c = lane % LANES * 8;
    const int most = min(P.full.capacity, P.codes.capacity);
    for (int b = tid; b < P.batch; b += kConvertThreads) first[b + 1] = ((long long)seq_slots(P.kv_len, most, b, P.status) * P.H + 31) / 32;
    if (tid == 0) first[0] = 0;
    __syncthreads();
    if (tid == 0)
        for (int b = 0; b < P.batch; ++b) first[b + 1] += first[b];
    __syncthreads();
    const long long groups = first[P.batch], total = groups * 2 * P.L, warps = (long long)gridDim.x * (kConvertThreads / 32);
    // a lane's row of group i: its slot (-1: none) and head, and the pages that hold it
    struct Row {
        int b, s, h, full, code;
    };
    auto page_of = [](const CacheView& C, int b, int s) {
        if (!C.paged) return 0;
        const int pi = C.page_shift >= 0 ? s >> C.page_shift : s / C.page_size;
        return pi < C.max_pages ? C.page_table[(size_t)b * C.max_pages + pi] : -1;
    };
    auto row_of = [&](long long i) {
        Row r = {0, -1, 0, -1, -1};
        if (i >= total) return r;
        const long long g = i % groups;
        int lo = 0, hi = P.batch - 1;                // the sequence of group g
        while (lo < hi) {
            const int m = (lo + hi + 1) >> 1;
            if (first[m] <= g) lo = m; else hi = m - 1;
        }
        const int n = min(max(P.kv_len[lo], 0), most);
        const long long k = (g - first[lo]) * 32 + lane;
        if (k >= (long long)n * P.H) return r;
        // rows in the order that the wider cache has them in
        r.b = lo;
        if (k >> 31) {
            r.s = (int)(P.full.paged ? k / P.H : k % n);
            r.h = (int)(P.full.paged ? k % P.H : k / n);
        } else {
            const unsigned by = (unsigned)(P.full.paged ? P.H : n), q = (unsigned)k / by, rest = (unsigned)k - q * by;
            r.s = (int)(P.full.paged ? q : rest);
            r.h = (int)(P.full.paged ? rest : q);
        }
        r.full = page_of(P.full, r.b, r.s);
        r.code = page_of(P.codes, r.b, r.s);
        return r;
    };
    auto place = [](const CacheView& C, int b, int s, int page, int& in) -> long long {
        if (!C.paged) return (long long)b * C.sb + (long long)s * C.st;
        if (page < 0 || page >= C.num_pages) return -1;
        in = C.page_shift >= 0 ? s & (C.page_size - 1) : s % C.page_size;
        return ((long long)page * C.page_size + in) * ((long long)C.H * D);
    };
    long long i = (long long)blockIdx.x * (kConvertThreads / 32) + (tid >> 5);
    Row next = row_of(i);
    for (; i < total; i += warps) {
        const Row r = next;
        next = row_of(i + warps);
        const long long unit = i / groups;
        const int l = (int)(unit >> 1);
        const bool key = !(unit & 1);
        long long full = -1, code = -1, scale = 0;
        if (r.s >= 0) {
            int in = 0;
            full = place(P.full, r.b, r.s, r.full, in);
            code = place(P.codes, r.b, r.s, r.code, in);
            if (full < 0 || code < 0) {
                set_status(P.status, KVX_DEV_PAGE_INVALID);
                full = code = -1;
            } else {
                full += cache_head(P.full) * r.h;
                code += cache_head(P.codes) * r.h;
                scale = (P.codes.paged ? (long long)r.code * P.H * P.codes.page_size + in : (long long)r.b * P.scales.sb + r.s) +
                        scale_head(P.codes, P.scales) * r.h;
            }
        }
        T* fp = (T*)(key ? P.full_k[l] : P.full_v[l]);
        uint8_t* cp = (uint8_t*)(key ? P.code_k[l] : P.code_v[l]);
        uint8_t* sp = key ? P.k_scale[l] : P.v_scale[l];
        unsigned mine = 0;                           // the lane's row's scale byte
        if (!TO_CODES && full >= 0) mine = sp[scale];
#pragma unroll 1
        for (int k0 = 0; k0 < 32; k0 += U * ROWS) {
            if constexpr (TO_CODES) {
                RowPart<T> x[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const long long f = __shfl_sync(0xffffffffu, full, k0 + u * ROWS + sub);
                    if (f >= 0) x[u].load(fp + f + c, D / 2);
                    else x[u] = {};
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const long long w = __shfl_sync(0xffffffffu, code, k0 + u * ROWS + sub);
                    float a[8], b[8];
                    x[u].get(0, a);
                    x[u].get(1, b);
                    uint2 lo, hi;
                    const unsigned s = quantise_row<LANES>(a, b, lo, hi), from = __shfl_sync(0xffffffffu, s, (lane - k0 - u * ROWS) * LANES & 31);
                    if (lane >= k0 + u * ROWS && lane < k0 + (u + 1) * ROWS) mine = from;
                    if (w >= 0) {
                        __stcs(reinterpret_cast<uint2*>(cp + w + c), lo);
                        __stcs(reinterpret_cast<uint2*>(cp + w + D / 2 + c), hi);
                    }
                }
            } else {
                uint2 x[U], y[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const long long w = __shfl_sync(0xffffffffu, code, k0 + u * ROWS + sub);
                    x[u] = y[u] = make_uint2(0u, 0u);
                    if (w >= 0) {
                        x[u] = __ldcs(reinterpret_cast<const uint2*>(cp + w + c));
                        y[u] = __ldcs(reinterpret_cast<const uint2*>(cp + w + D / 2 + c));
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const long long f = __shfl_sync(0xffffffffu, full, k0 + u * ROWS + sub);
                    const float z = scale_of(__shfl_sync(0xffffffffu, mine, k0 + u * ROWS + sub));
                    if (f >= 0) {
                        float a[8], e[8];
                        unpack_codes(x[u], z, a);
                        unpack_codes(y[u], z, e);
                        store8<T>(fp + f + c, a);
                        store8<T>(fp + f + D / 2 + c, e);
                    }
                }
            }
        }
        if (TO_CODES && full >= 0) sp[scale] = (uint8_t)mine;   // neighbouring slots' side by side
    }
}

// The slots of an 8-bit layer that a call's tokens see, as bf16 rows [batch][H][capacity][D] in the workspace: whole tiles of
// 128 slots, so that no tile of the attention that reads them holds what an earlier call left there.  Rows of pages that are
// not in the pool are zeros.
template <int D>
__global__ void __launch_bounds__(kConvertThreads) expand_kernel(const __grid_constant__ AttendParams P, __nv_bfloat16* to_k, __nv_bfloat16* to_v)
{
    // a warp's slots: as many as it has on their way at once
    constexpr int LANES = D / 16, ROWS = 32 / LANES, U = 4, GROUP = U * ROWS;
    extern __shared__ int4 ranges[];                 // slots [0, x) and [y, z) of a sequence; w: groups of slots before its first
    const int tid = threadIdx.x, lane = tid & 31, sub = lane / LANES, c = lane % LANES * 8;
    grid_dependency_wait();
    grid_launch_dependents();
    for (int b = tid; b < P.batch; b += kConvertThreads) {
        const Seq s = load_seq(P, b);
        const int L = s.n ? s.L : 0, a = min((s.pre + 127) / 128 * 128, L);
        ranges[b] = make_int4(a, max(max(window_lo(P, s.slot(0)), 0) / 128 * 128, a), L, 0);
    }
    __syncthreads();
    if (tid == 0) {
        int run = 0;
        for (int b = 0; b < P.batch; ++b) {
            ranges[b].w = run;
            run += (ranges[b].x + GROUP - 1) / GROUP + (max(ranges[b].z - ranges[b].y, 0) + GROUP - 1) / GROUP;
        }
        ranges[P.batch].w = run;
    }
    __syncthreads();
    const int groups = ranges[P.batch].w;            // (the workspace holds 2^18 slots)
    const int total = groups * 2 * P.H, warps = gridDim.x * (kConvertThreads / 32);
    for (int i = blockIdx.x * (kConvertThreads / 32) + (tid >> 5); i < total; i += warps) {
        // heads one after the other: a slot's lie side by side in a pool
        const int g = i / (2 * P.H), h = (i - g * 2 * P.H) >> 1;
        const bool key = !(i & 1);
        int lo = 0, hi = P.batch - 1;                // the sequence of group g
        while (lo < hi) {
            const int m = (lo + hi + 1) >> 1;
            if (ranges[m].w <= g) lo = m; else hi = m - 1;
        }
        const int b = lo;
        const int4 of = ranges[b];
        const int k = g - of.w, a = (of.x + GROUP - 1) / GROUP, s0 = k < a ? k * GROUP : of.y + (k - a) * GROUP, s = s0 + lane, L = of.z;
        long long code = -1;
        float scale = 0.0f;
        if (lane < GROUP && s < L) {
            const CodePlace at = code_place(P.cache, P.scales, b, s);
            if (at.row < 0) {
                set_status(P.status, KVX_DEV_PAGE_INVALID);
            } else {
                code = at.row + cache_head(P.cache) * h;
                scale = scale_of((key ? P.k_scale : P.v_scale)[at.scale + scale_head(P.cache, P.scales) * h]);
            }
        }
        const uint8_t* from = (const uint8_t*)(key ? P.ck : P.cv) + c;
        __nv_bfloat16* to = (key ? to_k : to_v) + (((long long)b * P.H + h) * P.cache.capacity + s0) * D + c;
        uint2 x[U], y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long w = __shfl_sync(0xffffffffu, code, u * ROWS + sub);
            x[u] = y[u] = make_uint2(0u, 0u);
            if (w >= 0) {
                x[u] = *reinterpret_cast<const uint2*>(from + w);
                y[u] = *reinterpret_cast<const uint2*>(from + w + D / 2);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = u * ROWS + sub;
            const float f = __shfl_sync(0xffffffffu, scale, r);
            if (s0 + r >= L) continue;
            float p[8], q[8];
            unpack_codes(x[u], f, p);
            unpack_codes(y[u], f, q);
            __nv_bfloat16* out = to + r * D;
            *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7]));
            *reinterpret_cast<uint4*>(out + D / 2) = make_uint4(pack_bf16(q[0], q[1]), pack_bf16(q[2], q[3]), pack_bf16(q[4], q[5]), pack_bf16(q[6], q[7]));
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
#pragma unroll 1
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
    constexpr int group = 4 * (512 / D);                 // (expand_kernel's)
    const long long groups = ((long long)P.cache.capacity + 2 * group - 1) / group * P.batch * P.H * 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)min((groups + kConvertThreads / 32 - 1) / (kConvertThreads / 32), (long long)num_sms * 8));
    cfg.blockDim = dim3(kConvertThreads);
    cfg.dynamicSmemBytes = (P.batch + 1) * sizeof(int4);
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
    // a block's heads share the sines: several, while that keeps the device full of blocks (9456 tokens of 36 heads of 128: 36.3,
    // 30.6 and 34.8 us with up to 2, 4 and 9 heads a block)
    int per = (int)(blocks * all / 2048);
    per = per < 1 ? 1 : per > 4 ? 4 : per;
    const dim3 grid((unsigned)blocks, (unsigned)((all + per - 1) / per));
    return dtype == KVX_BF16 ? run_append<__nv_bfloat16>(P, grid, per, stream) : run_append<float>(P, grid, per, stream);
}

}  // namespace kvx
