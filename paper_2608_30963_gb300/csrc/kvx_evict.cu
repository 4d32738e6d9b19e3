// kvx_evict.cu -- a cache cut down to the slots of the largest accumulated attention weight.
//
// Two launches.  select_kernel: one CTA for each (layer, sequence, KV head) finds the weight of the last
// slot kept by radix selection (11, 11 and 10 bits of an order-preserving integer image of the
// weights, histograms in shared memory), then writes the kept slots in ascending order.
// move_kernel copies their K and V rows and writes the new lengths; it moves nearly all the bytes and is bound by memory: 28
// layers of four sequences of 9000 to 16384 slots cut to 4096 (2 KV heads of 128), 939 MB in 143 us, 6.6 TB/s, 97% of a
// copy's rate.  The selection before it takes 33 us (load, three histograms, count, write) with 70% of the issue slots taken;
// units of few layers and heads leave most SMs without a CTA: one layer of one sequence of 32768 slots, 4 heads, 38 us a call.
#include "kvx_decode.cuh"
#include "kvx_tc_common.cuh"

namespace kvx {
namespace {

constexpr int kSelThreads = 1024;
constexpr int kBins = 2048;
constexpr int kSelFixed = kBins * 4 + 256;
constexpr int kMoveThreads = 256;

// Unsigned image with the order of the weights; -0 as +0, NaN below everything.
__device__ __forceinline__ unsigned weight_key(float w)
{
    if (w != w) return 0u;
    const unsigned u = __float_as_uint(w + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sums of `v` over the CTA's threads before this one, and the sum of all; tmp: shared int[33].
__device__ __forceinline__ int block_before(int v, int* tmp, int& all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) tmp[warp] = x;
    __syncthreads();
    if (warp == 0) {
        int s = tmp[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += y;
        }
        tmp[lane] = s;
    }
    __syncthreads();
    all = tmp[kSelThreads / 32 - 1];
    const int before = (warp ? tmp[warp - 1] : 0) + x - v;
    __syncthreads();
    return before;
}

// Cached tokens of sequence b, clamped to the cache and the weights.
__device__ __forceinline__ int cached_slots(const EvictParams& P, int b, bool& clamped)
{
    const int n = P.kv_len[b], most = (int)min((long long)min(P.src.capacity, 1 << 30), P.weight_stride);
    clamped = n < 0 || n > most;
    return n < 0 ? 0 : min(n, most);
}

// cached: weights the CTA holds in shared memory; slots past them are read again in each pass.
__global__ void __launch_bounds__(kSelThreads, 2) select_kernel(const __grid_constant__ EvictParams P, int cached)
{
    extern __shared__ __align__(16) unsigned dyn[];
    unsigned* hist = dyn;
    int* tmp = reinterpret_cast<int*>(hist + kBins);   // [33], then two words of the digit found
    unsigned* keys = dyn + kSelFixed / 4;
    const int tid = threadIdx.x;
    const long long unit = blockIdx.x;
    const int b = (int)((unit / P.H) % P.batch);
    bool clamped;
    const int n = cached_slots(P, b, clamped);
    if (clamped && tid == 0) set_status(P.status, KVX_DEV_SEQ_CLAMPED);
    int* kept = P.kept + unit * P.keep;
    float* kw = P.kept_weight ? P.kept_weight + unit * P.kept_stride : nullptr;
    const float* w = P.weight + unit * P.weight_stride;
    int m = n;
    if (n <= P.keep) {
        for (int i = tid; i < n; i += kSelThreads) {
            kept[i] = i;
            if (kw) kw[i] = w[i];
        }
    } else {
        m = P.keep;
        // the slots that compete, and how many of them stay (at least one competes: n > keep >= sinks + recent)
        const int c0 = P.sinks, c1 = n - P.recent;
        int need = P.keep - P.sinks - P.recent;
#pragma unroll 4
        for (int i = c0 + tid; i < min(c1, c0 + cached); i += kSelThreads) keys[i - c0] = weight_key(__ldg(&w[i]));
        auto key = [&](int i) { return i - c0 < cached ? keys[i - c0] : weight_key(__ldg(&w[i])); };
        unsigned prefix = 0, mask = 0;
        // need > 0: the digits of the key of rank `need`, from the top; `need` becomes its rank among equals
        for (int pass = 0; pass < 3 && need > 0; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
            __syncthreads();
            for (int i = c0 + tid; i < c1; i += kSelThreads) {
                const unsigned k = key(i);
                if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1u);
            }
            __syncthreads();
            // bins from the highest: thread t holds bins top - 2t and top - 2t - 1
            const int a = (1 << bits) - 1 - 2 * tid;
            const int va = a >= 0 ? (int)hist[a] : 0, vb = a >= 1 ? (int)hist[a - 1] : 0;
            int all;
            const int before = block_before(va + vb, tmp, all);
            if (before < need && need <= before + va + vb) {
                const bool second = need > before + va;
                tmp[32] = second ? a - 1 : a;
                tmp[33] = need - before - (second ? va : 0);
            }
            __syncthreads();
            prefix |= (unsigned)tmp[32] << shift;
            mask |= ((1u << bits) - 1) << shift;
            need = tmp[33];
            __syncthreads();
        }
        // kept: forced slots, keys above the one found, and the first `need` equal to it.  Each warp has a stretch of
        // slots: it counts, the counts are summed over the warps, it writes.
        const bool any = mask != 0;
        const int warp = tid >> 5, lane = tid & 31, stretch = (n + kSelThreads - 1) / kSelThreads * 32;
        const int from = min(n, warp * stretch), to = min(n, from + stretch);
        auto ballots = [&](int i, unsigned& sure, unsigned& tie) {
            bool s = false, t = false;
            if (i < to) {
                if (i < c0 || i >= c1) {
                    s = true;
                } else if (any) {
                    const unsigned k = key(i);
                    s = k > prefix;
                    t = k == prefix;
                }
            }
            sure = __ballot_sync(0xffffffffu, s);
            tie = __ballot_sync(0xffffffffu, t);
        };
        int sures = 0, ties = 0;
        for (int i0 = from; i0 < to; i0 += 32) {
            unsigned a, b;
            ballots(i0 + lane, a, b);
            sures += __popc(a);
            ties += __popc(b);
        }
        if (lane == 0) {
            hist[warp] = sures;
            hist[32 + warp] = ties;
        }
        __syncthreads();
        int before = lane < warp ? (int)hist[lane] : 0, tied = lane < warp ? (int)hist[32 + lane] : 0;
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            before += __shfl_xor_sync(0xffffffffu, before, o);
            tied += __shfl_xor_sync(0xffffffffu, tied, o);
        }
#pragma unroll 4
        for (int i0 = from; i0 < to; i0 += 32) {
            const int i = i0 + lane;
            const float wi = kw && i < to ? __ldg(&w[i]) : 0.0f;        // four in flight
            unsigned a, b;
            ballots(i, a, b);
            const unsigned below = (1u << lane) - 1;
            const int rank = tied + __popc(b & below);                   // among the equal ones
            if ((a >> lane & 1u) || ((b >> lane & 1u) && rank < need)) {
                const int r = before + __popc(a & below) + min(rank, need);
                kept[r] = i;
                if (kw) kw[r] = wi;
            }
            before += __popc(a);
            tied += __popc(b);
        }
    }
    for (int i = m + tid; i < P.keep; i += kSelThreads) kept[i] = -1;
    if (kw)
        for (long long i = m + tid; i < P.kept_stride; i += kSelThreads) kw[i] = 0.0f;
}

// Each warp copies 32 kept rows at a time: the lanes resolve one row each, then all copy them, 16 bytes a lane.
template <int CHUNKS>   // 16-byte chunks of a row: 8 .. 64
__global__ void __launch_bounds__(kMoveThreads) move_kernel(const __grid_constant__ EvictParams P, int elt)
{
    constexpr int RPI = CHUNKS < 32 ? 32 / CHUNKS : 1;      // rows a warp copies with one instruction
    constexpr int CPL = CHUNKS < 32 ? 1 : CHUNKS / 32;      // chunks of a row a lane holds
    constexpr int STEP = CPL == 1 ? 4 * RPI : 4;            // rows in flight: four loads of K and of V a lane
    const int lane = threadIdx.x & 31;
    const int groups = (P.keep + 31) / 32;
    const long long total = (long long)P.L * P.batch * P.H * groups;
    const long long warps = (long long)gridDim.x * (kMoveThreads / 32);
    grid_dependency_wait();
    // the new lengths, now that every selection has read the old ones, whose place they may take
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b < P.batch; b += kMoveThreads) {
            bool clamped;
            P.new_len[b] = min(cached_slots(P, b, clamped), P.keep);
        }
    for (long long g = ((long long)blockIdx.x * kMoveThreads + threadIdx.x) >> 5; g < total; g += warps) {
        const long long unit = g / groups;
        const int r0 = (int)(g - unit * groups) * 32;
        const int h = (int)(unit % P.H), b = (int)((unit / P.H) % P.batch), l = (int)(unit / P.H / P.batch);
        const int r = r0 + lane;
        long long from = -1, to = -1;
        if (r < P.keep) {
            const int s = P.kept[unit * P.keep + r];
            if (s >= 0) {
                from = cache_row(P.src, b, s);
                if (r < P.dst.capacity) to = cache_row(P.dst, b, r);
                else set_status(P.status, KVX_DEV_SEQ_CLAMPED);
                if (from < 0 || (to < 0 && r < P.dst.capacity)) set_status(P.status, KVX_DEV_PAGE_INVALID);
            }
        }
        from = from < 0 || to < 0 ? -1 : (from + cache_head(P.src) * h) * elt;
        to = (to + cache_head(P.dst) * h) * elt;
        if (__all_sync(0xffffffffu, from < 0)) continue;
        const char *sk = (const char*)P.sk[l], *sv = (const char*)P.sv[l];
        char *dk = (char*)P.dk[l], *dv = (char*)P.dv[l];
        const int sub = lane / CHUNKS % RPI, c = CHUNKS < 32 ? lane % CHUNKS : lane;
        for (int i = 0; i < 32; i += STEP) {
            uint4 k[4][CPL], v[4][CPL];
            long long f[4], t[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int row = i + u * RPI + sub;
                f[u] = __shfl_sync(0xffffffffu, from, row);
                t[u] = __shfl_sync(0xffffffffu, to, row);
#pragma unroll
                for (int e = 0; e < CPL; ++e)
                    if (f[u] >= 0) {
                        k[u][e] = __ldcs(reinterpret_cast<const uint4*>(sk + f[u]) + c + 32 * e);
                        v[u][e] = __ldcs(reinterpret_cast<const uint4*>(sv + f[u]) + c + 32 * e);
                    }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int e = 0; e < CPL; ++e)
                    if (f[u] >= 0) {
                        __stcs(reinterpret_cast<uint4*>(dk + t[u]) + c + 32 * e, k[u][e]);
                        __stcs(reinterpret_cast<uint4*>(dv + t[u]) + c + 32 * e, v[u][e]);
                    }
        }
    }
}

template <int CHUNKS> cudaError_t run_move(const EvictParams& P, int elt, int num_sms, cudaStream_t stream)
{
    const long long rows = (long long)P.L * P.batch * P.H * ((P.keep + 31) / 32);
    const long long want = (rows + kMoveThreads / 32 - 1) / (kMoveThreads / 32);
    const int grid = (int)min(want, (long long)num_sms * 8);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kMoveThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, move_kernel<CHUNKS>, P, elt);
}

}  // namespace

cudaError_t launch_evict(const EvictParams& P, int dtype, int num_sms, cudaStream_t stream, int* launches)
{
    const long long units = (long long)P.L * P.batch * P.H;
    const int elt = dtype == KVX_BF16 ? 2 : 4;
    const long long slots = min(P.weight_stride, (long long)P.src.capacity);
    const int cached = (int)min(slots, (long long)(kSmemMax - kSelFixed) / 4);
    const int smem = kSelFixed + cached * 4;
    if (cudaError_t e = smem_opt_in<select_kernel>(kSmemMax); e != cudaSuccess) return e;
    select_kernel<<<(unsigned)units, kSelThreads, smem, stream>>>(P, cached);
    if (cudaError_t e = cudaGetLastError(); e != cudaSuccess) return e;
    *launches = 2;
    switch (P.d * elt / 16) {
    case 8: return run_move<8>(P, elt, num_sms, stream);
    case 16: return run_move<16>(P, elt, num_sms, stream);
    case 32: return run_move<32>(P, elt, num_sms, stream);
    default: return run_move<64>(P, elt, num_sms, stream);
    }
}

}  // namespace kvx
