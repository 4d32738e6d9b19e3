// kvx_key_weight.cu -- the attention weight each cached slot receives, for bf16 caches on the tensor cores.
//
//   key_weight[b, h, j] += sum over the rows i of (b, h) that see j of exp(x_ij - lse_i)
// The scores are formed again now that every row's sum is known, slots by rows: S^T = K Q^T with 128 slots as the
// MMA's rows, so that a thread owns a slot and adds along its TMEM lane, in a fixed order and without
// atomics: one CTA has all rows of a slot tile.  Bound by the MMAs and the waits between them where rows are many
// (1792 rows of each of 4 KV heads over 16384 slots: 46 us; 16 us of MMAs), by reading K where they are few; four slot
// tiles for three CTAs leave a sixth of the device idle at the end of that call.
//   producer warps      two copy K of a slot tile with 16-byte cp.async, one brings Q by tensor copies: a row tile is
//                       the G query heads of 128 / G tokens, one box for each 64 channels
//   MMA thread          S^T into one of four score buffers
//   weight warps        four warpgroups, row tiles in turn, their sums added through shared memory
#include <limits.h>

#include "kvx_attend_rows.cuh"
#include "kvx_umma.cuh"

namespace kvx {
namespace {

constexpr int kKwGroups = 4;

template <int D> struct KwShape {
    static constexpr int TILE = 128 * D * 2;
    static constexpr int CTRL = 22 * 1024;                 // barriers; rows' lse and slots; sums; the units' plan
    static constexpr int SLOTS = (kSmemMax - CTRL) / TILE < 12 ? (kSmemMax - CTRL) / TILE : 12;   // K and Q tiles together
    static constexpr int SMEM = CTRL + SLOTS * TILE;
    static constexpr int THREADS = 128 + 128 * kKwGroups;
    static_assert(SLOTS >= 3 && 13312 + (kMaxAttendBatch + 1) * 8 <= CTRL);
};

// Barriers: full and empty of every tile, scores full and free of every buffer.
struct KwBars {
    static constexpr int full = 0, empty = 12, sfull = 24, sfree = sfull + kKwGroups, done = sfree + kKwGroups;
};

// A slot tile and KV head, and the tokens [t0, t1) that may see any of it, in tiles of `per` tokens.
struct KwUnit {
    int b, h, j0, t0, t1, tiles;
    Seq s;
};
__device__ __forceinline__ KwUnit kw_unit(const AttendParams& P, const long long* first, long long u, int per)
{
    KwUnit x;
    const long long ut = u / P.H;
    x.h = (int)(u - ut * P.H);
    int lo = 0, hi = P.batch - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= ut) lo = mid; else hi = mid - 1;
    }
    x.b = lo;
    x.j0 = (int)(ut - first[lo]) * 128;
    x.s = load_seq(P, lo);
    const int ctx = x.s.L - x.s.n;                         // slot of token 0
    const bool pre = x.j0 < x.s.pre;
    x.t0 = pre ? 0 : max(0, x.j0 - ctx);
    x.t1 = pre || P.window == 0 ? x.s.n : (int)min((long long)x.s.n, (long long)x.j0 + 127 + P.window - ctx);
    x.tiles = x.t1 > x.t0 ? (x.t1 - x.t0 + per - 1) / per : 0;
    return x;
}

template <int D, bool CAP>
__global__ void __launch_bounds__(KwShape<D>::THREADS, 1) key_weight_kernel(const __grid_constant__ AttendParams P, const __grid_constant__ CUtensorMap q_map, int k_slots)
{
    using C = KwShape<D>;
    using B = KwBars;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t s0 = smem_u32(smem);
    auto bar = [&](int i) { return s0 + (uint32_t)i * 8; };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + 512);
    int* abort = reinterpret_cast<int*>(smem + 516);
    float* row_lse = reinterpret_cast<float*>(smem + 1024);        // [4][2][128]: minus the rows' lse, log2 units
    int* row_slot = reinterpret_cast<int*>(smem + 5120);           // [4][2][128]: the rows' own slots
    float* sums = reinterpret_cast<float*>(smem + 9216);           // [2][4][128]
    long long* first = reinterpret_cast<long long*>(smem + 13312);  // [batch + 1]: slot tiles before each sequence's
    const uint32_t sT = s0 + C::CTRL;
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int q_slots = C::SLOTS - k_slots;
    const int per = 128 / P.G;                             // tokens a row tile

    if (warp == 3) tmem_alloc(smem_u32(tmem_slot), 512);
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::SLOTS; ++i) {
            mbar_init(bar(B::full + i), i < k_slots ? 64 : 1);
            mbar_init(bar(B::empty + i), 1);
        }
        for (int i = 0; i < kKwGroups; ++i) {
            mbar_init(bar(B::sfull + i), 1);
            mbar_init(bar(B::sfree + i), 4);
        }
        mbar_init(bar(B::done), 1);
        fence_mbar_init();
        *abort = 0;
    }
    // rows of a Q tile past the last whole token stay zero: their scores are zeros and get no weight
    for (uint32_t i = threadIdx.x; i < (uint32_t)(q_slots * C::TILE / 16); i += C::THREADS)
        *reinterpret_cast<uint4*>(smem + C::CTRL + (size_t)k_slots * C::TILE + i * 16) = make_uint4(0, 0, 0, 0);
    fence_proxy_async();
    for (int b = threadIdx.x; b < P.batch; b += C::THREADS) first[b + 1] = (load_seq(P, b).L + 127) / 128;
    __syncthreads();
    if (warp == 0) {
        long long run = 0;
        for (int b0 = 0; b0 < P.batch; b0 += 32) {
            long long v = b0 + lane < P.batch ? first[b0 + lane + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long w = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += w;
            }
            v += run;
            if (b0 + lane < P.batch) first[b0 + lane + 1] = v;
            run = __shfl_sync(0xffffffffu, v, 31);
        }
        if (lane == 0) first[0] = 0;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    const Waiter W{abort, P.status};
    const long long units = first[P.batch] * P.H;
    bool ok = true;
    auto wait = [&](int b, uint32_t parity) { ok = __all_sync(0xffffffffu, ok && W.wait(bar(b), parity)); };

    if (warp < 2) {
        // ---------------------------------------------------------------- K
        constexpr int CPR = D / 8, RPI = CPR < 32 ? 32 / CPR : 1;
        const int sub = lane / CPR;
        const uint32_t c0 = (uint32_t)(((lane % CPR & 7) ^ sub) << 4);
        const uint32_t d1 = (uint32_t)((lane % CPR >> 3) * (128 * 128) + (warp * 64 + sub) * 128);
        const __nv_bfloat16* src = (const __nv_bfloat16*)P.ck + lane % CPR * 8;
        uint32_t kn = 0;
        for (long long u = blockIdx.x; u < units; u += gridDim.x) {
            const KwUnit x = kw_unit(P, first, u, per);
            if (x.tiles == 0) continue;
            long long at[2];                               // the warp's rows lane and 32 + lane
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int j = x.j0 + warp * 64 + k * 32 + lane;
                at[k] = j < x.s.L ? cache_row(P.cache, x.b, j) : -1;
                if (at[k] >= 0) at[k] += cache_head(P.cache) * x.h;
            }
            const uint32_t ks = kn % (uint32_t)k_slots;
            wait(B::empty + (int)ks, ((kn / (uint32_t)k_slots) & 1) ^ 1);
            if (ok) {
#pragma unroll
                for (int r = 0; r < 64; r += RPI) {
                    const long long row = __shfl_sync(0xffffffffu, at[r / 32], (r & 31) + sub);
                    cp_async16_or_zero(sT + ks * C::TILE + d1 + (uint32_t)r * 128 + (c0 ^ (uint32_t)((r & 7) << 4)),
                                       row < 0 ? (const __nv_bfloat16*)P.ck : src + row, row >= 0);
                }
            }
            cp_async_arrive(bar(B::full + (int)ks));
            ++kn;
        }
        cp_async_wait_all();
    } else if (warp == 2) {
        // ---------------------------------------------------------------- Q
        uint32_t qn = 0, issued = 0;
        for (long long u = blockIdx.x; u < units; u += gridDim.x) {
            const KwUnit x = kw_unit(P, first, u, per);
            for (int i = 0; i < x.tiles; ++i, ++qn) {
                const uint32_t qs = (uint32_t)k_slots + qn % (uint32_t)q_slots, full = bar(B::full + (int)qs);
                wait(B::empty + (int)qs, ((qn / (uint32_t)q_slots) & 1) ^ 1);
                if (!ok) continue;
                issued = qn + 1;
                if (elect_one()) {
                    mbar_arrive_expect_tx(full, (uint32_t)(per * P.G) * D * 2);
#pragma unroll
                    for (int cb = 0; cb < D / 64; ++cb)
                        tma_box3(sT + qs * C::TILE + cb * (128 * 128), &q_map, cb * 64, x.h * P.G, x.s.t0 + x.t0 + i * per, full);
                }
                __syncwarp();
            }
        }
        if (!ok)
            for (uint32_t q = issued > (uint32_t)q_slots ? issued - (uint32_t)q_slots : 0; q < issued; ++q)
                drain(bar(B::full + k_slots + (int)(q % (uint32_t)q_slots)), (q / (uint32_t)q_slots) & 1);
    } else if (warp == 3) {
        // ---------------------------------------------------------------- MMA
        constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
        uint32_t kn = 0, qn = 0;
        for (long long u = blockIdx.x; u < units && ok; u += gridDim.x) {
            const int tiles = __shfl_sync(0xffffffffu, kw_unit(P, first, u, per).tiles, 0);
            if (tiles == 0) continue;
            const uint32_t ks = kn % (uint32_t)k_slots;
            wait(B::full + (int)ks, (kn / (uint32_t)k_slots) & 1);
            for (int i = 0; i < tiles && ok; ++i, ++qn) {
                const uint32_t qs = (uint32_t)k_slots + qn % (uint32_t)q_slots, buf = qn % kKwGroups;
                wait(B::full + (int)qs, (qn / (uint32_t)q_slots) & 1);
                wait(B::sfree + (int)buf, ((qn / kKwGroups) & 1) ^ 1);
                if (!ok) break;
                if (i == 0) fence_proxy_async();             // K came by thread copies
                tc_fence_after();
                const uint64_t kd = sw128_desc(sT + ks * C::TILE), qd = sw128_desc(sT + qs * C::TILE);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint64_t step = (uint64_t)((k >> 2) * (128 * 128 / 16) + (k & 3) * 2);
                        umma_bf16(tmem + buf * 128, kd + step, qd + step, idesc, k > 0);
                    }
                    umma_commit(bar(B::empty + (int)qs));
                    if (i == tiles - 1) umma_commit(bar(B::empty + (int)ks));
                    umma_commit(bar(B::sfull + (int)buf));
                }
                __syncwarp();
            }
            ++kn;
        }
        // every MMA issued has completed before TMEM is freed
        if (elect_one()) umma_commit(bar(B::done));
        const unsigned long long t0 = globaltimer();
        while (!mbar_try_wait(bar(B::done), 0) && globaltimer() - t0 < kWaitNs) {}
    } else {
        // ---------------------------------------------------------------- weights
        const int wg = (warp - 4) >> 2, quad = warp & 3, own = quad * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)wg * 128;
        const float inv_cap = CAP ? 1.0f / P.cap : 0.0f;
        const float c = CAP ? 1.0f : P.scale * kLog2e;
        const int my_tok = own / P.G, my_head = own - my_tok * P.G;   // this thread's row of every row tile
        const bool my_row = my_tok < per;
        uint32_t qn = 0, shared = 0, turn = 0;
        for (long long u = blockIdx.x; u < units; u += gridDim.x) {
            const KwUnit x = kw_unit(P, first, u, per);
            const int tiles = x.tiles;
            if (tiles == 0) continue;
            const int j = x.j0 + own;
            float w = 0.0f;
            const bool prefix = j < x.s.pre;
            const unsigned reach = P.window > 0 ? (unsigned)P.window : 1u << 30;   // slots differ by less than 2^30
            auto seen = [&](int at) { return ((unsigned)(at - j) < reach) | (prefix & (at != INT_MIN)); };   // no branches
            // minus the lse of this thread's row of row tile i: -infinity, a weight of zero, where it has none
            auto row_value = [&](int i) {
                const int t = x.t0 + i * per + my_tok;
                return my_row && i < tiles && t < x.t1
                           ? -__ldcg(&P.lse[(long long)(x.s.t0 + t) * P.Hq + x.h * P.G + my_head]) * kLog2e : -INFINITY;
            };
            const int i0 = (int)(((uint32_t)wg - qn) % kKwGroups);
            float next = row_value(i0);
            for (int i = i0; i < tiles; i += kKwGroups, ++turn) {
                const uint32_t n = qn + (uint32_t)i;
                const int t = x.t0 + i * per;
                float* lse = row_lse + (wg * 2 + (turn & 1)) * 128;
                int* slot = row_slot + (wg * 2 + (turn & 1)) * 128;
                lse[own] = next;
                slot[own] = my_row && t + my_tok < x.t1 ? x.s.slot(t + my_tok) : INT_MIN;
                group_sync(1 + wg, 128);
                next = row_value(i + kKwGroups);
                wait(B::sfull + wg, (n / kKwGroups) & 1);
                tc_fence_after();
                // do all rows of a whole tile see all its slots?
                const int lo_slot = x.s.slot(t), hi_slot = x.s.slot(t + per - 1);
                const bool all = t + per <= x.t1 &&
                                 ((x.j0 + 127 <= lo_slot && (P.window == 0 || hi_slot - x.j0 < P.window)) || x.j0 + 128 <= x.s.pre);
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                if (ok) {
#pragma unroll 1                                             // a body twice as long would miss the instruction cache
                    for (int k0 = 0; k0 < 128; k0 += 32) {
                        uint32_t s[32];
                        tmem_ld32_to(s, lanes + k0);
                        tmem_ld_wait();
                        pin32(s);
                        auto sf = [&](int k) -> float { return __uint_as_float(s[k]); };
                        // the weights of rows k .. k + 3
                        auto four = [&](int k0_, int k, float2& a, float2& b) {
                            const float4 z = *reinterpret_cast<const float4*>(lse + k0_ + k);
                            a = fma2(make_float2(sf(k), sf(k + 1)), make_float2(c, c), make_float2(z.x, z.y));
                            b = fma2(make_float2(sf(k + 2), sf(k + 3)), make_float2(c, c), make_float2(z.z, z.w));
                            a = make_float2(exp2_hw(a.x), exp2_hw(a.y));
                            b = make_float2(exp2_hw(b.x), exp2_hw(b.y));
                        };
                        if (k0 == 96) {                      // the buffer may be written again
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(bar(B::sfree + wg));
                        }
                        if constexpr (CAP) {
                            bool near = true;
#pragma unroll
                            for (int k = 0; k < 32; ++k) {
                                const float y = sf(k) * (P.scale * inv_cap);
                                near = near && fabsf(y) < 0.5f;
                                s[k] = __float_as_uint(y);
                            }
                            if (__all_sync(0xffffffffu, near)) {
#pragma unroll
                                for (int k = 0; k < 32; ++k) s[k] = __float_as_uint(P.cap * kLog2e * tanh_series(sf(k)));
                            } else {
#pragma unroll
                                for (int k = 0; k < 32; ++k)
                                    s[k] = __float_as_uint(P.cap * kLog2e * (fabsf(sf(k)) < 0.5f ? tanh_series(sf(k)) : tanh_far(sf(k))));
                            }
                        }
                        // two bodies without a branch in them: the loads, exponentials and sums of many rows overlap
                        if (all) {
#pragma unroll
                            for (int k = 0; k < 32; k += 4) {
                                float2 a, b;
                                four(k0, k, a, b);
                                sum[0] = add2(sum[0], a);
                                sum[1] = add2(sum[1], b);
                            }
                        } else {
#pragma unroll
                            for (int k = 0; k < 32; k += 4) {
                                float2 a, b;
                                four(k0, k, a, b);
                                const int4 at = *reinterpret_cast<const int4*>(slot + k0 + k);
                                a.x = seen(at.x) ? a.x : 0.0f;
                                a.y = seen(at.y) ? a.y : 0.0f;
                                b.x = seen(at.z) ? b.x : 0.0f;
                                b.y = seen(at.w) ? b.y : 0.0f;
                                sum[0] = add2(sum[0], a);
                                sum[1] = add2(sum[1], b);
                            }
                        }
                    }
                }
                w += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
            }
            // one tile: its warpgroup has the whole sum; more: the first adds all warpgroups' in order
            const bool mine = tiles == 1 ? i0 == 0 : wg == 0;
            if (tiles > 1) {
                float* part = sums + (shared & 1) * (kKwGroups * 128) + own;
                part[wg * 128] = w;
                group_sync(1 + kKwGroups, 128 * kKwGroups);
                if (wg == 0) w = (part[0] + part[128]) + (part[256] + part[384]);
                ++shared;
            }
            if (mine && ok && j < x.s.L && j < P.weight_stride) {
                float* to = P.key_weight + ((long long)x.b * P.H + x.h) * P.weight_stride + j;
                *to += w;
            }
            qn += (uint32_t)tiles;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 3) {
        tmem_relinquish();
        tmem_dealloc(tmem, 512);
    }
}

// The same sums from scores that the attention has left.  Few rows: a thread a slot, eight rows' scores in flight;
// bound by latency (1.5 M scores: 11 us from cold caches).
__global__ void __launch_bounds__(128) sum_few_scores_kernel(const __grid_constant__ AttendParams P)
{
    const int b = blockIdx.z, h = blockIdx.y, j = blockIdx.x * 128 + threadIdx.x;
    grid_dependency_wait();
    const Seq s = load_seq(P, b);
    if (j >= s.L || j >= P.weight_stride || s.n == 0) return;
    float* to = P.key_weight + ((long long)b * P.H + h) * P.weight_stride + j;
    float w = *to;
    for (int t = 0; t < s.n; ++t) {
        if (!sees(P, s, s.slot(t), j)) continue;
        const long long at = (long long)(s.t0 + t) * P.Hq + h * P.G;
        for (int g0 = 0; g0 < P.G; g0 += 8) {
            float x[8], z[8];
#pragma unroll
            for (int g = 0; g < 8; ++g) {
                const bool in = g0 + g < P.G;
                x[g] = in ? __ldcg(&P.scores[(at + g0 + g) * P.scores_stride + j]) : -INFINITY;
                z[g] = in ? __ldcg(&P.lse[at + g0 + g]) * kLog2e : 0.0f;
            }
            float sum = 0.0f;
#pragma unroll
            for (int g = 0; g < 8; ++g) sum += exp2_hw(x[g] - z[g]);
            w += sum;
        }
    }
    *to = w;
}
// Many: 32 slots a CTA, a lane each; a warp has all query heads of every 16th token, and the warps' sums are added
// in order.
__global__ void __launch_bounds__(512) sum_scores_kernel(const __grid_constant__ AttendParams P)
{
    __shared__ float part[16][33];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = blockIdx.z, h = blockIdx.y, j = blockIdx.x * 32 + lane;
    grid_dependency_wait();
    const Seq s = load_seq(P, b);
    if (blockIdx.x * 32 >= s.L) return;
    const bool in = j < s.L && j < P.weight_stride;
    float w = 0.0f;
    for (int t = warp; t < s.n; t += 16) {
        const bool seen = in && sees(P, s, s.slot(t), j);
        const long long at = (long long)(s.t0 + t) * P.Hq + h * P.G;
#pragma unroll 4
        for (int g = 0; g < P.G; ++g) {
            const float x = seen ? __ldcg(&P.scores[(at + g) * P.scores_stride + j]) : -INFINITY;
            const float z = __ldcg(&P.lse[at + g]) * kLog2e;
            w += seen ? exp2_hw(x - z) : 0.0f;
        }
    }
    part[warp][lane] = w;
    __syncthreads();
    if (warp == 0 && in) {
        w = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; ++k) w += part[k][lane];
        P.key_weight[((long long)b * P.H + h) * P.weight_stride + j] += w;
    }
}

template <int D, bool CAP> cudaError_t run_key_weight(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    using C = KwShape<D>;
    if (cudaError_t e = smem_opt_in<key_weight_kernel<D, CAP>>(C::SMEM); e != cudaSuccess) return e;
    // One row tile a slot tile: K is what is read, so most tiles are for it; else the rows' tiles are.  (Heads of 256: 18 rows
    // of each of four sequences of 16000 slots 124.6 us, with most tiles for the rows 130.8; narrower heads alike.)
    const bool few = (long long)P.T * P.G <= 128ll * P.batch;
    const int k_slots = few ? C::SLOTS - (C::SLOTS > 4 ? 2 : 1) : C::SLOTS > 4 ? 2 : 1;
    CUtensorMap map;
    const int per = 128 / P.G;
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)P.Hq, (cuuint64_t)P.T};
    const cuuint64_t strides[2] = {(cuuint64_t)P.q_h * 2, (cuuint64_t)P.q_t * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)P.G, (cuuint32_t)per}, one[3] = {1, 1, 1};
    const EncodeTiled enc = tiled_encoder();
    if (!enc || enc(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(P.q), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    key_weight_kernel<D, CAP><<<num_sms, C::THREADS, C::SMEM, stream>>>(P, map, k_slots);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_key_weight(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    // the capped scores' code apart: with it the plain kernels would be twice as long
    if (P.cap > 0.0f)
        return P.d == 64 ? run_key_weight<64, true>(P, num_sms, stream) : P.d == 128 ? run_key_weight<128, true>(P, num_sms, stream)
                                                                                       : run_key_weight<256, true>(P, num_sms, stream);
    return P.d == 64 ? run_key_weight<64, false>(P, num_sms, stream) : P.d == 128 ? run_key_weight<128, false>(P, num_sms, stream)
                                                                                    : run_key_weight<256, false>(P, num_sms, stream);
}

cudaError_t launch_sum_scores(const AttendParams& P, cudaStream_t stream)
{
    // (fp32, one sequence of 8000 slots: 14 rows 47.7 us with a thread a slot and 50.8 with a warp a token, 28 rows alike, 63
    // rows 79.5 and 75.4)
    const bool few = (long long)P.T * P.G <= 32ll * P.batch;
    const int slots = few ? 128 : 32;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((P.weight_stride + slots - 1) / slots), P.H, P.batch);
    cfg.blockDim = dim3(few ? 128 : 512);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return few ? cudaLaunchKernelEx(&cfg, sum_few_scores_kernel, P) : cudaLaunchKernelEx(&cfg, sum_scores_kernel, P);
}

}  // namespace kvx
