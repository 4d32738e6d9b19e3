// kvx_attend_tc.cuh -- attention of new tokens over a bf16 cache on the tensor cores (tcgen05).  Compiled twice, with
// and without the capped scores' code: with it the plain kernels would be twice as long.
//
//   S = Q K^T (fp32, TMEM),  P = exp2(c S - m),  O += P V (P bf16 from TMEM, O fp32 in TMEM)
// in one pass over the slots, with the running maximum m and sum l of a row in the registers of the thread
// that owns the row.  A CTA holds NT tiles of 128 rows and walks slot tiles of BN.
//   producer warps (3)  copy Q, K and V rows into 128-byte-swizzled tiles: Q by tensor copies (TMA), K and V by
//                       16-byte thread copies through the page table, a tile a warp.  A K tile is read as a
//                       K-major operand, a V tile, laid out alike, as an MN-major one.
//   MMA warp            unit u = (slot tile, row tile): S(u) into score buffer u mod 2, then, when P(u)
//                       is there, O += P(u) V; S(u + 2) is issued right behind it, so that the scores of
//                       one unit are formed while the other's softmax runs.
//   softmax warps       two warpgroups, for units of even and odd u: a row tile each (NT = 2), or every other
//                       slot tile of the one row tile (NT = 1), each with its own maximum, sum and O,
//                       which the first joins at the end.  Heads of 256, whose two O would not fit TMEM: both
//                       on every unit, half the columns each.  P takes the place of S.  O is rescaled only
//                       when a row's maximum has grown by more than 2^8 since the last time.
// P is rounded to bf16 for the MMA, as V is, in calls of many rows: out is then off by 2.2e-3 (relative, 4096 slots) where
// its own rounding to bf16 is 1.66e-3, and a second term everywhere would cost 4096 tokens over 32768 slots 43% (1.64 ms
// against 1.15).  Where the copies bound the kernel (one row tile: 99 us against 97 for a token of each of eight sequences),
// and where rows see few slots, so that the rounding of one weight shows (worst element over 16 slots 1.26 times as far off;
// 1 to 3 us of 30), P goes in as two bf16 terms, high and low: 1.66e-3.
//
// What bounds it.  Many rows: the chain S -> softmax -> P V of each row tile, which the other tile's MMAs only partly
// fill: 4096 tokens of 28 query heads (7 a KV head, 128 wide) over 32768 slots take 1.22 ms a call among others, 1.48 PFLOP/s
// or 78% of a large library product's burst rate (1.11 ms alone behind a flush of L2), with pages of 16 tokens, of 64 or
// none.  Few rows: the reading of K and V: one token of each of eight sequences over up to 32768 slots, 411 MB, 83 us, 4.9
// TB/s.  Heads of 256: the softmax, whose two warpgroups agree on a maximum for every 64 slots: 512 tokens of 8 query
// heads over 8192 slots 40 us, the tensor pipe 39% busy.  Short calls: latency, about 11 us from launch to end (three
// dependent reads from DRAM: lengths, page table, rows; code that is not in the instruction cache yet, which is why its
// loops are short where they can be).
#pragma once

#include <atomic>
#include <type_traits>

#include "kvx_attend_rows.cuh"
#include "kvx_kernels.h"
#include "kvx_umma.cuh"

namespace kvx {
namespace {

template <int D, int NT, bool CODES = false> struct TcShape {
    static constexpr int BM = 128 * NT, BN = NT == 1 ? 64 : 128, NB = 2 / NT;
    static constexpr bool COLS = D == 256;                 // the softmax warpgroups share every unit's columns
    static constexpr int STEP = COLS ? 1 : 2;              // a warpgroup's units: every, or every second
    static constexpr int OS = COLS ? 1 : 2;                // O accumulators
    static constexpr int TILE = BN * D * 2, QB = BM * D * 2;
    static constexpr int CTRL = 3072;                      // barriers and flags; what the warpgroups tell each other of rows
    // 8-bit caches: units of rows as codes (and their scales), which become bf16 tiles
    static constexpr int RU = D == 256 ? 32 : D == 128 || NT == 1 ? 64 : 128, RAW_STAGES = 4, RAW_UNIT = RU * D, UNITS = BN / RU;
    static constexpr int RAW = CODES ? RAW_STAGES * RAW_UNIT : 0, SCALES = D == 256 ? 256 : 2048;   // (their scales lie in the control block)
    static constexpr int STAGES = (kSmemMax - CTRL - QB - RAW) / TILE < 12 ? (kSmemMax - CTRL - QB - RAW) / TILE : 12;
    static constexpr int THREADS = CODES ? 512 : 384;
    static constexpr int S_COL = BN, O_COL = 2 * BN;       // TMEM columns: scores u mod 2, then the O tiles
    static constexpr int TMEM = 512;
    static constexpr int SMEM = CTRL + QB + STAGES * TILE + RAW;
    static_assert(SMEM <= kSmemMax && O_COL + OS * D <= TMEM);
    static_assert((kMaxAttendBatch + 2) * 8 <= STAGES * TILE);   // the plan's sums lie where the tiles come later
};

constexpr int kProdWarps = 3, kMmaWarp = 3;

// Bits [a, b) of the 32 columns from `base` on (a, b relative to column 0 of the tile).
__device__ __forceinline__ uint32_t range_bits(int a, int b, int base)
{
    const int lo = max(a - base, 0), hi = min(b - base, 32);
    if (hi <= lo) return 0u;
    return (hi == 32 ? 0xffffffffu : (1u << hi) - 1u) & ~((1u << lo) - 1u);
}

// Registers of a thread once the warps have taken their parts (two softmax warpgroups: 384 threads launched with 168, or 512
// with 128): 128 x 88 + 256 x 208 = 384 x 168, 256 x 56 + 256 x 200 = 512 x 128.

constexpr int kFewSlots = 512;   // rows that see fewer slots get their weights in two terms

// Sequences of up to 128 rows a KV head: one row tile, bound by the copies.  Eight sequences of 16384 slots, 7 query heads on
// each of 4 KV heads of 128: 126 rows 87.7 us with one row tile and 91.8 with two, 133 rows 127.6 and 92.8; heads of 64,
// 128 rows 41.6 and 43.7, 144 rows 48.8 and 43.7.  (The lengths are on the device, so the rule goes by the call's mean: one
// sequence of 256 tokens among 63 without any takes 111 us where two row tiles would take 83.)
__host__ __device__ __forceinline__ bool one_tile(const AttendParams& P) { return (long long)P.T * P.G <= 128ll * P.batch; }

// Sixteen codes of a row of scale f as bf16, exactly: first and second eight.  (By way of fp32: moving exponent and mantissa to
// bf16's places and multiplying there takes more instructions, and NaN codes and far scales more of them; 27 clocks of an SM
// for 512 codes against 20.)
__device__ __forceinline__ void row_bf16(uint4 w, float f, uint4& lo, uint4& hi)
{
    uint32_t v[8];
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
    const float2 f2 = make_float2(f, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 y = mul2(codes_f32((unsigned short)(in[i >> 1] >> (i & 1) * 16)), f2);
        v[i] = pack_bf16(y.x, y.y);
    }
    lo = make_uint4(v[0], v[1], v[2], v[3]);
    hi = make_uint4(v[4], v[5], v[6], v[7]);
}

// Whether an item's weights are multiplied in two terms: its first token sees fewest slots.
template <int D, int NT> __device__ __forceinline__ bool two_terms(const AttendParams& P, const Segment& g)
{
    if constexpr (NT == 1 && D < 256) return true;
    if (NT == 1 && one_tile(P)) return true;
    int ta, tb;
    row_tile_tokens(P, g.s, g.rt, ta, tb);
    const int own = g.s.slot(ta);
    return own < kFewSlots || (P.window > 0 && P.window < kFewSlots);
}

// How K and V tiles are brought: row by row (any page size), or in groups of 8 rows a fixed stride apart (contiguous caches
// and page sizes that are multiples of 8: 4096 tokens over 32768 slots 1.13 ms against 1.35).  (Tensor copies, a box a page,
// were slower: with pages of 16, 32 and 64 slots 2.06, 1.29 and 1.18 ms.)  kCodes: an 8-bit cache, row by row, by warps that copy
// codes and warps that convert them; 4 more warps, registers for it from the softmax warps' 208 (now 200).
enum Source { kRows, kGroups, kCodes };

template <int D, int NT, Source SRC, bool CAP>
__global__ void __launch_bounds__(TcShape<D, NT, SRC == kCodes>::THREADS, 1)
    attend_tc_kernel(const __grid_constant__ AttendParams P, const __grid_constant__ CUtensorMap q_map)
{
    using C = TcShape<D, NT, SRC == kCodes>;
    using B = Bars<C::STAGES>;
    // the barriers end before the scales of an 8-bit cache's units, or the flags at 512
    static_assert(8 * B::count <= (SRC == kCodes && C::COLS ? C::SCALES : 512));
    constexpr int BM = C::BM, BN = C::BN;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t s0 = smem_u32(smem);
    auto bar = [&](int i) { return s0 + (uint32_t)i * 8; };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + 512);
    int* abort = reinterpret_cast<int*>(smem + 516);
    int* beat = reinterpret_cast<int*>(smem + 520);
    const uint32_t sQ = s0 + C::CTRL, sT = sQ + C::QB;
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (warp == kMmaWarp) tmem_alloc(smem_u32(tmem_slot), C::TMEM);
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) {
            mbar_init(bar(B::full + i), SRC == kCodes ? 4 : 32);
            mbar_init(bar(B::empty + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(B::sfull + i), 1);
            mbar_init(bar(B::pfull + i), C::COLS ? 8 : 4);
            mbar_init(bar(B::ofull + i), 1);
        }
        if (SRC == kCodes)
            for (int i = 0; i < C::RAW_STAGES; ++i) {
                mbar_init(bar(B::raw_full + i), 33);
                mbar_init(bar(B::raw_empty + i), 4);
            }
        mbar_init(bar(B::qfull), 1);
        mbar_init(bar(B::qempty), 1);
        mbar_init(bar(B::done), 1);
        mbar_init(bar(B::mlfull), 4);
        mbar_init(bar(B::mlempty), 4);
        mbar_init(bar(B::added), 1);
        fence_mbar_init();
        *abort = 0;
        *beat = 0;
    }
    // the kernel before this one may still be ending: what it wrote is read from here on
    grid_dependency_wait();
    grid_launch_dependents();
    const Plan mine_plan = make_plan<BN, C::THREADS>(P, reinterpret_cast<long long*>(smem + C::CTRL + C::QB));
    Plan* plan = reinterpret_cast<Plan*>(smem + 544);               // the CTA's range, and where each warp stands on it
    if (threadIdx.x == 0) *plan = mine_plan;
    WalkState* state = reinterpret_cast<WalkState*>(smem + 640) + warp;
    static_assert(sizeof(Plan) <= 96 && sizeof(WalkState) * (C::THREADS / 32) <= 1024 - 640);
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const BeatWaiter W{abort, beat, P.status};
    SegmentWalk<BN> walk(P, plan, state);
    Segment g;

    if (warp < 4 || warp >= 12) {
    if constexpr (SRC == kCodes) regs_give<56>();
    else regs_give<88>();
    if (SRC == kCodes && warp != kMmaWarp) {
        // ---------------------------------------------------------------- producers, 8-bit caches
        // Three warps copy units of RU rows as they are, with their scales, every third unit each; four turn them into bf16
        // tiles, a quarter of every unit each.  (Warps that both copied and converted halves of every third tile spent most of
        // their time on one another's latency: 304 us for 1024 tokens over 16384 slots.)
        if constexpr (SRC == kCodes) {
            constexpr int CPR = D / 16, RPI = 32 / CPR, UNITS = C::UNITS;      // 16-code chunks of a row; rows of an instruction
            const int sub = lane / CPR, chunk = lane % CPR;
            const uint32_t sRaw = sT + C::STAGES * C::TILE;
            static_assert(C::SCALES + C::RAW_STAGES * C::RU <= (C::COLS ? 512 : C::CTRL));
            uint32_t pos = 0, items = 0;                 // units and items begun
            bool ok = true;
            auto wait = [&](int b, uint32_t parity) { ok = __all_sync(0xffffffffu, ok && W.wait(bar(b), parity)); };
            if (warp < kProdWarps) {
                uint32_t q_issued = 0;
                while (walk.next(g)) {
                    if (warp == 0) {
                        if (items > 0) wait(B::qempty, (items - 1) & 1);
                        q_issued += ok;
                        if (ok && elect_one()) {
                            mbar_arrive_expect_tx(bar(B::qfull), (uint32_t)P.tile_rows * D * 2);
#pragma unroll
                            for (int cb = 0; cb < D / 64; ++cb)
                                tma_box3(sQ + cb * (BM * 128), &q_map, cb * 64, g.h * P.G, g.s.t0 + g.rt * (P.tile_rows / P.G), bar(B::qfull));
                        }
                        __syncwarp();
                    }
                    ++items;
                    constexpr int LOOK = C::RU / 32;
                    const long long head = cache_head(P.cache) * g.h + chunk * 16, shead = scale_head(P.cache, P.scales) * g.h;
                    const int total = 2 * g.n, all = total * UNITS;
                    // unit r of the item: its first slot, and whether it is of K or V
                    auto first_slot = [&](int r, int& kv) {
                        const int x = r / UNITS;
                        kv = C::NB == 1 ? x & 1 : x == total - 1 || (x > 0 && !(x & 1));
                        const int i = C::NB == 1 ? x >> 1 : x == total - 1 ? g.n - 1 : kv ? (x >> 1) - 1 : (x + 1) >> 1;
                        return g.kv.at(g.i0 + i) * BN + (r - x * UNITS) * C::RU;
                    };
                    auto pages_of = [&](int r, int (&x)[LOOK]) {
                        int kv;
                        const int j0 = r < all ? first_slot(r, kv) : g.s.L;
#pragma unroll
                        for (int k = 0; k < LOOK; ++k) {
                            const int j = j0 + k * 32 + lane;
                            x[k] = -2;                   // past the end
                            if (j < g.s.L) {
                                x[k] = 0;
                                if (P.cache.paged) {
                                    const int pi = P.cache.page_shift >= 0 ? j >> P.cache.page_shift : j / P.cache.page_size;
                                    x[k] = pi < P.cache.max_pages ? P.cache.page_table[(size_t)g.b * P.cache.max_pages + pi] : -1;
                                }
                            }
                        }
                    };
                    int page[LOOK];
                    int r = (int)((kProdWarps + (uint32_t)warp - pos % kProdWarps) % kProdWarps);
                    pages_of(r, page);
                    for (; r < all; r += kProdWarps) {
                        const uint32_t p = pos + (uint32_t)r, st = p % C::RAW_STAGES, ph = (p / C::RAW_STAGES) & 1;
                        int kv;
                        const int j0 = first_slot(r, kv);
                        const uint8_t* src = (const uint8_t*)(kv ? P.cv : P.ck);
                        const unsigned char* scales = kv ? P.v_scale : P.k_scale;
                        long long at[LOOK];
                        uint32_t scale[LOOK];
#pragma unroll
                        for (int k = 0; k < LOOK; ++k) {
                            const int j = j0 + k * 32 + lane;
                            at[k] = -1;
                            scale[k] = 0;
                            if (page[k] == -2) continue;
                            long long z;
                            if (!P.cache.paged) {
                                at[k] = (long long)g.b * P.cache.sb + (long long)j * P.cache.st;
                                z = (long long)g.b * P.scales.sb + j;
                            } else {
                                if (page[k] < 0 || page[k] >= P.cache.num_pages) {
                                    set_status(P.status, KVX_DEV_PAGE_INVALID);
                                    continue;
                                }
                                const int in = P.cache.page_shift >= 0 ? j & (P.cache.page_size - 1) : j % P.cache.page_size;
                                at[k] = ((long long)page[k] * P.cache.page_size + in) * ((long long)P.cache.H * D);
                                z = (long long)page[k] * P.cache.H * P.cache.page_size + in;
                            }
                            scale[k] = scales[z + shead];
                        }
                        pages_of(r + kProdWarps, page);
                        wait(B::raw_empty + (int)st, ph ^ 1);
                        if (!ok) break;
                        const uint32_t d = sRaw + st * C::RAW_UNIT + (uint32_t)lane * 16;
#pragma unroll 8
                        for (int c = 0; c < C::RU / RPI; ++c) {
                            const long long row = __shfl_sync(0xffffffffu, at[LOOK == 1 ? 0 : c * RPI / 32], c * RPI % 32 + sub);
                            cp_async16_or_zero(d + (uint32_t)c * 512, row < 0 ? src : src + row + head, row >= 0);
                        }
                        cp_async_arrive(bar(B::raw_full + (int)st));
#pragma unroll
                        for (int k = 0; k < LOOK; ++k) smem[C::SCALES + st * C::RU + k * 32 + lane] = (uint8_t)scale[k];
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(B::raw_full + (int)st));
                    }
                    pos += (uint32_t)all;
                }
                cp_async_wait_all();
                if (!ok && warp == 0 && q_issued > 0) drain(bar(B::qfull), (q_issued - 1) & 1);
            } else {
                constexpr int QR = C::RU / 4, N = QR / RPI;                    // rows of a unit that this warp has; its instructions
                const int quarter = warp - 12;
                // where a row's first and second eight values go: with 8 lanes or more a row, half the lanes take them the other
                // way round, so that eight lanes' stores fall into different banks
                const bool swap = D >= 128 && (lane & 4);
                const uint32_t q0 = (uint32_t)(2 * chunk + (swap ? 1 : 0)), block = (q0 >> 3) * (uint32_t)(BN * 128), in0 = q0 & 7;
                while (ok && walk.next(g)) {
                    const int all = 2 * g.n * UNITS;
                    for (int r = 0; r < all && ok; ++r, ++pos) {
                        const uint32_t rs = pos % C::RAW_STAGES, p = pos / UNITS, st = p % C::STAGES;
                        wait(B::raw_full + (int)rs, (pos / C::RAW_STAGES) & 1);
                        if (pos % UNITS == 0) wait(B::empty + (int)st, ((p / C::STAGES) & 1) ^ 1);
                        if (!ok) break;
                        uint4 w[N];
                        float f[N];
                        const int row0 = quarter * QR + sub;
#pragma unroll
                        for (int c = 0; c < N; ++c) {
                            w[c] = lds128(sRaw + rs * C::RAW_UNIT + (uint32_t)((quarter * N + c) * 512 + lane * 16));
                            f[c] = scale_of(smem[C::SCALES + rs * C::RU + row0 + c * RPI]);
                        }
                        const uint32_t d = sT + st * C::TILE + block + (uint32_t)((int)(pos % UNITS) * C::RU + row0) * 128;
#pragma unroll
                        for (int c = 0; c < N; ++c) {
                            uint4 lo, hi;
                            row_bf16(w[c], f[c], lo, hi);
                            const uint32_t x = (uint32_t)((row0 + c * RPI) & 7);
                            sts128(d + c * RPI * 128 + ((in0 ^ x) << 4), swap ? hi : lo);
                            sts128(d + c * RPI * 128 + ((in0 ^ 1 ^ x) << 4), swap ? lo : hi);
                        }
                        const bool last = pos % UNITS == UNITS - 1;
                        if (last) fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) {
                            mbar_arrive(bar(B::raw_empty + (int)rs));
                            if (last) mbar_arrive(bar(B::full + (int)st));
                        }
                    }
                }
            }
        }
    } else if (warp < kProdWarps) {
        // ---------------------------------------------------------------- producers
        constexpr int CPR = D / 8;                       // 16-byte chunks of a row
        constexpr int RPI = CPR < 32 ? 32 / CPR : 1;     // rows a warp copies with one instruction
        const int sub = lane / CPR;
        const uint32_t place = (uint32_t)((lane % CPR >> 3)), c0 = (uint32_t)(((lane % CPR & 7) ^ sub) << 4);
        uint32_t pos = 0, items = 0;                     // tiles and items begun
        uint32_t q_issued = 0;                           // tensor copies of Q
        bool ok = true;
        auto wait = [&](int b, uint32_t parity) { ok = __all_sync(0xffffffffu, ok && W.wait(bar(b), parity)); };
        // The copies of a batch announce themselves: each thread's arrival follows its own copies.  The MMA warp
        // orders them before its reads (fence_proxy_async after the wait).
        while (walk.next(g)) {
            if (warp == 0) {
                // Q: the G query heads of tile_rows / G tokens, a box for each 64 channels; what it brings past the
                // sequence's tokens is in rows that nothing is read from
                if (items > 0) wait(B::qempty, (items - 1) & 1);
                q_issued += ok;
                if (ok && elect_one()) {
                    mbar_arrive_expect_tx(bar(B::qfull), (uint32_t)P.tile_rows * D * 2);
#pragma unroll
                    for (int cb = 0; cb < D / 64; ++cb)
                        tma_box3(sQ + cb * (BM * 128), &q_map, cb * 64, g.h * P.G, g.s.t0 + g.rt * (P.tile_rows / P.G), bar(B::qfull));
                }
                __syncwarp();
            }
            ++items;
            const long long head = cache_head(P.cache) * g.h;
            // tile i as K, tile i - NB + 1 as V, and at the end the V tiles left
            // Each warp takes every third tile: a part of every tile each would spend most of its time on what a
            // tile costs anyway (4096 tokens over 32768 slots 1.32 ms against 1.12, a token each of 8 sequences over
            // 32768 slots 166 us against 117).  The next tile's pages are read while this one's copies are
            // issued, and looked at only then.
            constexpr int PER = SRC == kGroups ? 8 : 1;      // rows a stride apart: a lane finds the first of them
            constexpr int FIND = BN / PER;                   // of these a tile has
            constexpr int LOOK = (FIND + 31) / 32;
            const long long stride = P.cache.paged ? (long long)P.cache.H * D : P.cache.st;
            const long long mine = head + (PER > 1 ? sub * stride : 0) + lane % CPR * 8;
            const int total = 2 * g.n;
            // tile r of the item in the order of the ring: K or V, and the slot tile
            auto tile_of = [&](int r, int& kv) {
                if (C::NB == 1) {
                    kv = r & 1;
                    return r >> 1;
                }
                kv = r == total - 1 || (r > 0 && !(r & 1));
                return r == total - 1 ? g.n - 1 : kv ? (r >> 1) - 1 : (r + 1) >> 1;
            };
            auto pages_of = [&](int r, int (&x)[LOOK]) {
                int kv;
                const int j0 = r < total ? g.kv.at(g.i0 + tile_of(r, kv)) * BN : g.s.L;
#pragma unroll
                for (int k = 0; k < LOOK; ++k) {
                    const int j = j0 + (k * 32 + lane) * PER;
                    x[k] = -2;                               // past the end
                    if (k * 32 + lane < FIND && j < g.s.L) {
                        x[k] = 0;
                        if (P.cache.paged) {
                            const int pi = P.cache.page_shift >= 0 ? j >> P.cache.page_shift : j / P.cache.page_size;
                            x[k] = pi < P.cache.max_pages ? P.cache.page_table[(size_t)g.b * P.cache.max_pages + pi] : -1;
                        }
                    }
                }
            };
            auto row_at = [&](int j, int page) -> long long {
                if (page == -2) return -1;
                if (!P.cache.paged) return (long long)g.b * P.cache.sb + (long long)j * P.cache.st;
                if (page < 0 || page >= P.cache.num_pages) {
                    set_status(P.status, KVX_DEV_PAGE_INVALID);
                    return -1;
                }
                const int in = P.cache.page_shift >= 0 ? j & (P.cache.page_size - 1) : j % P.cache.page_size;
                return ((long long)page * P.cache.page_size + in) * stride;
            };
            int next[LOOK];
            int r = (int)((kProdWarps + (uint32_t)warp - pos % kProdWarps) % kProdWarps);
            pages_of(r, next);
            for (; r < total; r += kProdWarps) {
                int kv;
                const int j0 = g.kv.at(g.i0 + tile_of(r, kv)) * BN;
                const __nv_bfloat16* src = (const __nv_bfloat16*)(kv ? P.cv : P.ck);
                const uint32_t p = pos + (uint32_t)r, st = p % C::STAGES, ph = (p / C::STAGES) & 1;
                long long at[LOOK];
#pragma unroll
                for (int k = 0; k < LOOK; ++k) at[k] = row_at(j0 + (k * 32 + lane) * PER, next[k]);
                pages_of(r + kProdWarps, next);
                wait(B::empty + (int)st, ph ^ 1);
                if (ok) {
                    const uint32_t d0 = sT + st * C::TILE + place * (BN * 128) + (uint32_t)sub * 128;
                    if constexpr (SRC == kGroups) {
#pragma unroll 1
                        for (int q = 0; q < BN / 8; ++q) {
                            const long long first = __shfl_sync(0xffffffffu, at[0], q);
                            const int left = g.s.L - (j0 + q * 8);   // rows of the sequence from here on
                            const __nv_bfloat16* s1 = src + first + mine;
                            if (first >= 0 && left >= 8) {
#pragma unroll
                                for (int k = 0; k < 8; k += RPI)
                                    cp_async16(d0 + (uint32_t)(q * 1024 + k * 128) + (c0 ^ (uint32_t)(k << 4)), s1 + k * stride);
                            } else {
#pragma unroll
                                for (int k = 0; k < 8; k += RPI) {
                                    const bool real = first >= 0 && k + sub < left;
                                    cp_async16_or_zero(d0 + (uint32_t)(q * 1024 + k * 128) + (c0 ^ (uint32_t)(k << 4)), real ? s1 + k * stride : src,
                                                       real);
                                }
                            }
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < BN; k += RPI) {
                            const long long row = __shfl_sync(0xffffffffu, at[k / 32], (k & 31) + sub);
                            cp_async16_or_zero(d0 + (uint32_t)k * 128 + (c0 ^ (uint32_t)((k & 7) << 4)), row < 0 ? src : src + row + mine, row >= 0);
                        }
                    }
                }
                cp_async_arrive(bar(B::full + (int)st));
            }
            pos += (uint32_t)total;
        }
        cp_async_wait_all();
        if (!ok && warp == 0 && q_issued > 0) drain(bar(B::qfull), (q_issued - 1) & 1);
    } else {
        // ---------------------------------------------------------------- MMA
        // The whole warp walks and waits, so that stages and descriptors stay in uniform registers (a lane of its own
        // moves every operand there first: 120 clocks an MMA instead of 64); one lane issues.
        constexpr uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
        constexpr uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
        // Two row tiles: a slot tile's V and the next one's K are waited for, and fenced, while the first unit's softmax
        // runs (behind it the fences stood in the MMAs' way: 150 clocks each).
        constexpr bool EARLY = NT == 2;
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        uint32_t base = 0, units = 0, items = 0;         // tiles and units of the items before; items begun
        bool ok = true;
        auto wait = [&](int b, uint32_t parity) { ok = __all_sync(0xffffffffu, ok && W.wait(bar(b), parity)); };
        while (ok && walk.next(g)) {
            const int n = __shfl_sync(0xffffffffu, g.n, 0), U = n * NT;
            const bool two = __shfl_sync(0xffffffffu, (int)two_terms<D, NT>(P, g), 0);
            auto scores = [&](int u) {
                const int i = u / NT, t = u - i * NT;
                const uint32_t p = base + (uint32_t)(C::NB == 1 ? 2 * i : i == 0 ? 0 : 2 * i - 1), st = p % C::STAGES;
                if (u == 0) wait(B::qfull, items & 1);
                if (t == 0 && !(EARLY && u > 0)) wait(B::full + (int)st, (p / C::STAGES) & 1);
                if (!ok) return;
                if (SRC != kCodes && t == 0 && !(EARLY && u > 0)) fence_proxy_async();
                tc_fence_after();
                const uint32_t d = tm + ((units + u) & 1) * C::S_COL;
                // descriptors count 16-byte units in their low bits: steps along an operand are added
                const uint64_t qd = sw128_desc(sQ + t * (128 * 128)), kd = sw128_desc(sT + st * C::TILE);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        umma_bf16(d, qd + (k >> 2) * (BM * 128 / 16) + (k & 3) * 2, kd + (k >> 2) * (BN * 128 / 16) + (k & 3) * 2, idesc_s, k > 0);
                    if (t == NT - 1) umma_commit(bar(B::empty + st));
                    if (u == U - 1) umma_commit(bar(B::qempty));
                    umma_commit(bar(B::sfull + ((units + u) & 1)));
                }
                __syncwarp();
            };
            scores(0);
            if (U > 1) scores(1);
            for (int u = 0; u < U && ok; ++u) {
                const int i = u / NT, t = u - i * NT;
                const uint32_t gu = units + u;
                const uint32_t p = base + (uint32_t)(C::NB == 1 || i == n - 1 ? 2 * i + 1 : 2 * i + 2), st = p % C::STAGES;
                if (EARLY && t == 0) {
                    wait(B::full + (int)st, (p / C::STAGES) & 1);
                    if (i + 1 < n) wait(B::full + (int)((p + 1) % C::STAGES), ((p + 1) / C::STAGES) & 1);
                    if (SRC != kCodes) fence_proxy_async();
                }
                wait(B::pfull + (int)(gu & 1), (gu >> 1) & 1);
                if (!EARLY && t == 0) wait(B::full + (int)st, (p / C::STAGES) & 1);
                if (!ok) break;
                if (SRC != kCodes && !EARLY && t == 0) fence_proxy_async();
                tc_fence_after();
                const uint64_t vd = mn_desc(sT + st * C::TILE, BN * 128);
                const uint32_t wg = C::COLS ? 0 : gu & 1;
                const uint32_t od = tm + C::O_COL + wg * D, pd = tm + (gu & 1) * C::S_COL;
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < BN / 16; ++k) umma_bf16_ts(od, pd + k * 8, vd + k * (2048 / 16), idesc_o, u >= C::OS || k > 0);
                    if (two)
#pragma unroll
                        for (int k = 0; k < BN / 16; ++k) umma_bf16_ts(od, pd + BN / 2 + k * 8, vd + k * (2048 / 16), idesc_o, 1);
                    if (t == NT - 1) umma_commit(bar(B::empty + st));
                    if (C::OS == 1) umma_commit(bar(B::added));   // phase: the unit
                    if (u >= U - C::OS) umma_commit(bar(B::ofull + wg));
                }
                __syncwarp();
                if (u + 2 < U) scores(u + 2);
            }
            base += 2 * (uint32_t)n;
            units += (uint32_t)U;
            ++items;
        }
        // every MMA issued has completed before TMEM is freed
        if (elect_one()) umma_commit(bar(B::done));
        const unsigned long long t0 = globaltimer();
        while (!mbar_try_wait(bar(B::done), 0) && globaltimer() - t0 < kWaitNs) {}
        __syncwarp();
    }
    } else {
        // ---------------------------------------------------------------- softmax
        if constexpr (SRC == kCodes) regs_take<200>();
        else regs_take<208>();
        const int wg = (warp - 4) >> 2, t = NT == 2 ? wg : 0, quad = warp & 3;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
        const float inv_cap = CAP ? 1.0f / P.cap : 0.0f;
        const float c = CAP ? 1.0f : P.scale * kLog2e;   // factor of the (capped) scores in log2 units
        constexpr bool JOIN = NT == 1 && !C::COLS;       // two warpgroups on one row tile, each with its own slot tiles
        constexpr int CW = C::COLS ? BN / 2 : BN;        // columns of a unit that this thread takes, from c0 on
        const int c0 = C::COLS ? wg * CW : 0, o_col = C::O_COL + (C::COLS ? 0 : wg * D);
        float2* ml = reinterpret_cast<float2*>(smem + 1024) + quad * 32 + lane;
        float* shared_max = reinterpret_cast<float*>(smem + 1024) + quad * 32 + lane;   // [2][128]
        float* shared_sum = reinterpret_cast<float*>(smem + 2048) + quad * 32 + lane;   // [2][128]
        const int my_r = t * 128 + quad * 32 + lane, my_tok = my_r / P.G, my_head = my_r - my_tok * P.G;   // this thread's row of a tile
        uint32_t units = 0, items = 0, filled[2] = {0, 0};   // filled: times each O has been completed
        bool ok = true;                                  // the same in the lanes of a warp
        auto wait = [&](int b, uint32_t parity) { ok = __all_sync(0xffffffffu, ok && W.wait(bar(b), parity)); };
        bool have = false;
        while (walk.next(g)) {
            have = true;
            const int ta = g.rt * (P.tile_rows / P.G);            // the tile's first token
            const int rows = min(P.tile_rows, (g.s.n - ta) * P.G);
            const bool real = my_r < rows;
            // rows without a token see what the last one sees, so that they send no tile the way of masks; nothing is read from them
            const int own = g.s.slot(real ? ta + my_tok : g.s.n - 1 < ta + P.tile_rows / P.G - 1 ? g.s.n - 1 : ta + P.tile_rows / P.G - 1);
            const int hi = min(own + 1, g.s.L), lo = max(window_lo(P, own), 0), pre = g.s.pre;
            const RowId id = {ta + my_tok, g.h * P.G + my_head};
            const int row = g.rt * P.tile_rows + my_r;
            const bool two = two_terms<D, NT>(P, g);
            float* my_scores = nullptr;
            if (NT == 1 && P.scores && real) {
                my_scores = P.scores + ((long long)(g.s.t0 + id.t) * P.Hq + id.head) * P.scores_stride;
            }
            const int U = g.n * NT;
            const int u0 = C::COLS ? 0 : NT == 2 ? t : (int)((units + (uint32_t)wg) & 1);   // this warpgroup's first unit
            float m = -INFINITY, l = 0.0f;
            if (JOIN && wg == 1 && items > 0) wait(B::mlempty, (items - 1) & 1);   // its sums of the last item are read
            for (int u = u0; u < U; u += C::STEP) {
                const int i = u / NT;
                const uint32_t gu = units + (uint32_t)u;
                wait(B::sfull + (gu & 1), (gu >> 1) & 1);
                if (!C::COLS && !ok) break;              // (with shared columns the warps go on to meet at the barriers)
                tc_fence_after();
                const uint32_t at = lanes + (gu & 1) * C::S_COL;
                const int j0 = g.kv.at(g.i0 + i) * BN;
                const bool all = __all_sync(0xffffffffu, (j0 >= lo && j0 + BN <= hi) || j0 + BN <= pre);
                uint32_t x[CW];
#pragma unroll
                for (int k = 0; k < CW; k += 32) tmem_ld32_to(x + k, at + c0 + k);
                tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < CW; k += 32) pin32(x + k);
                auto xf = [&](int k) -> float { return __uint_as_float(x[k]); };
                if constexpr (CAP) {
                    bool near = true;                    // all scores where the series holds: no branch per score
#pragma unroll
                    for (int k = 0; k < CW; ++k) {
                        const float y = xf(k) * (P.scale * inv_cap);
                        near = near && fabsf(y) < 0.5f;
                        x[k] = __float_as_uint(y);
                    }
                    if (__all_sync(0xffffffffu, near)) {
#pragma unroll
                        for (int k = 0; k < CW; ++k) x[k] = __float_as_uint(P.cap * kLog2e * tanh_series(xf(k)));
                    } else {
#pragma unroll
                        for (int k = 0; k < CW; ++k)
                            x[k] = __float_as_uint(P.cap * kLog2e * (fabsf(xf(k)) < 0.5f ? tanh_series(xf(k)) : tanh_far(xf(k))));
                    }
                }
                if (!all) {
#pragma unroll
                    for (int k0 = 0; k0 < CW; k0 += 32) {
                        const uint32_t seen = range_bits(lo, hi, j0 + c0 + k0) | range_bits(0, pre, j0 + c0 + k0);
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (!(seen >> k & 1u)) x[k0 + k] = 0xff800000u;
                    }
                }
                if (NT == 1 && P.scores && real && j0 < P.scores_stride) {   // for the weight sums, in log2 units
                    float4* to = reinterpret_cast<float4*>(my_scores + j0 + c0);
#pragma unroll
                    for (int k = 0; k < CW; k += 4) __stcg(to + k / 4, make_float4(xf(k) * c, xf(k + 1) * c, xf(k + 2) * c, xf(k + 3) * c));
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int k = 0; k < CW; k += 2) top[k >> 1 & 3] = max3(top[k >> 1 & 3], xf(k), xf(k + 1));
                const float mine = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * c;
                float next = fmaxf(m, mine);
                // A row that grew by more than 2^8 (or had seen nothing) takes its new maximum, and its warp with it;
                // with shared columns both warpgroups hold the same maximum and decide together.  Only rows of the
                // sequence have a say: the others hold the next one's queries, or what an earlier kernel left in
                // shared memory, and the result's bits may depend on neither.
                bool grown = __any_sync(0xffffffffu, real && (next > m + 8.0f || (m == -INFINITY && next > m)));
                if constexpr (C::COLS) {
                    grown = group_any(4, 256, grown && ok);
                    if (grown) {
                        shared_max[wg * 128] = mine;
                        group_sync(4, 256);
                        next = fmaxf(next, shared_max[(wg ^ 1) * 128]);
                    }
                }
                if (grown) {
                    const float w = next == -INFINITY ? 1.0f : exp2_hw(m - next);
                    m = next;
                    l *= w;
                    if (u >= C::OS) {
                        // The product that last added to this O must be complete.  With two O it is the one of unit u - 2,
                        // issued before S(u); with one it is that of unit u - 1, issued after S(u) (and the next waits for
                        // this unit's P, so that the barrier is at most one phase ahead).
                        if constexpr (C::OS == 1) {
                            wait(B::added, (gu - 1) & 1);
                            tc_fence_after();
                        }
#pragma unroll 1
                        for (int k = C::COLS ? wg * (D / 2) : 0; k < (C::COLS ? (wg + 1) * (D / 2) : D); k += 16) {
                            uint32_t o[16];
                            tmem_ld16(lanes + o_col + k, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * w);
                            tmem_st16(lanes + o_col + k, o);
                        }
                    }
                }
                const float base = m == -INFINITY ? 0.0f : m;
                const float2 c2 = make_float2(c, c), b2 = make_float2(-base, -base);
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                // S is in registers by now, so P can begin to take its place
                auto weights = [&](int k) {
                    float2 y = fma2(make_float2(xf(k), xf(k + 1)), c2, b2);
                    y.x = exp2_hw(y.x);
                    y.y = exp2_hw(y.y);
                    sum[k >> 1 & 1] = add2(sum[k >> 1 & 1], y);
                    return y;
                };
                constexpr int STORE = CW < 64 ? CW : 64;   // columns of S whose P goes out with one store
                if (two) {
#pragma unroll
                    for (int k0 = 0; k0 < CW; k0 += STORE) {
                        uint32_t low[STORE / 2];
#pragma unroll
                        for (int k = 0; k < STORE; k += 2) {
                            const float2 y = weights(k0 + k);
                            const uint32_t w = pack_bf16(y.x, y.y);
                            x[(k0 + k) >> 1] = w;
                            low[k >> 1] = pack_bf16(y.x - bf_lo(w), y.y - bf_hi(w));
                        }
                        store_p<STORE / 2>(at + (c0 + k0) / 2, x + k0 / 2);
                        store_p<STORE / 2>(at + (BN + c0 + k0) / 2, low);
                    }
                } else {
#pragma unroll
                    for (int k0 = 0; k0 < CW; k0 += STORE) {
#pragma unroll
                        for (int k = 0; k < STORE; k += 2) {
                            const float2 y = weights(k0 + k);
                            x[(k0 + k) >> 1] = pack_bf16(y.x, y.y);
                        }
                        store_p<STORE / 2>(at + (c0 + k0) / 2, x + k0 / 2);
                    }
                }
                const float2 s2 = add2(sum[0], sum[1]);
                l += s2.x + s2.y;
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(B::pfull + (gu & 1)));
            }
            const int u1 = u0 ^ 1;                           // the other warpgroup's first unit (a slot tile each)
            units += (uint32_t)U;
            if (ok && u0 < U) wait(B::ofull + (C::COLS ? 0 : wg), filled[0] & 1);
            filled[0] += u0 < U;
            bool other = false;                              // join: the other warpgroup has sums, too
            float w0 = 1.0f, w1 = 0.0f;
            if constexpr (JOIN) {
                if (wg == 1) {
                    *ml = make_float2(m, l);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(B::mlfull));
                    ++items;
                    continue;
                }
                if (ok) wait(B::mlfull, items & 1);
                other = u1 < U;
                if (ok && other) wait(B::ofull + 1, filled[1] & 1);
                filled[1] += other;
                const float2 x = *ml;
                const float top = fmaxf(m, x.x), base = top == -INFINITY ? 0.0f : top;
                w0 = exp2_hw(m - base);
                w1 = exp2_hw(x.x - base);
                l = l * w0 + x.y * w1;
                m = top;
            }
            if constexpr (C::COLS) {                         // the sums of both halves, added alike
                shared_sum[wg * 128] = l;
                group_sync(4, 256);
                l = shared_sum[0] + shared_sum[128];
            }
            ++items;
            tc_fence_after();
            const bool whole = g.whole();
            const float inv = whole ? (l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l)) : 1.0f;
            const float lse2 = l == 0.0f ? -INFINITY : m + log2f(l);
            const int quad_rows = rows - (my_r & ~3);        // real rows from the first of this lane's four on
            const long long out_row = (long long)(g.s.t0 + id.t) * P.o_t + (long long)id.head * P.o_h;
            long long out_of[4];                             // where the four rows' outputs begin
#pragma unroll
            for (int r = 0; r < 4; ++r) out_of[r] = __shfl_sync(0xffffffffu, out_row, (lane & ~3) + r);
            const size_t part = (size_t)(2 * blockIdx.x + (g.first ? 0 : 1)) * BM + my_r;
            bool fine = true;
            if (ok) {
#pragma unroll 1                                             // short code: a cold instruction cache costs small calls most
                for (int k = C::COLS ? wg * (D / 2) : 0; k < (C::COLS ? (wg + 1) * (D / 2) : D); k += 32) {
                    uint32_t o[32];
                    if (!JOIN || u0 < U) {
                        tmem_ld32(lanes + o_col + k, o);
                        tmem_ld_wait();
                    }
                    if constexpr (JOIN) {
                        uint32_t o1[32];
                        if (other) {
                            tmem_ld32(lanes + C::O_COL + D + k, o1);
                            tmem_ld_wait();
                        }
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            o[e] = __float_as_uint((u0 < U ? __uint_as_float(o[e]) * w0 : 0.0f) + (other ? __uint_as_float(o1[e]) * w1 : 0.0f));
                    }
                    // Four lanes exchange chunks, so that a store writes 64 bytes of each of 8 rows (a row a lane: 16 of 32)
                    if (whole) {
                        uint32_t v[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            const float y0 = l == 0.0f ? 0.0f : __uint_as_float(o[e]) * inv, y1 = l == 0.0f ? 0.0f : __uint_as_float(o[e + 1]) * inv;
                            fine = fine && fabsf(y0) <= 3.0e38f && fabsf(y1) <= 3.0e38f;
                            v[e >> 1] = pack_bf16(y0, y1);
                        }
                        transpose_quad(v);
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (quad_rows > r)
                                *reinterpret_cast<uint4*>((__nv_bfloat16*)P.out + out_of[r] + k + (lane & 3) * 8) =
                                    make_uint4(v[r * 4], v[r * 4 + 1], v[r * 4 + 2], v[r * 4 + 3]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 16) {
                            uint32_t v[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) v[i] = o[e + i];
                            transpose_quad(v);
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (quad_rows > r)
                                    __stcg(reinterpret_cast<uint4*>(P.part_o + (part - (lane & 3) + r) * D + k + e + (lane & 3) * 4),
                                           make_uint4(v[r * 4], v[r * 4 + 1], v[r * 4 + 2], v[r * 4 + 3]));
                        }
                    }
                    __syncwarp();
                }
            }
            tc_fence_before();
            if constexpr (JOIN) {
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(B::mlempty));
            }
            if (whole) {
                if (real && P.lse && !(C::COLS && wg)) P.lse[(long long)(g.s.t0 + id.t) * P.Hq + id.head] = lse2 * kLn2;
                for (uint32_t bad = __ballot_sync(0xffffffffu, real && !fine && l == l); bad; bad &= bad - 1) {
                    const int who = __ffs(bad) - 1;
                    float o[D / 32];
                    resum_row<__nv_bfloat16, D>(P, g.s, g.b, g.h, row - lane + who, __shfl_sync(0xffffffffu, lse2, who), o, beat);
                    const RowId bid = row_id(P, g.s, g.h, row - lane + who);
                    if (!C::COLS || lane >> 4 == wg)         // a half of the channels is this warpgroup's
                        store_f32<__nv_bfloat16, D / 32>((__nv_bfloat16*)P.out + (long long)(g.s.t0 + bid.t) * P.o_t + (long long)bid.head * P.o_h +
                                                             lane * (D / 32), o);
                }
            } else {
                if (real && !(C::COLS && wg)) __stcg(P.part_ml + part, make_float2(m, l));
            }
        }
        if (threadIdx.x == 128) leave_split(P, *plan, g, have);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tmem_relinquish();
        tmem_dealloc(tmem, C::TMEM);
    }
}

template <int D, int NT, Source SRC, bool CAP> cudaError_t start_tc(const AttendParams& P, const CUtensorMap& q_map, int num_sms, cudaStream_t stream)
{
    using C = TcShape<D, NT, SRC == kCodes>;
    const int grid = min(num_sms, kAttendMaxRows / C::BM / 2);
    if (cudaError_t e = smem_opt_in<attend_tc_kernel<D, NT, SRC, CAP>>(C::SMEM); e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaError_t e = cudaLaunchKernelEx(&cfg, attend_tc_kernel<D, NT, SRC, CAP>, P, q_map); e != cudaSuccess) return e;
    return run_join<__nv_bfloat16, D, C::BM>(P, grid, stream);
}
template <int D, int NT, bool CAP, bool CODES> cudaError_t run_tc(const AttendParams& call, int num_sms, cudaStream_t stream)
{
    using C = TcShape<D, NT>;
    AttendParams P = call;
    P.tile_rows = C::BM / P.G * P.G;               // whole tokens: with 7 query heads a KV head 126 or 252 rows
    CUtensorMap q_map;                             // (channel, head, token), boxes of 64 channels of a row tile
    const EncodeTiled enc = tiled_encoder();
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)P.Hq, (cuuint64_t)P.T};
    const cuuint64_t strides[2] = {(cuuint64_t)P.q_h * 2, (cuuint64_t)P.q_t * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)P.G, (cuuint32_t)(C::BM / P.G)}, one[3] = {1, 1, 1};
    if (!enc || enc(&q_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(P.q), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    if constexpr (CODES) return start_tc<D, NT, kCodes, CAP>(P, q_map, num_sms, stream);
    else if (!P.cache.paged || P.cache.page_size % 8 == 0) return start_tc<D, NT, kGroups, CAP>(P, q_map, num_sms, stream);
    else return start_tc<D, NT, kRows, CAP>(P, q_map, num_sms, stream);
}
template <bool CAP, bool CODES = false> cudaError_t run_attend_tc(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    const bool one = one_tile(P);
    if (P.d == 64) return one ? run_tc<64, 1, CAP, CODES>(P, num_sms, stream) : run_tc<64, 2, CAP, CODES>(P, num_sms, stream);
    if (P.d == 128) return one ? run_tc<128, 1, CAP, CODES>(P, num_sms, stream) : run_tc<128, 2, CAP, CODES>(P, num_sms, stream);
    return run_tc<256, 1, CAP, CODES>(P, num_sms, stream);
}

}  // namespace
}  // namespace kvx
