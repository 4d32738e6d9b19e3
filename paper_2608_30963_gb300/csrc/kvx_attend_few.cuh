// kvx_attend_few.cuh -- attention of few new tokens over an 8-bit cache on the tensor cores, its codes multiplied as they are
// (library-internal; tcgen05 kind::f8f6f4).  Compiled twice, with and without the capped scores' code.
//
//   S^T = K (Qh + Ql / 16)^T,   P = exp2(f S^T - m),   O^T += V^T (P1 + P2 / 32 + P3 / 1024)
// With few rows (query heads of a token) the products have room to spare, and what costs is bringing K and V: so the
// cache's codes are the operands, straight from memory, and the other side is split into e4m3 terms that make up for its
// 4 bits.  A query row is scaled by a power of two and split in two (bf16's 8 bits exactly, down to 2^-14 of the row's largest
// value, below that to 2^-22 of it), a weight in three (to 2^-12 of itself, 2^-23 of the largest of some thousand slots).  Terms lie side by
// side as columns of one product; sums are fp32.  Slots are the rows of S^T and channels those of O^T, so the rows of a tile
// are its columns: 256 slots by 8, 16 or 32 rows.
//   copying warps (7)   128-byte blocks of K and V rows into 128-byte-swizzled tiles, every seventh each
//   MMA warp            tile i: S(i + 2) into S(i)'s place once that has been read; O of warpgroup i mod 2 += V P(i) when P(i) is there
//   softmax warps (8)   two warpgroups, every other tile each; a thread has a slot.  A score x takes its K row's scale; a weight
//                       takes its V row's, in its exponent, z = x + log2 of it, and a reference n of its own beside the sums'
//                       reference m, so that far scales do not leave e4m3's range.  A row takes new references when z has grown by
//                       more than 1 (a factor of two) beyond n, or x by 64 beyond m (sums in fp32 have room), and every 32 tiles
//                       of the warpgroup, down as well as up; each has its own references, sums and O, joined at the end.
// The last rows of the split work are joined as those of the other attention kernels.
//
// What bounds it.  8 rows: the reading of K and V.  Long ranges run at a copy's rate (a token of each of 38 sequences over 65001 slots, 7
// query heads on each of 4 KV heads of 128, 2.55 GB, 378 us, 6.7 TB/s); where a CTA has some twenty tiles what comes before and
// after them shows (eight sequences of up to 32768 slots, 207 MB, 47 us, 4.4 TB/s: 31 us at that rate, 16 the plan, the first reads,
// the ends and the join).  16 and 32 rows: the softmax warps (two exponentials
// and three terms a weight): 4 tokens of 8 query heads on each of 8 KV heads over up to 16384 slots of four sequences, 111 MB, 56 us, over
// 32000 slots of 19, 1.26 GB, 256 us, 4.9 TB/s; the schedulers issue in 34% of a launch's clocks, and for each instruction issued a
// warp waits 1.4 at barriers and 1.0 for code to arrive.  (32 rows, four sequences of 16384 slots, 63 us: with four softmax warpgroups, two on a tile's rows, 69; with references agreed on
// while the weights are taken, 79; with one exponential, times a factor, for the two, no less.)  Short calls: latency,
// 12 us from launch to end.  (The first case with 128 slots a tile and the scales read by the softmax threads, whose reads take as long
// as the copies on their way, 54 us; with P stored byte by byte, 57; with the rows' ends unrolled, a code that is always
// cold, 52.)
#pragma once

#include "kvx_attend_rows.cuh"
#include "kvx_kernels.h"
#include "kvx_umma.cuh"

namespace kvx {
namespace {

template <int D, int R> struct FewShape {
    // A tile has 256 slots, two a thread (what a tile costs anyway, and the latencies, shared by two: with 128 a token each of 8
    // sequences over up to 32768 slots took 54 us, and 46 with no tile copied at all), or 128 where TMEM has no room for more.
    static constexpr int HB = D == 256 && R == 32 ? 1 : 2, BN = 128 * HB, DB = D / 128;   // halves of a tile; 128-channel blocks of a head
    static constexpr int NQ = 2 * R, NP = (3 * R + 31) / 32 * 32;  // columns of S^T and of O^T
    static constexpr int UNIT = 128 * 128, UNITS = HB * DB;    // a block of half a K or V tile; units of a tile
    static constexpr int CTRL = 7168, QB = NQ * 128 * DB, PB = BN * NP;
    // Scales of a tile's K and V rows, 8 tiles: a unit of tile i + 8 is copied only when a later one than V's of tile i has been
    // multiplied (11 tiles of K or V lie between them, more than the ring holds).
    static constexpr int TURNS = 8, SCALES = TURNS * 2 * BN;
    static constexpr int FIT = (kSmemMax - CTRL - QB - 2 * PB - SCALES) / UNIT, STAGES = FIT < 12 ? FIT : 12;
    static constexpr int SMEM = CTRL + STAGES * UNIT + QB + 2 * PB + SCALES;
    static constexpr int THREADS = 512, COPY = 7;
    static constexpr int O_COL = 2 * HB * NQ;                  // TMEM columns: S^T of even and odd tiles, then O^T of each
    static constexpr int USED = O_COL + 2 * NP * DB, TMEM = USED <= 128 ? 128 : USED <= 256 ? 256 : 512;
    static_assert(SMEM <= kSmemMax && USED <= 512 && COPY <= STAGES && 2 * UNITS <= STAGES && STAGES <= 11 * UNITS);
    static_assert((kMaxAttendBatch + 2) * 8 <= STAGES * UNIT);
    // the control block: barriers up to 512, plan and states up to 1024, then rows' tables
    static constexpr int SEES = 1024, REF = SEES + 32 * 16, LESS = REF + 2 * 32 * 16, RED = LESS + 2 * 32 * 8, SUM = RED + 2 * 4 * 32 * 8,
                         BAD = SUM + 2 * 4 * 32 * 4;
    static_assert(BAD + 8 * 4 <= CTRL);
};

// D[tmem] (+)= A[smem] . B[smem], e4m3 inputs, fp32 accumulate
__device__ __forceinline__ void umma_e4m3(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// N columns of the warp's lanes
template <int N> __device__ __forceinline__ void tmem_load(uint32_t at, uint32_t (&v)[N])
{
    static_assert(N == 4 || N == 8);
    if constexpr (N == 8) tmem_ld8(at, v);
    else asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at));
}
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t (&v)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
// Two values rounded to e4m3, and `by` times what that leaves of them.
__device__ __forceinline__ uint32_t take_term(float2& y, float by)
{
    const uint32_t t = to_codes(y.x, y.y);
    y = fma2(codes_f32((unsigned short)t), make_float2(-by, -by), mul2(y, make_float2(by, by)));     // (exact)
    return t;
}
// MN-major operand in blocks of 32 bytes a row, 32-byte-swizzled: lbo between the blocks, 256 bytes between 8-row groups.
__device__ __forceinline__ uint64_t mn32_desc(uint32_t saddr, uint32_t lbo)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)((lbo >> 4) & 0x3FFFu) << 16 | (uint64_t)(256u >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)6 << 61;
}

// A row of a tile sees the slots [lo, hi) and [0, pre).
struct __align__(16) FewSees {
    int lo, hi, pre;
};
// The factor of its scores, and a warpgroup's references (log2 units): m of x, and d = 7 + m - n, so that a weight is exp2((x - m) +
// (log2 of V's scale + d)): its exponent is a sum of small numbers however large the scores are.  What x has not been seen yet has
// kNoRef (not an infinity, so that differences are numbers).
// n follows the weights up at once, and down every kLower tiles of a warpgroup: the third term of a weight ends at 2^-23 of the
// largest that n was taken for, and without a way down a long tail of smaller ones behind it would be lost (of 524288 slots of
// 2^-23.6 each all that this warpgroup has).  O is fp32 and has room for weights that are small beside what it holds, so n may lie up
// to kLowest below the largest it has been (`low` says how much; not below kDeepest beside m: 2^-d has to be a normal number).
// What a row loses to the terms' end is then at most the slots of kLower tiles (8192) times 2^-23 of the largest contribution that
// their reference was taken for, 2^-10 of that, however many slots follow.  (4 tokens of 8 query heads on each of 8 KV heads over
// 32000 slots of 19 sequences, us with a way down every 16 and 32 tiles and without one: 260, 256 and 251.)
struct __align__(16) FewRef {
    float f, m, d, low;
};
constexpr int kLower = 32;
constexpr float kLowest = 24.0f, kDeepest = -100.0f;
constexpr float kNoRef = -3.0e38f;
// The end of a row.
struct FewEnd {
    long long to;          // element of the output
    float a, b;            // factors of both warpgroups' O
    float lse2, sum;
};
// Row `row` of an item whose query holds an infinity and no NaN: e4m3 has no infinity, so its scores came out NaN, but they are
// infinite, or numbers where they are capped.  One warp takes its maximum, sum and output along the segment's slots in fp32 (up
// to the first score that is NaN; about 1 us a slot) and writes it, or its part of a split row's.
template <int D, int BN>
__device__ __noinline__ void infinite_row(const AttendParams& P, const Segment& g, int row, size_t part, volatile int* beat)
{
    constexpr int C = D / 32;
    const int lane = threadIdx.x & 31;
    const RowId id = row_id(P, g.s, g.h, g.rt * P.tile_rows + row);
    const long long token = g.s.t0 + id.t;
    float q[C], x[C], o[C], m = -INFINITY, l = 0.0f;
    load_f32<__nv_bfloat16, C>((const __nv_bfloat16*)P.q + token * P.q_t + (long long)id.head * P.q_h + lane * C, q);
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] = 0.0f;
    const int i = g.s.slot(id.t);
    const float inv_cap = P.cap > 0.0f ? 1.0f / P.cap : 0.0f;
    for (int t = 0; t < g.n && l == l; ++t) {
        if ((t & 7) == 0 && lane == 0) *beat = *beat + 1;          // waits elsewhere in the CTA go on
        const int j0 = g.kv.at(g.i0 + t) * BN;
        for (int j = j0; j < min(j0 + BN, g.s.L) && l == l; ++j) {
            if (!sees(P, g.s, i, j)) continue;
            const CodePlace at = code_place(P.cache, P.scales, g.b, j);
            const long long off = at.row + cache_head(P.cache) * g.h + lane * C, scale = at.scale + scale_head(P.cache, P.scales) * g.h;
            auto load = [&](const void* rows, const unsigned char* scales) {
#pragma unroll
                for (int c = 0; c < C; ++c) x[c] = 0.0f;           // (pages that are not in the pool)
                if (at.row >= 0) load_codes<C>((const uint8_t*)rows + off, scale_of(scales[scale]), x);
            };
            load(P.ck, P.k_scale);
            float dot = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c) dot = fmaf(q[c], x[c], dot);
#pragma unroll
            for (int k = 16; k; k >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, k);
            float v = dot * P.scale;
            if (P.cap > 0.0f) v = capped(v, P.cap, inv_cap);
            v *= kLog2e;
            const float next = fmaxf(m, v), base = next == -INFINITY ? 0.0f : next, w = exp2_hw(m - base), p = exp2_hw(v - base);
            m = next;
            l = fmaf(l, w, p);
            load(P.cv, P.v_scale);
#pragma unroll
            for (int c = 0; c < C; ++c) o[c] = fmaf(p, x[c], o[c] * w);
        }
    }
    if (g.whole()) {
        const float inv = l > 0.0f ? 1.0f / l : l;                 // (NaN stays)
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] = l == 0.0f ? 0.0f : o[c] * inv;
        store_f32<__nv_bfloat16, C>((__nv_bfloat16*)P.out + token * P.o_t + (long long)id.head * P.o_h + lane * C, o);
        if (P.lse && lane == 0) P.lse[token * P.Hq + id.head] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c) __stcg(P.part_o + part * D + lane * C + c, o[c]);
        if (lane == 0) __stcg(P.part_ml + part, make_float2(m, l));
    }
}
constexpr float kAhead = 4.0f;   // references are taken so far above the largest, so that they last (a tile with new ones costs 1200 clocks)
__device__ __forceinline__ float warp_max(float x)
{
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}

template <int D, int R, bool GROUPS, bool CAP>
__global__ void __launch_bounds__(512, 1) attend_few_kernel(const __grid_constant__ AttendParams P)
{
    using C = FewShape<D, R>;
    constexpr int BN = C::BN, DB = C::DB, HB = C::HB;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t s0 = smem_u32(smem);
    constexpr int kFull = 0, kEmpty = C::STAGES, kS = 2 * C::STAGES, kP = kS + 2, kO = kP + 2, kFree = kO + 2, kScale = kFree + 2, kQ = kScale + C::TURNS, kDone = kQ + 1;
    static_assert(8 * (kDone + 1) <= 512);
    auto bar = [&](int i) { return s0 + (uint32_t)i * 8; };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + 512);
    int* abort = reinterpret_cast<int*>(smem + 516);
    int* beat = reinterpret_cast<int*>(smem + 520);
    const uint32_t sT = s0 + C::CTRL, sQ = sT + C::STAGES * C::UNIT, sP = sQ + C::QB;
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (warp == 3) tmem_alloc(smem_u32(tmem_slot), C::TMEM);
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) {
            mbar_init(bar(kFull + i), 32);
            mbar_init(bar(kEmpty + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(kS + i), 1);
            mbar_init(bar(kP + i), 4);
            mbar_init(bar(kO + i), 1);
            mbar_init(bar(kFree + i), 4);
        }
        for (int i = 0; i < C::TURNS; ++i) mbar_init(bar(kScale + i), 2 * HB);
        mbar_init(bar(kQ), 8);
        mbar_init(bar(kDone), 1);
        fence_mbar_init();
        *abort = 0;
        *beat = 0;
    }
    // the kernel before this one may still be ending: what it wrote is read from here on
    grid_dependency_wait();
    grid_launch_dependents();
    const Plan mine_plan = make_plan<BN, C::THREADS>(P, reinterpret_cast<long long*>(smem + C::CTRL));
    Plan* plan = reinterpret_cast<Plan*>(smem + 544);
    if (threadIdx.x == 0) *plan = mine_plan;
    WalkState* state = reinterpret_cast<WalkState*>(smem + 640) + warp;
    static_assert(sizeof(Plan) <= 96 && sizeof(WalkState) * (C::THREADS / 32) <= 1024 - 640);
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const BeatWaiter W{abort, beat, P.status};
    SegmentWalk<BN> walk(P, plan, state);
    Segment g;
    bool ok = true;
    auto wait = [&](int b, uint32_t parity) { ok = __all_sync(0xffffffffu, ok && W.wait(bar(b), parity)); };

    if (warp < 4 || warp >= 12) {
        regs_give<56>();
        if (warp != 3) {
            // ---------------------------------------------------------------- copies
            const int me = warp < 3 ? warp : warp - 9, sub = lane >> 3;        // a row of an instruction: 8 lanes
            const uint32_t c0 = (uint32_t)(((lane & 7) ^ sub) << 4);
            uint8_t* scale_to = smem + C::SMEM - C::SCALES;
            uint32_t pos = 0;                            // units of the items before
            constexpr int PER = GROUPS ? 8 : 1, FIND = 128 / PER, LOOK = (FIND + 31) / 32;
            const long long stride = P.cache.paged ? (long long)P.cache.H * D : P.cache.st, per_page = (long long)P.cache.H * P.cache.page_size;
            while (walk.next(g)) {
                const int total = 2 * g.n, all = total * C::UNITS;
                const long long mine = cache_head(P.cache) * g.h + (PER > 1 ? sub * stride : 0) + (lane & 7) * 16;
                // First slot of unit r of the item in the order of the ring, in which the MMA warp takes them (so that a wait for an empty one by
                // parity cannot pass a phase early): K0 K1 K2 V0 K3 V1 .. and the last three V.
                auto tile_of = [&](int r, int& kv, int& i) {
                    const int x = r / C::UNITS, end = max(total - 2, g.n);
                    kv = x >= end || (x >= 3 && (x & 1));
                    i = x >= end ? x - g.n : x < 3 ? x : kv ? (x - 3) >> 1 : (x >> 1) + 1;
                    return g.kv.at(g.i0 + i) * BN + (r - x * C::UNITS) / DB * 128;
                };
                auto pages_of = [&](int r, int (&x)[LOOK]) {
                    int kv, i;
                    const int j0 = r < all ? tile_of(r, kv, i) : g.s.L;
#pragma unroll
                    for (int k = 0; k < LOOK; ++k) {
                        const int j = j0 + (k * 32 + lane) * PER;
                        x[k] = -2;                       // past the end
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
                int r = (int)((C::COPY + (uint32_t)me - pos % C::COPY) % C::COPY);
                pages_of(r, next);
                for (; r < all; r += C::COPY) {
                    int kv, tile;
                    const int j0 = tile_of(r, kv, tile);
                    const uint8_t* src = (const uint8_t*)(kv ? P.cv : P.ck) + (r % DB) * 128;
                    const uint32_t p = pos + (uint32_t)r, st = p % C::STAGES, ph = (p / C::STAGES) & 1;
                    long long at[LOOK];
#pragma unroll
                    for (int k = 0; k < LOOK; ++k) at[k] = row_at(j0 + (k * 32 + lane) * PER, next[k]);
                    // the scales of a half tile's rows, four a lane, with its first block
                    const bool with_scales = r % DB == 0;
                    uint32_t scale[4] = {};
                    if (with_scales) {
                        const unsigned char* from = (kv ? P.v_scale : P.k_scale) + scale_head(P.cache, P.scales) * g.h;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int j = j0 + k * 32 + lane, page = GROUPS ? __shfl_sync(0xffffffffu, next[0], k * 4 + (lane >> 3)) : next[LOOK == 1 ? 0 : k];
                            if (j >= g.s.L) continue;
                            if (!P.cache.paged) scale[k] = from[(long long)g.b * P.scales.sb + j];
                            else if (page >= 0 && page < P.cache.num_pages)
                                scale[k] = from[per_page * (unsigned)page + (P.cache.page_shift >= 0 ? j & (P.cache.page_size - 1) : j % P.cache.page_size)];
                        }
                    }
                    pages_of(r + C::COPY, next);
                    wait(kEmpty + (int)st, ph ^ 1);
                    if (!ok) break;
                    const uint32_t d0 = sT + st * C::UNIT + (uint32_t)sub * 128;
                    if constexpr (GROUPS) {
#pragma unroll 4
                        for (int q = 0; q < 16; ++q) {
                            const long long first = __shfl_sync(0xffffffffu, at[0], q);
                            const int left = g.s.L - (j0 + q * 8);
                            const uint8_t* s1 = src + first + mine;
                            if (first >= 0 && left >= 8) {
#pragma unroll
                                for (int k = 0; k < 8; k += 4) cp_async16(d0 + (uint32_t)(q * 1024 + k * 128) + (c0 ^ (uint32_t)(k << 4)), s1 + k * stride);
                            } else {
#pragma unroll
                                for (int k = 0; k < 8; k += 4) {
                                    const bool real = first >= 0 && k + sub < left;
                                    cp_async16_or_zero(d0 + (uint32_t)(q * 1024 + k * 128) + (c0 ^ (uint32_t)(k << 4)), real ? s1 + k * stride : src, real);
                                }
                            }
                        }
                    } else {
#pragma unroll 4
                        for (int k = 0; k < 128; k += 4) {
                            const long long row = __shfl_sync(0xffffffffu, at[k / 32], (k & 31) + sub);
                            cp_async16_or_zero(d0 + (uint32_t)k * 128 + (c0 ^ (uint32_t)((k & 7) << 4)), row < 0 ? src : src + row + mine, row >= 0);
                        }
                    }
                    cp_async_arrive(bar(kFull + (int)st));
                    if (with_scales) {
                        const uint32_t turn = (pos / (2 * C::UNITS) + (uint32_t)tile) % C::TURNS;
                        uint8_t* to = scale_to + (turn * 2 + (uint32_t)kv) * BN + (r % C::UNITS) / DB * 128 + lane;
#pragma unroll
                        for (int k = 0; k < 4; ++k) to[k * 32] = (uint8_t)scale[k];
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(kScale + (int)turn));
                    }
                }
                pos += (uint32_t)all;
            }
            cp_async_wait_all();
        } else {
            // ---------------------------------------------------------------- MMA
            constexpr uint32_t idesc_s = (1u << 4) | ((uint32_t)(C::NQ >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
            constexpr uint32_t idesc_o = (1u << 4) | (1u << 15) | (1u << 16) | ((uint32_t)(C::NP >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
            const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
            uint32_t base = 0, tiles = 0, items = 0;     // units and tiles of the items before; items begun
            while (ok && walk.next(g)) {
                const int n = __shfl_sync(0xffffffffu, g.n, 0);
                wait(kQ, items & 1);
                auto scores = [&](int i) {
                    const uint32_t p = base + (uint32_t)(i < 3 ? i : 2 * i - 2) * C::UNITS, d = tm + ((tiles + i) & 1) * (HB * C::NQ);
#pragma unroll
                    for (int x = 0; x < C::UNITS; ++x) wait(kFull + (int)((p + x) % C::STAGES), ((p + x) / C::STAGES) & 1);
                    if (!ok) return;
                    fence_proxy_async();
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int x = 0; x < C::UNITS; ++x) {
                            const uint64_t kd = sw128_desc(sT + (p + x) % C::STAGES * C::UNIT), qd = sw128_desc(sQ + x % DB * (C::NQ * 128));
#pragma unroll
                            for (int k = 0; k < 4; ++k) umma_e4m3(d + x / DB * C::NQ, kd + k * 2, qd + k * 2, idesc_s, x % DB > 0 || k > 0);
                            umma_commit(bar(kEmpty + (int)((p + x) % C::STAGES)));
                        }
                        umma_commit(bar(kS + (int)((tiles + i) & 1)));
                    }
                    __syncwarp();
                };
                scores(0);
                if (n > 1) scores(1);
                for (int i = 0; i < n && ok; ++i) {
                    const uint32_t gu = tiles + (uint32_t)i, wg = gu & 1;
                    // S(i) has been read: its place is S(i + 2)'s
                    wait(kFree + (int)wg, (gu >> 1) & 1);
                    if (ok && i + 2 < n) scores(i + 2);
                    const uint32_t p = base + (uint32_t)(i >= n - 2 ? n + i : 2 * i + 3) * C::UNITS;
#pragma unroll
                    for (int x = 0; x < C::UNITS; ++x) wait(kFull + (int)((p + x) % C::STAGES), ((p + x) / C::STAGES) & 1);
                    fence_proxy_async();
                    wait(kP + (int)wg, (gu >> 1) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int x = 0; x < C::UNITS; ++x) {
                            const uint64_t vd = mn_desc(sT + (p + x) % C::STAGES * C::UNIT, C::UNIT), pd = mn32_desc(sP + wg * C::PB + x / DB * 4096, BN * 32);
                            const uint32_t od = tm + C::O_COL + (wg * DB + x % DB) * C::NP;
#pragma unroll
                            for (int k = 0; k < 4; ++k) umma_e4m3(od, vd + k * (4096 / 16), pd + k * (1024 / 16), idesc_o, i >= 2 || x / DB > 0 || k > 0);
                            umma_commit(bar(kEmpty + (int)((p + x) % C::STAGES)));
                        }
                        umma_commit(bar(kO + (int)wg));
                    }
                    __syncwarp();
                }
                base += 2 * (uint32_t)n * C::UNITS;
                tiles += (uint32_t)n;
                ++items;
            }
            // every MMA issued has completed before TMEM is freed
            if (elect_one()) umma_commit(bar(kDone));
            const unsigned long long t0 = globaltimer();
            while (!mbar_try_wait(bar(kDone), 0) && globaltimer() - t0 < kWaitNs) {}
            __syncwarp();
        }
    } else {
        // ---------------------------------------------------------------- softmax
        regs_take<200>();
        const int sw = warp - 4, wg = sw >> 2, quad = warp & 3, slot = quad * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
        const float inv_cap = CAP ? 1.0f / P.cap : 0.0f;
        FewSees* sees_of = reinterpret_cast<FewSees*>(smem + C::SEES);           // [32]
        FewRef* refs = reinterpret_cast<FewRef*>(smem + C::REF);                 // [warpgroup][32]
        FewRef* ref = refs + wg * 32;
        float2* less = reinterpret_cast<float2*>(smem + C::LESS) + wg * 32;      // what sums and O are multiplied by
        float2* red = reinterpret_cast<float2*>(smem + C::RED) + wg * 4 * 32;    // [warp][32]
        float* sums = reinterpret_cast<float*>(smem + C::SUM);                   // [warpgroup][warp][32]
        uint32_t* bad = reinterpret_cast<uint32_t*>(smem + C::BAD);              // [warp]
        FewEnd* ends = reinterpret_cast<FewEnd*>(smem + C::RED);                 // [32] (when no maxima are exchanged)
        // where this thread's slot of P lies: 32 bytes in each block of 32 columns, their 16-byte halves exchanged every fourth slot
        const uint32_t p_row = sP + wg * C::PB + (uint32_t)slot * 32, p_swap = (uint32_t)(slot >> 2 & 1) << 4;
        uint32_t tiles = 0, done = 0;                    // tiles of the items before; products of this warpgroup waited for
        bool have = false;
        while (walk.next(g)) {
            have = true;
            const int ta = g.rt * (P.tile_rows / P.G), rows = min(P.tile_rows, (g.s.n - ta) * P.G);
            // the queries' terms, a row a warp, and what the rows see
            uint32_t odd_rows = 0;                       // this warp's whose queries hold infinities
            for (int r = sw; r < R; r += 8) {
                constexpr int CH = D / 32;               // channels of a lane
                float q[CH];
                const RowId id = row_id(P, g.s, g.h, g.rt * P.tile_rows + r);
#pragma unroll
                for (int c = 0; c < CH; ++c) q[c] = 0.0f;
                if (r < rows) load_f32<__nv_bfloat16, CH>((const __nv_bfloat16*)P.q + (long long)(g.s.t0 + id.t) * P.q_t + (long long)id.head * P.q_h + lane * CH, q);
                float top = 0.0f;
                bool infinite = false, none = false;
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    infinite = infinite || fabsf(q[c]) == INFINITY;
                    none = none || q[c] != q[c];
                    if (!(fabsf(q[c]) <= 3.402823466e38f)) q[c] = __uint_as_float(0x7fffffffu);   // (its scores are NaN; infinities: infinite_row)
                    top = fmaxf(top, fabsf(q[c]));
                }
                if (__any_sync(0xffffffffu, infinite) && !__any_sync(0xffffffffu, none)) odd_rows |= 1u << r;
#pragma unroll
                for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const unsigned s = scale_for(top);
                const float inv = inv_scale(s);
                uint32_t hi[CH / 4], lo[CH / 4];
#pragma unroll
                for (int c = 0; c < CH; c += 2) {
                    float2 y = make_float2(q[c] * inv, q[c + 1] * inv);
                    const uint32_t h = take_term(y, 16.0f), l = to_codes(y.x, y.y);
                    if (c % 4 == 0) {
                        hi[c / 4] = h;
                        lo[c / 4] = l;
                    } else {
                        hi[c / 4] |= h << 16;
                        lo[c / 4] |= l << 16;
                    }
                }
                const int ch = lane * CH, block = ch >> 7, chunk = (ch & 127) >> 4, in = ch & 15;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int n = t * R + r;
                    uint32_t* to = reinterpret_cast<uint32_t*>(smem + (sQ - s0) + block * (C::NQ * 128) + n * 128 + ((chunk ^ (n & 7)) << 4) + in);
#pragma unroll
                    for (int c = 0; c < CH / 4; ++c) to[c] = t ? lo[c] : hi[c];
                }
                if (lane == 0) {
                    const int own = g.s.slot(id.t);
                    const bool real = r < rows;
                    sees_of[r] = {real ? max(window_lo(P, own), 0) : 0, real ? min(own + 1, g.s.L) : 0, real ? g.s.pre : 0};
                    refs[r] = refs[32 + r] = {real ? scale_of(s) * (P.scale * (CAP ? inv_cap : kLog2e)) : 0.0f, kNoRef, -kNoRef, 0.0f};
                }
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kQ));
            group_sync(3, 256);
            const int tb = min(g.s.n, ta + P.tile_rows / P.G) - 1;             // slots that every row sees: [all_lo, all_hi), [0, pre)
            const int all_lo = max(window_lo(P, g.s.slot(tb)), 0), all_hi = min(g.s.slot(ta) + 1, g.s.L);

            // Rows are taken 8 at a time, by the same instructions each time (4 tokens of 8 query heads on each of 8 KV heads over up to
            // 16384 slots of four sequences 57 us, 16 at a time 62: the code of two warpgroups, copies and products shares one
            // cache); their sums take each other's place after each part, so that a thread keeps them all in registers.
            constexpr int RH = 8, PARTS = R / RH;
            float2 l[PARTS][RH / 2];
#pragma unroll
            for (int r = 0; r < R / 2; ++r) l[2 * r / RH][r % (RH / 2)] = make_float2(0.0f, 0.0f);
            // their factors, their references (m with the other sign), in pairs; a weight is 128 where z is its reference
            float2 f[RH / 2], m[RH / 2], d[RH / 2];
            auto load_refs = [&](int r0) {
#pragma unroll
                for (int r = 0; r < RH; r += 2) {
                    const FewRef v = ref[r0 + r], w = ref[r0 + r + 1];
                    f[r / 2] = make_float2(v.f, w.f);
                    m[r / 2] = make_float2(-v.m, -w.m);
                    d[r / 2] = make_float2(v.d, w.d);
                }
            };
            load_refs(0);
            const int u0 = (int)((tiles + (uint32_t)wg) & 1);
            for (int u = u0; u < g.n; u += 2) {
                const uint32_t gu = tiles + (uint32_t)u;
                wait(kS + wg, (gu >> 1) & 1);
                tc_fence_after();
                wait(kScale + (int)(gu % C::TURNS), (gu / C::TURNS) & 1);
                float kf[HB], vz[HB];                    // K's scale; log2 of V's
#pragma unroll
                for (int h = 0; h < HB; ++h) {
                    const uint8_t* from = smem + C::SMEM - C::SCALES + (gu % C::TURNS) * 2 * BN + h * 128 + slot;
                    const unsigned ks = from[0], vs = from[BN];
                    // (an infinite scale: a product of either sign and an infinity is among the sum's, or 0 times one, so the score
                    // is NaN; the codes' sum alone would give it a sign)
                    kf[h] = __uint_as_float(ks == 255u ? 0x7fffffffu : ks << 23);
                    vz[h] = vs == 0u ? -INFINITY : vs == 255u ? INFINITY : (float)((int)vs - 127);
                }
                const int j0 = g.kv.at(g.i0 + u) * BN, j = j0 + slot;
                const bool all = (j0 >= all_lo && j0 + BN <= all_hi) || j0 + BN <= g.s.pre;
                const bool lower = ((u - u0) & (2 * kLower - 1)) == 2 * kLower - 2;
                // the product that last added to this O, and read P, is complete
                if (u > u0) {
                    wait(kO + wg, done & 1);
                    ++done;
                    tc_fence_after();
                }
#pragma unroll 1
                for (int r0 = 0; r0 < R; r0 += RH) {
                    float2 x[HB][RH / 2];
#pragma unroll
                    for (int h = 0; h < HB; ++h) {
                        uint32_t hi[RH], lo[RH];
                        tmem_load<RH>(lanes + (wg * HB + h) * C::NQ + r0, hi);
                        tmem_load<RH>(lanes + (wg * HB + h) * C::NQ + R + r0, lo);
                        tmem_ld_wait();
#pragma unroll
                        for (int r = 0; r < RH; r += 2)
                            x[h][r / 2] = fma2(make_float2(__uint_as_float(lo[r]), __uint_as_float(lo[r + 1])), make_float2(0.0625f, 0.0625f),
                                               make_float2(__uint_as_float(hi[r]), __uint_as_float(hi[r + 1])));
                    }
                    if (r0 + RH == R) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(kFree + wg));
                    }
                    if (PARTS > 1) load_refs(r0);
#pragma unroll
                    for (int h = 0; h < HB; ++h)
#pragma unroll
                        for (int r = 0; r < RH / 2; ++r) {
                            float2 y = mul2(mul2(x[h][r], f[r]), make_float2(kf[h], kf[h]));
                            if constexpr (CAP) {
                                const float c = P.cap * kLog2e;
                                y.x = c * (fabsf(y.x) < 0.5f ? tanh_series(y.x) : tanh_far(y.x));
                                y.y = c * (fabsf(y.y) < 0.5f ? tanh_series(y.y) : tanh_far(y.y));
                            }
                            x[h][r] = y;
                        }
                    if (!all) {
#pragma unroll
                        for (int r = 0; r < RH; ++r) {
                            const FewSees v = sees_of[r0 + r];
#pragma unroll
                            for (int h = 0; h < HB; ++h)
                                if (!((j + h * 128 >= v.lo && j + h * 128 < v.hi) || j + h * 128 < v.pre)) (r & 1 ? x[h][r / 2].y : x[h][r / 2].x) = -INFINITY;
                        }
                    }
                    float ahead = -INFINITY, ahead_z = -INFINITY;   // by how much a score is beyond its references
#pragma unroll
                    for (int h = 0; h < HB; ++h)
#pragma unroll
                        for (int r = 0; r < RH / 2; ++r) {
                            const float2 a = add2(x[h][r], m[r]), b = add2(a, add2(d[r], make_float2(vz[h], vz[h])));
                            ahead = max3(ahead, a.x, a.y);
                            ahead_z = max3(ahead_z, b.x, b.y);
                        }
                    if (group_any(1 + wg, 128, (ahead > 64.0f || ahead_z > 8.0f || lower) && ok)) {
#pragma unroll
                        for (int r = 0; r < RH; ++r) {
                            float a = -INFINITY, b = -INFINITY;      // the warp's largest x, and by how much z is beyond that
#pragma unroll
                            for (int h = 0; h < HB; ++h) a = fmaxf(a, r & 1 ? x[h][r / 2].y : x[h][r / 2].x);
                            a = warp_max(a);
#pragma unroll
                            for (int h = 0; h < HB; ++h) b = fmaxf(b, ((r & 1 ? x[h][r / 2].y : x[h][r / 2].x) - a) + vz[h]);
                            b = warp_max(b);
                            if (lane == 0) red[quad * 32 + r] = make_float2(a, b);
                        }
                        group_sync(1 + wg, 128);
                        if (slot < RH) {
                            const FewRef old = ref[r0 + slot];
                            float m1 = -INFINITY, n1 = -INFINITY;    // n1: beyond m1
#pragma unroll
                            for (int w = 0; w < 4; ++w) m1 = fmaxf(m1, red[w * 32 + slot].x);
                            m1 = fmaxf(old.m, m1 + kAhead);
#pragma unroll
                            for (int w = 0; w < 4; ++w) n1 = fmaxf(n1, red[w * 32 + slot].y + (red[w * 32 + slot].x - m1));
                            const float n0 = (old.m - m1) + (7.0f - old.d);
                            n1 = fmaxf(lower ? fmaxf(n0 - (kLowest - old.low), fminf(n0, kDeepest)) : n0, n1 + kAhead);
                            const float d1 = fminf(7.0f - n1, -kNoRef);
                            ref[r0 + slot].m = m1;
                            ref[r0 + slot].d = d1;
                            ref[r0 + slot].low = fmaxf(old.low - (n1 - n0), 0.0f);     // (no references before: 0)
                            less[slot] = make_float2(exp2_hw(old.m - m1), exp2_hw((old.m - m1) + (d1 - old.d)));
                        }
                        group_sync(1 + wg, 128);
                        load_refs(r0);
#pragma unroll
                        for (int r = 0; r < RH / 2; ++r) l[0][r] = mul2(l[0][r], make_float2(less[2 * r].x, less[2 * r + 1].x));
                        if (u > u0) {
#pragma unroll 1
                            for (int k = 0; k < 3 * DB; ++k) {
                                const uint32_t at = lanes + C::O_COL + (wg * DB + k / 3) * C::NP + k % 3 * R + r0;
                                uint32_t o[RH];
                                tmem_load<RH>(at, o);
                                tmem_ld_wait();
#pragma unroll
                                for (int r = 0; r < RH; ++r) o[r] = __float_as_uint(__uint_as_float(o[r]) * less[r].y);
                                tmem_store(at, o);
                            }
                            tmem_st_wait();
                        }
                    }
                    // weights, 128 for the largest, at most 256 (so that 32 times what a term leaves is at most 256, too)
#pragma unroll
                    for (int h = 0; h < HB; ++h) {
                        float2 y[RH / 2];
#pragma unroll
                        for (int r = 0; r < RH / 2; ++r) {
                            const float2 a = add2(x[h][r], m[r]), b = add2(a, add2(d[r], make_float2(vz[h], vz[h])));
                            l[0][r] = add2(l[0][r], make_float2(exp2_hw(a.x), exp2_hw(a.y)));
                            y[r] = make_float2(exp2_hw(b.x), exp2_hw(b.y));
                        }
                        uint32_t w[3][RH / 4];
#pragma unroll
                        for (int t = 0; t < 3; ++t)
#pragma unroll
                            for (int r = 0; r < RH; r += 4) {
                                const uint32_t a = t < 2 ? take_term(y[r / 2], 32.0f) : to_codes(y[r / 2].x, y[r / 2].y);
                                const uint32_t b = t < 2 ? take_term(y[r / 2 + 1], 32.0f) : to_codes(y[r / 2 + 1].x, y[r / 2 + 1].y);
                                w[t][r / 4] = a | b << 16;
                            }
                        // column t R + r
                        const uint32_t to = p_row + h * 4096;
                        if constexpr (R == 8) {
                            sts128(to + p_swap, make_uint4(w[0][0], w[0][1], w[1][0], w[1][1]));
                            sts128(to + (p_swap ^ 16u), make_uint4(w[2][0], w[2][1], 0u, 0u));
                        } else {
#pragma unroll
                            for (int t = 0; t < 3; ++t) {
                                const uint32_t n = (uint32_t)(t * R + r0);
                                sts64(to + n / 32 * (BN * 32) + (p_swap ^ (n & 16u)) + (n & 8u), w[t][0], w[t][1]);
                            }
                        }
                    }
                    if constexpr (PARTS > 1)
#pragma unroll
                        for (int r = 0; r < RH / 2; ++r) {
                            const float2 t = l[0][r];
#pragma unroll
                            for (int i = 1; i < PARTS; ++i) l[i - 1][r] = l[i][r];
                            l[PARTS - 1][r] = t;
                        }
                }
                fence_proxy_async();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kP + wg));
            }
            if (u0 < g.n) {
                wait(kO + wg, done & 1);
                ++done;
            }
            tiles += (uint32_t)g.n;
            // the rows' sums over a warp's lanes: halves of the rows change places with a lane each, until a lane has one row
            {
                float v[R];
#pragma unroll
                for (int r = 0; r < R; ++r) v[r] = r & 1 ? l[r / RH][r % RH / 2].y : l[r / RH][r % RH / 2].x;
                int row = 0;
#pragma unroll
                for (int w = R / 2, o = 16; w; w >>= 1, o >>= 1) {
                    const bool up = lane & o;
#pragma unroll
                    for (int i = 0; i < w; ++i) {
                        const float other = __shfl_xor_sync(0xffffffffu, up ? v[i] : v[i + w], o);
                        v[i] = (up ? v[i + w] : v[i]) + other;
                    }
                    row += up ? w : 0;
                }
#pragma unroll
                for (int o = 16 / R; o; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
                if (R == 32 || lane % (32 / R) == 0) sums[(wg * 4 + quad) * 32 + row] = v[0];
            }
            group_sync(3, 256);
            tc_fence_after();
            const bool whole = g.whole(), one = g.n > (int)((tiles - g.n) & 1), two = g.n > (int)((tiles - g.n + 1) & 1);   // warpgroups that had tiles
            // a row's end, by a thread: its reference and sum over both warpgroups, what each O is multiplied by (128 for a weight
            // of one), and where it goes
            if (sw * 32 + lane < rows) {
                const int row = sw * 32 + lane;
                const float ma = one ? refs[row].m : kNoRef, mb = two ? refs[32 + row].m : kNoRef, top = fmaxf(ma, mb);
                float sum = 0.0f;
                if (one) sum += (sums[row] + sums[32 + row] + sums[64 + row] + sums[96 + row]) * exp2_hw(ma - top);
                if (two) sum += (sums[128 + row] + sums[160 + row] + sums[192 + row] + sums[224 + row]) * exp2_hw(mb - top);
                const RowId id = row_id(P, g.s, g.h, g.rt * P.tile_rows + row);
                const float inv = !whole ? 1.0f : sum > 0.0f ? 1.0f / sum : sum;       // (nothing seen: zeros; NaN stays)
                FewEnd e;
                e.to = (long long)(g.s.t0 + id.t) * P.o_t + (long long)id.head * P.o_h;
                e.a = one ? exp2_hw((ma - top) - refs[row].d) * inv : 0.0f;
                e.b = two ? exp2_hw((mb - top) - refs[32 + row].d) * inv : 0.0f;
                e.lse2 = sum == 0.0f ? -INFINITY : top + log2f(sum);
                e.sum = sum;
                ends[row] = e;
                if (whole && P.lse) P.lse[(long long)(g.s.t0 + id.t) * P.Hq + id.head] = e.lse2 * kLn2;
                if (!whole) __stcg(P.part_ml + (size_t)(2 * blockIdx.x + (g.first ? 0 : 1)) * R + row, make_float2(sum == 0.0f ? -INFINITY : top, sum));
            }
            group_sync(3, 256);
            // heads of 128: half the rows a warpgroup, heads of 256: half the channels
            constexpr int RW = DB == 1 ? R / 2 : R;
            const int first_row = DB == 1 ? wg * RW : 0, block = DB == 1 ? 0 : wg, channel = block * 128 + slot;
            float* part = P.part_o + (size_t)(2 * blockIdx.x + (g.first ? 0 : 1)) * R * D + channel;
            uint32_t not_fine = 0;
#pragma unroll 1                                             // short code: a cold instruction cache costs small calls most
            for (int r0 = first_row; ok && r0 < min(first_row + RW, rows); r0 += 4) {
                uint32_t v[2][3][4];
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int t = 0; t < 3; ++t) tmem_load<4>(lanes + C::O_COL + (x * DB + block) * C::NP + t * R + r0, v[x][t]);
                tmem_ld_wait();
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (r0 + r >= rows) break;
                    const FewEnd e = ends[r0 + r];
                    auto joined = [&](int x) {
                        return fmaf(__uint_as_float(v[x][2][r]), 0x1p-10f, fmaf(__uint_as_float(v[x][1][r]), 0x1p-5f, __uint_as_float(v[x][0][r])));
                    };
                    float y = (one ? joined(0) * e.a : 0.0f) + (two ? joined(1) * e.b : 0.0f);
                    if (whole) {
                        if (e.sum == 0.0f) y = 0.0f;
                        ((__nv_bfloat16*)P.out)[e.to + channel] = __float2bfloat16_rn(y);
                        if (!(fabsf(y) <= 3.0e38f) && e.sum == e.sum) not_fine |= 1u << (r0 + r);
                    } else {
                        __stcg(part + (size_t)(r0 + r) * D, y);
                    }
                }
            }
            tc_fence_before();
            if (whole) {
                not_fine = __reduce_or_sync(0xffffffffu, not_fine);
                if (lane == 0) bad[sw] = not_fine;
                group_sync(3, 256);
                uint32_t all_bad = 0;
#pragma unroll
                for (int x = 0; x < 8; ++x) all_bad |= bad[x];
                for (int row = sw; row < rows; row += 8) {
                    if (!(all_bad >> row & 1u)) continue;
                    float o[D / 32];
                    resum_row<__nv_bfloat16, D>(P, g.s, g.b, g.h, g.rt * P.tile_rows + row, ends[row].lse2, o, beat);
                    store_f32<__nv_bfloat16, D / 32>((__nv_bfloat16*)P.out + ends[row].to + lane * (D / 32), o);
                }
            }
            group_sync(3, 256);                          // the tables and the sums are the next item's
            if (odd_rows) {
                const Segment item = g;
                for (int row = sw; row < rows; row += 8)
                    if (odd_rows >> row & 1u) infinite_row<D, BN>(P, item, row, (size_t)(2 * blockIdx.x + (g.first ? 0 : 1)) * R + row, beat);
            }
        }
        if (threadIdx.x == 128) leave_split(P, *plan, g, have);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 3) {
        tmem_relinquish();
        tmem_dealloc(tmem, C::TMEM);
    }
}

template <int D, int R, bool GROUPS, bool CAP> cudaError_t start_few(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    using C = FewShape<D, R>;
    const int grid = min(num_sms, kAttendMaxRows / R / 2);
    if (cudaError_t e = smem_opt_in<attend_few_kernel<D, R, GROUPS, CAP>>(C::SMEM); e != cudaSuccess) return e;
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
    if (cudaError_t e = cudaLaunchKernelEx(&cfg, attend_few_kernel<D, R, GROUPS, CAP>, P); e != cudaSuccess) return e;
    return run_join<__nv_bfloat16, D, R>(P, grid, stream);
}
template <int D, int R, bool CAP> cudaError_t run_few(const AttendParams& call, int num_sms, cudaStream_t stream)
{
    AttendParams P = call;
    P.tile_rows = R / P.G * P.G;
    if (!P.cache.paged || P.cache.page_size % 8 == 0) return start_few<D, R, true, CAP>(P, num_sms, stream);
    return start_few<D, R, false, CAP>(P, num_sms, stream);
}

}  // namespace
}  // namespace kvx
