// kvx_attend_tc.cu -- attention of new tokens over a bf16 cache on the tensor cores (tcgen05).
//
//   S = Q K^T (fp32, TMEM),  P = exp2(c S - m),  O += P V (P bf16 from TMEM, O fp32 in TMEM)
// in one pass over the slots, with the running maximum m and sum l of a row in the registers of the thread
// that owns the row.  A CTA holds NT tiles of 128 rows and walks slot tiles of BN.
//   producer warps (3)  copy Q, K and V rows into 128-byte-swizzled tiles.  Q: 16-byte cp.async.  K and V: one
//                       tensor copy (TMA) for each page, or for a whole tile of a contiguous cache, by one
//                       warp, a box a lane; caches that boxes of 8 or more rows cannot describe (odd page
//                       sizes) take cp.async too.  A K tile is read as a K-major operand, a V tile, laid
//                       out alike, as an MN-major one.
//   MMA thread          unit u = (slot tile, row tile): S(u) into score buffer u mod 2, then, when P(u)
//                       is there, O += P(u) V; S(u + 2) is issued right behind it, so that the scores of
//                       one unit are formed while the other's softmax runs.
//   softmax warps       a warpgroup a row tile (two row tiles), one for all units (one row tile).  P takes the
//                       place of S.  O is rescaled only when a row's maximum has grown by more than
//                       2^8 since the last time.
// P is rounded to bf16 for the MMA, as V is.  Where a row sees few slots the roundings of its few weights do
// not average out, and the error comes near 2^-8 |v|; there, and where the copies bound the kernel
// anyway (one row tile), P goes in as two bf16 terms, high and low, at the price of a second product.
#include <cuda.h>

#include <atomic>

#include "kvx_attend_rows.cuh"
#include "kvx_kernels.h"
#include "kvx_tc_common.cuh"

namespace kvx {
namespace {

template <int D, int NT> struct TcShape {
    static constexpr int BM = 128 * NT, BN = D == 256 ? 64 : 128, NB = 2 / NT;
    static constexpr int TILE = BN * D * 2, QB = BM * D * 2;
    static constexpr int STAGES = D == 64 ? 8 : D == 128 ? (NT == 2 ? 5 : 6) : 5;
    static constexpr int THREADS = 128 + 128 * NT;
    static constexpr int S_COL = BN, O_COL = 2 * BN;       // TMEM columns: scores u mod 2, then the O tiles
    static constexpr int TMEM = 512;
    static constexpr int CTRL = 1024;                      // barriers and flags
    static constexpr int SMEM = CTRL + QB + STAGES * TILE;
    static_assert(SMEM <= kSmemMax && O_COL + NT * D <= TMEM);
    static_assert((kMaxAttendBatch + 2) * 8 <= STAGES * TILE);   // the plan's sums lie where the tiles come later
};

constexpr int kProdWarps = 3, kMmaWarp = 3;

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// D[tmem] (+)= A[tmem] . B[smem], bf16 inputs, fp32 accumulate
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// MN-major 128-byte-swizzled operand: lbo between 64-channel blocks, 1024 bytes between 8-row groups.
__device__ __forceinline__ uint64_t mn_desc(uint32_t saddr, uint32_t lbo)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)((lbo >> 4) & 0x3FFFu) << 16 | (uint64_t)(1024u >> 4) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(r)
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)),
          "l"(reinterpret_cast<unsigned long long&>(c)));
    return reinterpret_cast<float2&>(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return reinterpret_cast<float2&>(r);
}
// Bits [a, b) of the 32 columns from `base` on (a, b relative to column 0 of the tile).
__device__ __forceinline__ uint32_t range_bits(int a, int b, int base)
{
    const int lo = max(a - base, 0), hi = min(b - base, 32);
    if (hi <= lo) return 0u;
    return (hi == 32 ? 0xffffffffu : (1u << hi) - 1u) & ~((1u << lo) - 1u);
}

// Registers of a thread once the warps have taken their parts (two row tiles: 384 threads launched with 168):
// 128 x 88 + 256 x 208 = 384 x 168.
template <int N> __device__ __forceinline__ void regs_give() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_take() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

constexpr int kFewSlots = 512;   // rows that see fewer slots get their weights in two terms

// Whether an item's weights are multiplied in two terms: its first token sees fewest slots.
template <int BM, int NT> __device__ __forceinline__ bool two_terms(const AttendParams& P, const Segment& g)
{
    if (NT == 1 && (long long)P.T * P.G <= 128ll * P.batch) return true;
    int ta, tb;
    row_tile_tokens<BM>(P, g.s, g.rt, ta, tb);
    const int own = g.s.slot(ta);
    return own < kFewSlots || (P.window > 0 && P.window < kFewSlots);
}

// Tensor maps of K and V, and the rows of a box: a paged cache as (channel, head, slot in page, page), a
// contiguous one as (channel, slot, head, sequence); boxes of 64 channels of one head.
struct TileMaps {
    CUtensorMap k, v;
    int box_rows;
};
__device__ __forceinline__ void tma_box4(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t mbar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
        "l"(map), "r"(mbar), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}

// Barriers (8 bytes each) in the control block.
template <int STAGES> struct Bars {
    static constexpr int full = 0, empty = STAGES, sfull = 2 * STAGES, pfull = sfull + 2, ofull = pfull + 2, qfull = ofull + 2,
                         qempty = qfull + 1, done = qempty + 1;
};

template <int D, int NT, bool TMA>
__global__ void __launch_bounds__(TcShape<D, NT>::THREADS, 1)
    attend_tc_kernel(const __grid_constant__ AttendParams P, const __grid_constant__ TileMaps maps)
{
    using C = TcShape<D, NT>;
    using B = Bars<C::STAGES>;
    constexpr int BM = C::BM, BN = C::BN;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t s0 = smem_u32(smem);
    auto bar = [&](int i) { return s0 + (uint32_t)i * 8; };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + 512);
    int* abort = reinterpret_cast<int*>(smem + 516);
    const uint32_t sQ = s0 + C::CTRL, sT = sQ + C::QB;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (warp == kMmaWarp) tmem_alloc(smem_u32(tmem_slot), C::TMEM);
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) {
            mbar_init(bar(B::full + i), TMA ? 1 : kProdWarps);
            mbar_init(bar(B::empty + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(B::sfull + i), 1);
            mbar_init(bar(B::pfull + i), 4);
            mbar_init(bar(B::ofull + i), 1);
        }
        mbar_init(bar(B::qfull), kProdWarps);
        mbar_init(bar(B::qempty), 1);
        mbar_init(bar(B::done), 1);
        fence_mbar_init();
        *abort = 0;
    }
    const Plan plan = make_plan<BM, BN, C::THREADS>(P, reinterpret_cast<long long*>(smem + C::CTRL + C::QB));
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const Waiter W{abort, P.status};
    SegmentWalk<BM, BN> walk(P, plan);
    Segment g;

    if (warp < 4) {
    if constexpr (NT == 2) regs_give<88>();
    if (warp < kProdWarps) {
        // ---------------------------------------------------------------- producers
        constexpr int CPR = D / 8;                       // 16-byte chunks of a row
        constexpr int RPI = CPR < 32 ? 32 / CPR : 1;     // rows a warp copies with one instruction
        const int chunk = lane % CPR, sub = lane / CPR;
        uint32_t pos = 0, items = 0;                     // tiles issued; items begun
        int pending[2] = {-1, -1};                       // barriers of the last two batches, not announced yet
        bool ok = true;
        auto announce = [&](int b) {
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(b));
        };
        auto batch = [&](int b) {                        // a batch of copies ends: the one before the last is complete
            cp_commit();
            cp_wait<2>();
            if (pending[0] >= 0) announce(pending[0]);
            pending[0] = pending[1];
            pending[1] = b;
        };
        auto flush = [&]() {
            cp_wait<0>();
            for (int i = 0; i < 2; ++i) {
                if (pending[i] >= 0) announce(pending[i]);
                pending[i] = -1;
            }
        };
        // rows r of a tile of R at base: lane 32 k + l of `off` has row 32 k + l's element offset, -1 for zeros
        auto copy_rows = [&](uint32_t base, const __nv_bfloat16* src, const long long* off, int R, int colblk) {
            for (int r0 = warp * RPI; r0 < R; r0 += kProdWarps * RPI) {
                const int r = r0 + sub;
                const int k = r0 >> 5;                   // RPI divides 32: the rows of one instruction share a block
                const long long mine = k == 0 ? off[0] : k == 1 ? off[1] : k == 2 ? off[2] : off[3];
                const long long at = __shfl_sync(0xffffffffu, mine, r & 31);
                const uint32_t d = base + (uint32_t)((chunk >> 3) * colblk + (r >> 3) * 1024 + (r & 7) * 128 + (((chunk & 7) ^ (r & 7)) << 4));
                cp_async16_or_zero(d, src + (at < 0 ? 0 : at + chunk * 8), at >= 0);
            }
        };
        while (walk.next(g)) {
            const int rows = min(BM, g.s.n * P.G - g.rt * BM);
            flush();
            if (items > 0) ok = ok && W.wait(bar(B::qempty), (items - 1) & 1);
            for (int part = 0; part < NT; ++part) {
                long long off[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int r = part * 128 + k * 32 + lane;
                    off[k] = -1;
                    if (r < rows) {
                        const RowId id = row_id(P, g.s, g.h, g.rt * BM + r);
                        off[k] = (long long)(g.s.t0 + id.t) * P.q_t + (long long)id.head * P.q_h;
                    }
                }
                if (ok) copy_rows(sQ + part * (128 * D * 2), (const __nv_bfloat16*)P.q, off, 128, 128 * 128);
            }
            batch(B::qfull);
            ++items;
            const long long head = cache_head(P.cache) * g.h;
            // tile i as K, tile i - NB + 1 as V, and at the end the V tiles left
            if constexpr (TMA) {
                if (warp > 0) {
                    flush();
                    continue;
                }
                // lanes take the boxes of a tile: box e is rows [r, r + box_rows) of channel block e mod D/64
                const int boxes = BN / maps.box_rows * (D / 64);
                for (int i = 0; i < g.n + C::NB - 1; ++i) {
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        const int t = kv ? i - (C::NB - 1) : i;
                        if (t < 0 || t >= g.n) continue;
                        const int j0 = g.kv.at(g.i0 + t) * BN;
                        const uint32_t st = pos % C::STAGES, ph = (pos / C::STAGES) & 1;
                        ok = ok && W.wait(bar(B::empty + st), ph ^ 1);
                        ok = __all_sync(0xffffffffu, ok);
                        ++pos;
                        if (!ok) continue;
                        if (lane == 0) mbar_arrive_expect_tx(bar(B::full + st), C::TILE);
                        __syncwarp();
                        for (int e = lane; e < boxes; e += 32) {
                            const int cb = e % (D / 64), r = e / (D / 64) * maps.box_rows, j = j0 + r;
                            const uint32_t dst = sT + st * C::TILE + (uint32_t)(cb * (BN * 128) + r * 128);
                            const CUtensorMap* map = kv ? &maps.v : &maps.k;
                            if (P.cache.paged) {
                                int page = -1;           // outside the pool: the box is filled with zeros
                                if (j < g.s.L) {
                                    const int pi = j >> P.cache.page_shift;
                                    if (pi < P.cache.max_pages) page = __ldg(&P.cache.page_table[(size_t)g.b * P.cache.max_pages + pi]);
                                    if (page < 0 || page >= P.cache.num_pages) {
                                        page = -1;
                                        set_status(P.status, KVX_DEV_PAGE_INVALID);
                                    }
                                }
                                tma_box4(dst, map, cb * 64, g.h, j & (P.cache.page_size - 1), page, bar(B::full + st));
                            } else {
                                tma_box4(dst, map, cb * 64, j, g.h, g.b, bar(B::full + st));
                            }
                        }
                        __syncwarp();
                    }
                    if (i == 0) flush();                 // the queries, behind the first tiles' copies
                }
            } else
            for (int i = 0; i < g.n + C::NB - 1; ++i) {
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    const int t = kv ? i - (C::NB - 1) : i;
                    if (t < 0 || t >= g.n) continue;
                    const int j0 = g.kv.at(g.i0 + t) * BN;
                    long long off[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int j = j0 + k * 32 + lane;
                        off[k] = -1;
                        if (k * 32 < BN && j < g.s.L) {
                            const long long at = cache_row(P.cache, g.b, j);
                            if (at >= 0) off[k] = at + head;
                            else set_status(P.status, KVX_DEV_PAGE_INVALID);
                        }
                    }
                    const uint32_t st = pos % C::STAGES, ph = (pos / C::STAGES) & 1;
                    ok = ok && W.wait(bar(B::empty + st), ph ^ 1);
                    if (ok) copy_rows(sT + st * C::TILE, (const __nv_bfloat16*)(kv ? P.cv : P.ck), off, BN, BN * 128);
                    batch(B::full + (int)st);
                    ++pos;
                }
            }
        }
        flush();
    } else {
        // ---------------------------------------------------------------- MMA
        if (lane == 0) {
            constexpr uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
            constexpr uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
            uint32_t base = 0, units = 0, items = 0;     // tiles and units of the items before; items begun
            bool ok = true, issued = false;
            while (ok && walk.next(g)) {
                const int U = g.n * NT;
                auto k_pos = [&](int i) { return base + (uint32_t)(C::NB == 1 ? 2 * i : i == 0 ? 0 : 2 * i - 1); };
                auto v_pos = [&](int i) { return base + (uint32_t)(C::NB == 1 ? 2 * i + 1 : i == g.n - 1 ? 2 * i + 1 : 2 * i + 2); };
                auto scores = [&](int u) {
                    const int i = u / NT, t = u - i * NT;
                    const uint32_t p = k_pos(i), st = p % C::STAGES;
                    if (u == 0) ok = ok && W.wait(bar(B::qfull), items & 1);
                    if (t == 0) ok = ok && W.wait(bar(B::full + st), (p / C::STAGES) & 1);
                    if (!ok) return;
                    tc_fence_after();
                    const uint32_t d = tmem + ((units + u) & 1) * C::S_COL;
                    // descriptors count 16-byte units in their low bits: steps along an operand are added
                    const uint64_t qd = sw128_desc(sQ + t * (128 * D * 2)), kd = sw128_desc(sT + st * C::TILE);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        umma_bf16(d, qd + (k >> 2) * (128 * 128 / 16) + (k & 3) * 2, kd + (k >> 2) * (BN * 128 / 16) + (k & 3) * 2, idesc_s, k > 0);
                    issued = true;
                    if (t == NT - 1) umma_commit(bar(B::empty + st));
                    if (u == U - 1) umma_commit(bar(B::qempty));
                    umma_commit(bar(B::sfull + ((units + u) & 1)));
                };
                const bool two = two_terms<BM, NT>(P, g);
                scores(0);
                if (U > 1) scores(1);
                for (int u = 0; u < U && ok; ++u) {
                    const int i = u / NT, t = u - i * NT;
                    const uint32_t gu = units + u, p = v_pos(i), st = p % C::STAGES;
                    ok = ok && W.wait(bar(B::pfull + (gu & 1)), (gu >> 1) & 1);
                    if (t == 0) ok = ok && W.wait(bar(B::full + st), (p / C::STAGES) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t vd = mn_desc(sT + st * C::TILE, BN * 128);
                    const uint32_t od = tmem + C::O_COL + t * D, pd = tmem + (gu & 1) * C::S_COL;
#pragma unroll
                    for (int k = 0; k < BN / 16; ++k) umma_bf16_ts(od, pd + k * 8, vd + k * (2048 / 16), idesc_o, i > 0 || k > 0);
                    if (two)
#pragma unroll
                        for (int k = 0; k < BN / 16; ++k) umma_bf16_ts(od, pd + BN / 2 + k * 8, vd + k * (2048 / 16), idesc_o, 1);
                    if (t == NT - 1) umma_commit(bar(B::empty + st));
                    if (i == g.n - 1) umma_commit(bar(B::ofull + t));
                    if (u + 2 < U) scores(u + 2);
                }
                base += 2 * (uint32_t)g.n;
                units += (uint32_t)U;
                ++items;
            }
            // every MMA issued has completed before TMEM is freed
            if (issued) {
                umma_commit(bar(B::done));
                const unsigned long long t0 = globaltimer();
                while (!mbar_try_wait(bar(B::done), 0) && globaltimer() - t0 < kWaitNs) {}
            }
        }
        __syncwarp();
    }
    } else {
        // ---------------------------------------------------------------- softmax
        if constexpr (NT == 2) regs_take<208>();
        const int t = NT == 2 ? (warp - 4) >> 2 : 0, quad = warp & 3;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
        const float inv_cap = P.cap > 0.0f ? 1.0f / P.cap : 0.0f;
        const float c = P.cap > 0.0f ? 1.0f : P.scale * kLog2e;   // factor of the (capped) scores in log2 units
        uint32_t units = 0, items = 0, base_tile = 0;
        bool ok = true;                                  // the same in the lanes of a warp
        auto wait = [&](int b, uint32_t parity) { ok = __all_sync(0xffffffffu, ok && W.wait(bar(b), parity)); };
        bool have = false;
        while (walk.next(g)) {
            have = true;
            const int row = g.rt * BM + t * 128 + quad * 32 + lane;
            const bool real = row < g.s.n * P.G;
            const int own = real ? g.s.slot(row / P.G) : -1;     // rows past the end see nothing
            const int hi = min(own + 1, g.s.L), lo = max(window_lo(P, own), 0), pre = real ? g.s.pre : 0;
            const bool two = two_terms<BM, NT>(P, g);
            float m = -INFINITY, l = 0.0f;
            for (int i = 0; i < g.n; ++i) {
                const uint32_t gu = units + (uint32_t)(i * NT + t);
                wait(B::sfull + (gu & 1), (gu >> 1) & 1);
                if (!ok) break;
                tc_fence_after();
                const uint32_t at = lanes + (gu & 1) * C::S_COL;
                uint32_t x[BN];
#pragma unroll
                for (int k = 0; k < BN; k += 32) tmem_ld32(at + k, *reinterpret_cast<uint32_t(*)[32]>(x + k));
                tmem_ld_wait();
                auto xf = [&](int k) -> float { return __uint_as_float(x[k]); };
                if (P.cap > 0.0f) {
                    bool near = true;                    // all scores where the series holds: no branch per score
#pragma unroll
                    for (int k = 0; k < BN; ++k) {
                        const float y = xf(k) * (P.scale * inv_cap);
                        near = near && fabsf(y) < 0.5f;
                        x[k] = __float_as_uint(y);
                    }
                    if (__all_sync(0xffffffffu, near)) {
#pragma unroll
                        for (int k = 0; k < BN; ++k) x[k] = __float_as_uint(P.cap * kLog2e * tanh_series(xf(k)));
                    } else {
#pragma unroll
                        for (int k = 0; k < BN; ++k)
                            x[k] = __float_as_uint(P.cap * kLog2e * (fabsf(xf(k)) < 0.5f ? tanh_series(xf(k)) : tanh_far(xf(k))));
                    }
                }
                const int j0 = g.kv.at(g.i0 + i) * BN;
                if (TMA && j0 + BN > g.s.L && t == 0) {
                    // the boxes brought what the cache holds past the sequence's end: zeros in V's place, before
                    // any P is announced for it
                    const uint32_t p = base_tile + (uint32_t)(C::NB == 1 ? 2 * i + 1 : i == g.n - 1 ? 2 * i + 1 : 2 * i + 2), st = p % C::STAGES;
                    wait(B::full + (int)st, (p / C::STAGES) & 1);
                    if (!ok) break;
                    const int from = max(g.s.L - j0, 0);
                    uint8_t* tile = smem + C::CTRL + C::QB + st * C::TILE;
                    for (int e = (int)threadIdx.x - 128 + from * 8; e < BN * 8; e += 128)
#pragma unroll
                        for (int cb = 0; cb < D / 64; ++cb) *reinterpret_cast<uint4*>(tile + cb * (BN * 128) + e * 16) = make_uint4(0, 0, 0, 0);
                    fence_proxy_async();
                }
                const bool all = (j0 >= lo && j0 + BN <= hi) || j0 + BN <= pre;
                if (!__all_sync(0xffffffffu, all)) {
#pragma unroll
                    for (int k0 = 0; k0 < BN; k0 += 32) {
                        const uint32_t seen = range_bits(lo, hi, j0 + k0) | range_bits(0, pre, j0 + k0);
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (!(seen >> k & 1u)) x[k0 + k] = 0xff800000u;
                    }
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int k = 0; k < BN; ++k) top[k & 3] = fmaxf(top[k & 3], xf(k));
                const float next = fmaxf(m, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * c);
                // a row that grew by more than 2^8 (or had seen nothing) takes its new maximum, and its warp with it
                if (__any_sync(0xffffffffu, next > m + 8.0f || (m == -INFINITY && next > m))) {
                    const float w = next == -INFINITY ? 1.0f : exp2_hw(m - next);
                    m = next;
                    l *= w;
                    if (i > 0) {                         // S(u) complete: so is the MMA that last added to O
#pragma unroll
                        for (int k = 0; k < D; k += 16) {
                            uint32_t o[16];
                            tmem_ld16(lanes + C::O_COL + t * D + k, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * w);
                            tmem_st16(lanes + C::O_COL + t * D + k, o);
                        }
                    }
                }
                const float base = m == -INFINITY ? 0.0f : m;
                const float2 c2 = make_float2(c, c), b2 = make_float2(-base, -base);
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                if (two) {
                    uint32_t low[BN / 2];
#pragma unroll
                    for (int k = 0; k < BN; k += 2) {
                        float2 y = fma2(make_float2(xf(k), xf(k + 1)), c2, b2);
                        y.x = exp2_hw(y.x);
                        y.y = exp2_hw(y.y);
                        sum[k >> 1 & 1] = add2(sum[k >> 1 & 1], y);
                        const uint32_t h = pack_bf16(y.x, y.y);
                        x[k >> 1] = h;
                        low[k >> 1] = pack_bf16(y.x - bf_lo(h), y.y - bf_hi(h));
                    }
#pragma unroll
                    for (int k = 0; k < BN / 2; k += 32) tmem_st32(at + BN / 2 + k, low + k);
                } else {
#pragma unroll
                    for (int k = 0; k < BN; k += 2) {
                        float2 y = fma2(make_float2(xf(k), xf(k + 1)), c2, b2);
                        y.x = exp2_hw(y.x);
                        y.y = exp2_hw(y.y);
                        sum[k >> 1 & 1] = add2(sum[k >> 1 & 1], y);
                        x[k >> 1] = pack_bf16(y.x, y.y);
                    }
                }
                const float2 s2 = add2(sum[0], sum[1]);
                l += s2.x + s2.y;
#pragma unroll
                for (int k = 0; k < BN / 2; k += 32) tmem_st32(at + k, x + k);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(B::pfull + (gu & 1)));
            }
            units += (uint32_t)(g.n * NT);
            base_tile += 2 * (uint32_t)g.n;
            if (ok) wait(B::ofull + t, items & 1);
            ++items;
            tc_fence_after();
            const bool whole = g.whole();
            const float inv = whole ? (l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l)) : 1.0f;
            const float lse2 = l == 0.0f ? -INFINITY : m + log2f(l);
            const RowId id = row_id(P, g.s, g.h, row);
            __nv_bfloat16* out = (__nv_bfloat16*)P.out + (long long)(g.s.t0 + id.t) * P.o_t + (long long)id.head * P.o_h;
            const size_t part = (size_t)(2 * blockIdx.x + (g.first ? 0 : 1)) * BM + (row - g.rt * BM);
            bool fine = true;
            if (ok) {
#pragma unroll
                for (int k = 0; k < D; k += 32) {
                    uint32_t o[32];
                    tmem_ld32(lanes + C::O_COL + t * D + k, o);
                    tmem_ld_wait();
                    if (whole && real) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const float v = l == 0.0f ? 0.0f : __uint_as_float(o[e]) * inv;
                            fine = fine && fabsf(v) <= 3.0e38f;
                            o[e] = __float_as_uint(v);
                        }
#pragma unroll
                        for (int e = 0; e < 32; e += 8)
                            *reinterpret_cast<uint4*>(out + k + e) =
                                make_uint4(pack_bf16(__uint_as_float(o[e]), __uint_as_float(o[e + 1])),
                                           pack_bf16(__uint_as_float(o[e + 2]), __uint_as_float(o[e + 3])),
                                           pack_bf16(__uint_as_float(o[e + 4]), __uint_as_float(o[e + 5])),
                                           pack_bf16(__uint_as_float(o[e + 6]), __uint_as_float(o[e + 7])));
                    } else if (real) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            __stcg(reinterpret_cast<uint4*>(P.part_o + part * D + k + e), make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]));
                    }
                    __syncwarp();
                }
            }
            tc_fence_before();
            if (whole) {
                if (real && P.lse) P.lse[(long long)(g.s.t0 + id.t) * P.Hq + id.head] = lse2 * kLn2;
                for (uint32_t bad = __ballot_sync(0xffffffffu, real && !fine); bad; bad &= bad - 1) {
                    const int who = __ffs(bad) - 1;
                    float o[D / 32];
                    resum_row<__nv_bfloat16, D>(P, g.s, g.b, g.h, row - lane + who, __shfl_sync(0xffffffffu, lse2, who), o);
                    const RowId bid = row_id(P, g.s, g.h, row - lane + who);
                    store_f32<__nv_bfloat16, D / 32>((__nv_bfloat16*)P.out + (long long)(g.s.t0 + bid.t) * P.o_t + (long long)bid.head * P.o_h +
                                                         lane * (D / 32), o);
                }
            } else {
                if (real) __stcg(P.part_ml + part, make_float2(m, l));
            }
        }
        if (threadIdx.x == 128) leave_split(P, plan, g, have);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tmem_relinquish();
        tmem_dealloc(tmem, C::TMEM);
    }
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled tiled_encoder()
{
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return (EncodeTiled)p;
    }();
    return fn;
}

// The maps of a call's cache, tiles of bn slots; false where boxes cannot describe it.
bool make_maps(const AttendParams& P, int bn, TileMaps& m)
{
    const CacheView& c = P.cache;
    const EncodeTiled enc = tiled_encoder();
    if (!enc || c.capacity < 1 || (c.paged && (c.page_shift < 3))) return false;
    m.box_rows = c.paged && c.page_size < bn ? c.page_size : bn;
    const cuuint64_t H = (cuuint64_t)c.H, d = (cuuint64_t)c.d;
    const cuuint64_t dims_p[4] = {d, H, (cuuint64_t)c.page_size, (cuuint64_t)c.num_pages};
    const cuuint64_t str_p[3] = {d * 2, H * d * 2, (cuuint64_t)c.page_size * H * d * 2};
    const cuuint64_t dims_c[4] = {d, (cuuint64_t)c.capacity, H, (cuuint64_t)P.batch};
    const cuuint64_t str_c[3] = {(cuuint64_t)c.st * 2, (cuuint64_t)c.sh * 2, (cuuint64_t)c.sb * 2};
    const cuuint32_t box_p[4] = {64, 1, (cuuint32_t)m.box_rows, 1}, box_c[4] = {64, (cuuint32_t)m.box_rows, 1, 1};
    const cuuint32_t one[4] = {1, 1, 1, 1};
    for (int i = 0; i < 2; ++i)
        if (enc(i ? &m.v : &m.k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(i ? P.cv : P.ck), c.paged ? dims_p : dims_c,
                c.paged ? str_p : str_c, c.paged ? box_p : box_c, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return false;
    return true;
}

template <int D, int NT, bool TMA> cudaError_t start_tc(const AttendParams& P, const TileMaps& maps, int num_sms, cudaStream_t stream)
{
    using C = TcShape<D, NT>;
    if (cudaError_t e = smem_opt_in<attend_tc_kernel<D, NT, TMA>>(C::SMEM); e != cudaSuccess) return e;
    const int grid = min(num_sms, kAttendMaxRows / C::BM / 2);
    attend_tc_kernel<D, NT, TMA><<<grid, C::THREADS, C::SMEM, stream>>>(P, maps);
    if (cudaError_t e = cudaGetLastError(); e != cudaSuccess) return e;
    return run_join<__nv_bfloat16, D, C::BM>(P, grid, stream);
}
template <int D, int NT> cudaError_t run_tc(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    TileMaps maps;
    if (make_maps(P, TcShape<D, NT>::BN, maps)) return start_tc<D, NT, true>(P, maps, num_sms, stream);
    return start_tc<D, NT, false>(P, maps, num_sms, stream);
}

}  // namespace

cudaError_t launch_attend_tc(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    // sequences of up to 128 rows a KV head: one row tile, whose two score buffers keep the MMAs going
    const bool one = (long long)P.T * P.G <= 128ll * P.batch;
    if (P.d == 64) return one ? run_tc<64, 1>(P, num_sms, stream) : run_tc<64, 2>(P, num_sms, stream);
    if (P.d == 128) return one ? run_tc<128, 1>(P, num_sms, stream) : run_tc<128, 2>(P, num_sms, stream);
    return run_tc<256, 1>(P, num_sms, stream);
}

}  // namespace kvx
