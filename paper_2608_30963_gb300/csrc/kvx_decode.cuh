// kvx_decode.cuh -- parameters and device helpers of the kernels that go on from a cache
// (library-internal): cache addressing, the masks of attention, and how its work is split.
#pragma once

#include "kvx_common.cuh"

namespace kvx {

constexpr int kMaxAttendBatch = 1024;   // sequences one attention launch takes (its plan's shared memory)

// A cache of one layer, read or written by slot.
struct CacheView {
    int paged, capacity;                // slots a sequence may hold
    long long sb, sh, st;               // contiguous: element strides
    const int* page_table;
    int max_pages, page_size, num_pages;
    int page_shift;                     // log2(page_size), or -1
    int H, d;
};

// Lengths and tables are read by plain loads: one through the read-only path might be moved up past the wait for the
// kernel before, which may have written them.
// Element offset of slot s of sequence b, head 0 (add head_stride * h), or -1 if its page is not in the pool.
__device__ __forceinline__ long long cache_row(const CacheView& C, int b, int s)
{
    if (!C.paged) return (long long)b * C.sb + (long long)s * C.st;
    const int pi = C.page_shift >= 0 ? s >> C.page_shift : s / C.page_size;
    const int in = s - pi * C.page_size;
    const int page = pi < C.max_pages ? C.page_table[(size_t)b * C.max_pages + pi] : -1;
    if (page < 0 || page >= C.num_pages) return -1;
    return ((long long)page * C.page_size + in) * ((long long)C.H * C.d);
}
__host__ __device__ __forceinline__ long long cache_head(const CacheView& C) { return C.paged ? C.d : C.sh; }

struct AppendParams {
    int T, batch, Hq, H, d, rhalf, rope, max_position;
    const int* seq_off;
    const int* kv_len;
    const int* pos;
    const unsigned long long* turns;
    const void *q, *k, *v;
    void* q_out;
    long long q_t, q_h, k_t, k_h, v_t, v_h, o_t, o_h;
    void *ck, *cv;
    CacheView cache;
    unsigned* status;
};
cudaError_t launch_append(const AppendParams& P, int dtype, cudaStream_t stream);

// A row tile and KV head whose tiles several CTAs have, as the CTA where it begins leaves it; parts = 0: none.
struct SplitItem {
    int b, rt, h, rows;       // rows of the tile that exist
    int token;                // packed index of its first token
    int parts, slot0, lines;
};

struct AttendParams {
    int T, batch, Hq, H, G, d;
    int tile_rows;        // rows of a row tile: of the kernel's, those it uses
    const int* seq_off;
    const int* kv_len;
    const void* q;
    void* out;
    const void *ck, *cv;
    long long q_t, q_h, o_t, o_h;
    CacheView cache;
    float scale;          // of q.k
    float cap;            // 0: none
    int window;
    const int* prefix_len;
    float* lse;
    float* key_weight;
    long long weight_stride;
    unsigned* status;
    // workspace of split rows: two partial results a CTA, and the item that begins in it and goes on in the next
    float* part_o;        // [2 * grid][BM][d]
    float2* part_ml;      // [2 * grid][BM]: running maximum (log2 units) and sum
    SplitItem* split;     // [grid]
    // scores of few rows, kept for the weight sums (log2 units): [T][Hq][scores_stride], or NULL
    float* scores;
    long long scores_stride;
};

struct EvictParams {
    int L, batch, H, d, keep, sinks, recent;
    const int* kv_len;
    const float* weight;
    long long weight_stride, kept_stride;
    int* kept;
    int* new_len;
    float* kept_weight;
    CacheView src, dst;
    unsigned* status;
    const void* sk[KVX_MAX_TARGET_LAYERS];
    const void* sv[KVX_MAX_TARGET_LAYERS];
    void* dk[KVX_MAX_TARGET_LAYERS];
    void* dv[KVX_MAX_TARGET_LAYERS];
};
cudaError_t launch_evict(const EvictParams& P, int dtype, int num_sms, cudaStream_t stream, int* launches);

// Workspace of split rows: rows of partial results (2 x grid x BM, so grids stay within it) and split items.
constexpr int kAttendMaxRows = 2 * 152 * 4 * 64;
constexpr long long kAttendScores = 16ll << 20;   // floats of kept scores: eight sequences of 64K, 32 query heads
constexpr int kAttendMaxCtas = kAttendMaxRows / 2 / 16;
cudaError_t launch_sum_scores(const AttendParams& P, cudaStream_t stream);
cudaError_t launch_key_weight(const AttendParams& P, int num_sms, cudaStream_t stream);
cudaError_t launch_attend_tc_capped(const AttendParams& P, int num_sms, cudaStream_t stream);
cudaError_t launch_attend_tc(const AttendParams& P, int num_sms, cudaStream_t stream);
cudaError_t launch_attend(const AttendParams& P, int dtype, int num_sms, cudaStream_t stream, int* launches);

// ------------------------------------------------------------------ sequences and masks
// Cached tokens of sequence b, clamped to the cache.
__device__ __forceinline__ int seq_slots(const int* kv_len, int capacity, int b, unsigned* status)
{
    int n = kv_len[b];
    if (n < 0 || n > capacity) {
        set_status(status, KVX_DEV_SEQ_CLAMPED);
        n = n < 0 ? 0 : capacity;
    }
    return n;
}

// One sequence of an attention call.
struct Seq {
    int t0, n, L, pre;     // first packed token, new tokens, cached slots, prefix slots
    // slot of new token t (may be negative when kv_len counts fewer tokens than the call has)
    __device__ __forceinline__ int slot(int t) const { return L - n + t; }
};
__device__ __forceinline__ Seq load_seq(const AttendParams& P, int b)
{
    Seq s;
    s.t0 = min(max(P.seq_off[b], 0), P.T);
    s.n = min(max(P.seq_off[b + 1], s.t0), P.T) - s.t0;
    s.L = seq_slots(P.kv_len, P.cache.capacity, b, P.status);
    s.pre = P.prefix_len ? min(max(P.prefix_len[b], 0), s.L) : 0;
    return s;
}
// First slot that the window leaves the token in slot i, and whether it sees slot j < L.
__device__ __forceinline__ int window_lo(const AttendParams& P, int i) { return P.window > 0 ? i - P.window + 1 : 0; }
__device__ __forceinline__ bool sees(const AttendParams& P, const Seq& s, int i, int j)
{
    return j < s.L && ((j <= i && j >= window_lo(P, i)) || j < s.pre);
}

// The slot tiles of BN that tokens [ta, tb] of a sequence see: tiles [0, n1) hold prefix slots, tiles
// [s2, s2 + n2) the rest.  At least one tile, so that rows that see nothing are written too.
struct KvTiles {
    int n1, s2, count;
    __device__ __forceinline__ int at(int i) const { return i < n1 ? i : s2 + (i - n1); }
};
template <int BN> __device__ __forceinline__ KvTiles kv_tiles(const AttendParams& P, const Seq& s, int ta, int tb)
{
    KvTiles k;
    const int hi = min(max(s.slot(tb) + 1, 0), s.L);
    const int lo = max(window_lo(P, s.slot(ta)), 0);
    k.n1 = (s.pre + BN - 1) / BN;
    k.s2 = max(lo / BN, k.n1);
    const int e2 = hi > lo ? (hi + BN - 1) / BN : 0;
    k.count = max(k.n1 + max(e2 - k.s2, 0), 1);
    return k;
}

// A row tile: tile_rows consecutive (token, query head) rows of one (sequence, KV head), row r = t * G + g.
__device__ __forceinline__ int row_tiles(const AttendParams& P, const Seq& s) { return (s.n * P.G + P.tile_rows - 1) / P.tile_rows; }
__device__ __forceinline__ void row_tile_tokens(const AttendParams& P, const Seq& s, int rt, int& ta, int& tb)
{
    ta = rt * P.tile_rows / P.G;
    tb = min(s.n, (rt * P.tile_rows + P.tile_rows - 1) / P.G + 1) - 1;
}

// ------------------------------------------------------------------ the split of the work
// The work is a line of slot tiles: for each sequence, each row tile its tiles in order.  A line for each KV head,
// H CTAs side by side on the same tiles of the H lines (their rows of K and V lie next to one another in
// memory), so CTA c = k H + h of N H takes [k W / N, (k + 1) W / N) of the W tiles of head h's line; where H does
// not divide the grid well, one line with the heads of a row tile one after the other.  Every CTA has the
// same number of tiles, whatever the lengths; a range may begin and end inside a row's tiles, whose partial
// results a second launch joins in order.  Every CTA finds its range itself: a warp per sequence
// sums the tiles of its row tiles.
struct Plan {
    long long W, lo, hi;      // tiles of a line; this CTA's range
    int N;                    // CTAs a line that have a range: no more than there are tiles
    int lines, line, cta;     // lines; this CTA's line and place on it
    int b, rt;                // row tile of the first one
    long long at;             // first tile of (b, rt) on the line
    __device__ __forceinline__ int heads(int H) const { return lines == 1 ? H : 1; }   // heads one after the other
};
__host__ __device__ inline int plan_lines(int grid, int H) { return grid / H * H * 10 >= grid * 9 ? H : 1; }

// sums: shared long long[batch + 1].  All threads call it; returns the same in each.
template <int BN, int THREADS>
__device__ Plan make_plan(const AttendParams& P, long long* sums)
{
    Plan p;
    p.lines = plan_lines(gridDim.x, P.H);
    p.line = blockIdx.x % p.lines;
    p.cta = blockIdx.x / p.lines;
    const int heads = p.heads(P.H);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int b = warp; b < P.batch; b += THREADS / 32) {
        const Seq s = load_seq(P, b);
        const int rts = row_tiles(P, s);
        long long w = 0;
        for (int rt = lane; rt < rts; rt += 32) {
            int ta, tb;
            row_tile_tokens(P, s, rt, ta, tb);
            w += kv_tiles<BN>(P, s, ta, tb).count;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
        if (lane == 0) sums[b + 1] = w * heads;
    }
    if (threadIdx.x == 0) sums[0] = 0;
    __syncthreads();
    if (warp == 0) {          // running sums over the sequences
        long long run = 0;
        for (int b0 = 0; b0 < P.batch; b0 += 32) {
            long long v = b0 + lane < P.batch ? sums[b0 + lane + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long u = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += u;
            }
            v += run;
            if (b0 + lane < P.batch) sums[b0 + lane + 1] = v;
            run = __shfl_sync(0xffffffffu, v, 31);
        }
    }
    __syncthreads();
    p.W = sums[P.batch];
    p.N = (int)min((long long)(gridDim.x / p.lines), p.W);
    p.b = 0; p.rt = 0; p.at = 0;
    if (p.cta >= p.N) { p.lo = p.hi = 0; return p; }
    p.lo = p.W * p.cta / p.N;
    p.hi = p.W * (p.cta + 1) / p.N;
    int l = 0, h = P.batch - 1;                  // the sequence that holds tile lo
    while (l < h) {
        const int m = (l + h + 1) >> 1;
        if (sums[m] <= p.lo) l = m; else h = m - 1;
    }
    p.b = l;
    p.at = sums[l];
    const Seq s = load_seq(P, l);
    const int rts = row_tiles(P, s);
    for (int r0 = 0; r0 < rts; r0 += 32) {       // and its row tile (each warp alike)
        long long w = 0;
        if (r0 + lane < rts) {
            int ta, tb;
            row_tile_tokens(P, s, r0 + lane, ta, tb);
            w = (long long)kv_tiles<BN>(P, s, ta, tb).count * heads;
        }
        long long v = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        const unsigned past = __ballot_sync(0xffffffffu, p.at + v > p.lo && r0 + lane < rts);
        if (past) {
            const int first = __ffs(past) - 1;
            p.rt = r0 + first;
            p.at += __shfl_sync(0xffffffffu, v - w, first);
            break;
        }
        p.at += __shfl_sync(0xffffffffu, v, 31);
    }
    return p;
}

// CTA of a line that holds tile x of W split over N.
__device__ __forceinline__ int tile_cta(long long x, long long W, int N)
{
    int c = (int)((x * N) / W);                  // c W / N <= x up to rounding down
    while (c > 0 && W * c / N > x) --c;
    while (c + 1 < N && W * (c + 1) / N <= x) ++c;
    return c;
}

// One CTA's share of one item (the tiles of a row tile and KV head): tiles [i0, i0 + n) of `count`.
struct Segment {
    int b, rt, h, i0, n;
    Seq s;
    KvTiles kv;
    long long start;          // first tile of the item on the line
    bool first;               // the CTA's first segment (its partial result goes to the CTA's slot 0, else 1)
    __device__ __forceinline__ bool whole() const { return n == kv.count; }
};
// Where a warp stands on its CTA's range.
struct WalkState {
    long long x, at;          // next tile; first tile of (b, rt) on the line
    int b, rt;
};
// plan and state may lie in shared memory (whole warps call next): in registers they would be live through a kernel's
// inner loop.
template <int BN> struct SegmentWalk {
    const AttendParams& P;
    const Plan* p;
    WalkState* w;
    __device__ __forceinline__ SegmentWalk(const AttendParams& P_, const Plan* p_, WalkState* w_) : P(P_), p(p_), w(w_)
    {
        __syncwarp();
        *w = {p->lo, p->at, p->b, p->rt};
        __syncwarp();
    }
    __device__ __forceinline__ bool next(Segment& g)
    {
        WalkState s = *w;
        if (s.x >= p->hi) return false;
        while (true) {
            g.s = load_seq(P, s.b);
            if (s.rt < row_tiles(P, g.s)) break;
            ++s.b;                               // a sequence without new tokens, or past its last row tile
            s.rt = 0;
        }
        int ta, tb;
        row_tile_tokens(P, g.s, s.rt, ta, tb);
        g.kv = kv_tiles<BN>(P, g.s, ta, tb);
        g.b = s.b;
        g.rt = s.rt;
        const int k = (int)((s.x - s.at) / g.kv.count);
        g.h = p->lines == 1 ? k : p->line;
        g.start = s.at + (long long)k * g.kv.count;
        g.i0 = (int)(s.x - g.start);
        g.n = (int)min((long long)(g.kv.count - g.i0), p->hi - s.x);
        g.first = s.x == p->lo;
        s.x += g.n;
        if (s.x == s.at + (long long)g.kv.count * p->heads(P.H)) {
            s.at = s.x;
            ++s.rt;
        }
        __syncwarp();
        *w = s;
        __syncwarp();
        return true;
    }
};

// The partial results of a split item: the CTAs of places c0 .. c0 + parts - 1 on a line hold them, the first in
// its slot slot0, the others in their slot 0; CTA c has slots 2 c and 2 c + 1.
struct Parts {
    int cta0, lines, parts, slot0;
    __device__ __forceinline__ int slot(int i) const { return 2 * (cta0 + i * lines) + (i == 0 ? slot0 : 0); }
};
__device__ __forceinline__ Parts item_parts(const Plan& p, const Segment& g)
{
    Parts r;
    const int c0 = tile_cta(g.start, p.W, p.N);
    r.lines = p.lines;
    r.cta0 = c0 * p.lines + p.line;
    r.parts = tile_cta(g.start + g.kv.count - 1, p.W, p.N) - c0 + 1;
    r.slot0 = g.start > p.W * c0 / p.N;
    return r;
}

// Base-2 exponential of the hardware (2 ulp).  The argument is at most 0, but for the weights of the tensor-core attention:
// there a row's maximum may stay behind by up to 8.
__device__ __forceinline__ float exp2_hw(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// tanh: an odd polynomial near zero, where 1 - 2 / (1 + e^2x) would lose the leading bits of a capped score;
// the Taylor series to x^13 leaves a relative error below 1e-7 up to |x| = 0.5.
__device__ __forceinline__ float tanh_series(float x)
{
    const float y = x * x;
    float p = 21844.0f / 6081075.0f;
    p = fmaf(p, y, -1382.0f / 155925.0f);
    p = fmaf(p, y, 62.0f / 2835.0f);
    p = fmaf(p, y, -17.0f / 315.0f);
    p = fmaf(p, y, 2.0f / 15.0f);
    p = fmaf(p, y, -1.0f / 3.0f);
    return fmaf(p * y, x, x);
}
__device__ __forceinline__ float tanh_far(float x)
{
    const float e = exp2_hw(fminf(fabsf(x), 20.0f) * -2.885390081777927f);   // e^(-2|x|)
    return copysignf(__fdividef(1.0f - e, 1.0f + e), x);
}
__device__ __forceinline__ float capped(float s, float cap, float inv_cap)
{
    const float x = s * inv_cap;
    return cap * (fabsf(x) < 0.5f ? tanh_series(x) : tanh_far(x));
}

}  // namespace kvx
