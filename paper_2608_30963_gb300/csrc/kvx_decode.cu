// kvx_decode.cu -- host side of the calls that go on from a cache: kvx_decoder_*, kvx_append,
// kvx_attend and kvx_evict (argument checks, workspace, launches).
#include <float.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <new>

#include "kvx_decode.cuh"

using namespace kvx;

struct kvx_decoder {
    kvx_decoder_desc desc;
    int num_sms = 0, max_position = 0, last_launches = 0;
    unsigned long long* turns = nullptr;   // fixed-point turns [head_dim/2]
    unsigned* status = nullptr;
    float* part_o = nullptr;               // partial results of split attention rows (kvx_decode.cuh)
    float2* part_ml = nullptr;
    SplitItem* split = nullptr;
    float* scores = nullptr;               // scores kept for the weight sums
};

namespace {

kvx_status fail(kvx_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
kvx_status fail(kvx_status s, const char* fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_last_error(buf);
    return s;
}

void free_decoder(kvx_decoder* d)
{
    if (d->turns) cudaFree(d->turns);
    if (d->status) cudaFree(d->status);
    if (d->part_o) cudaFree(d->part_o);
    if (d->part_ml) cudaFree(d->part_ml);
    if (d->split) cudaFree(d->split);
    if (d->scores) cudaFree(d->scores);
    delete d;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
int vec_of(const kvx_decoder* d) { return d->desc.dtype == KVX_BF16 ? 8 : 4; }

// Checks rows of `heads` heads a token.
kvx_status check_rows(const kvx_decoder* d, const char* who, const char* what, const kvx_rows* r)
{
    const int vec = vec_of(d);
    if (!r || !r->ptr) return fail(KVX_ERR_INVALID_ARG, "%s: %s is NULL", who, what);
    if (!aligned16(r->ptr) || r->stride_t < 1 || r->stride_h < 1 || r->stride_t % vec || r->stride_h % vec)
        return fail(KVX_ERR_INVALID_ARG, "%s: %s must be 16-byte aligned with strides that are positive multiples of %d elements",
                    who, what, vec);
    return KVX_OK;
}

kvx_status check_tokens(const kvx_decoder* d, const char* who, const kvx_new_tokens* tok)
{
    if (!tok) return fail(KVX_ERR_INVALID_ARG, "%s: NULL argument", who);
    if (tok->batch < 1 || tok->total_tokens < 0) return fail(KVX_ERR_INVALID_ARG, "%s: bad batch or total_tokens", who);
    if (!tok->seq_off || !tok->kv_len) return fail(KVX_ERR_INVALID_ARG, "%s: seq_off and kv_len must be set", who);
    if ((long long)tok->total_tokens * d->desc.num_q_heads >= 1ll << 30)
        return fail(KVX_ERR_UNSUPPORTED, "%s: 2^30 or more (token, query head) rows in one call", who);
    return KVX_OK;
}

// The view of a cache, layers [l0, l0 + n) of it checked.
kvx_status make_view(const kvx_decoder* d, const char* who, const char* what, const kvx_dst_kv* c, int l0, int n, CacheView& v)
{
    const int vec = vec_of(d), dim = d->desc.model.head_dim;
    if (!c || !c->k || !c->v) return fail(KVX_ERR_INVALID_ARG, "%s: %s is NULL", who, what);
    memset(&v, 0, sizeof v);
    v.H = d->desc.model.num_kv_heads;
    v.d = dim;
    v.paged = c->paged != 0;
    v.page_shift = -1;
    if (!c->paged) {
        if (c->stride_t < dim || c->stride_h < 1 || c->stride_b < 1 || c->stride_t % vec || c->stride_h % vec ||
            c->stride_b % vec || c->max_seq < 0 || c->max_seq > 1 << 30)
            return fail(KVX_ERR_INVALID_ARG, "%s: strides of %s must be positive multiples of %d elements with stride_t >= head_dim, "
                                             "max_seq in [0, 2^30]", who, what, vec);
        v.capacity = c->max_seq;
        v.sb = c->stride_b; v.sh = c->stride_h; v.st = c->stride_t;
    } else {
        if (!c->page_table || c->page_size < 1 || c->max_pages_per_seq < 1 || c->num_pages < 1)
            return fail(KVX_ERR_INVALID_ARG, "%s: a paged %s needs page_table, page_size, max_pages_per_seq and num_pages >= 1", who,
                        what);
        const long long cap = (long long)c->page_size * c->max_pages_per_seq;
        v.capacity = (int)(cap < 1 << 30 ? cap : 1 << 30);
        v.page_table = c->page_table;
        v.max_pages = c->max_pages_per_seq; v.page_size = c->page_size; v.num_pages = c->num_pages;
        if ((c->page_size & (c->page_size - 1)) == 0) v.page_shift = __builtin_ctz((unsigned)c->page_size);
    }
    for (int l = l0; l < l0 + n; ++l) {
        if (!c->k[l] || !c->v[l]) return fail(KVX_ERR_INVALID_ARG, "%s: NULL cache pointer in %s, layer %d", who, what, l);
        if (!aligned16(c->k[l]) || !aligned16(c->v[l]))
            return fail(KVX_ERR_INVALID_ARG, "%s: cache pointers must be 16-byte aligned (%s, layer %d)", who, what, l);
    }
    return KVX_OK;
}

// Do `units` rows of sa floats from a and of sb floats from b share an address?  (Without products, which could wrap.)
bool rows_overlap(long long units, const float* a, long long sa, const float* b, long long sb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x <= y ? (y - x) / 4 / (uintptr_t)units < (uintptr_t)sa : (x - y) / 4 / (uintptr_t)units < (uintptr_t)sb;
}

kvx_status check_layer(const kvx_decoder* d, const char* who, int layer)
{
    if (layer < 0 || layer >= d->desc.model.num_layers)
        return fail(KVX_ERR_INVALID_ARG, "%s: layer %d outside [0, %d)", who, layer, d->desc.model.num_layers);
    return KVX_OK;
}

}  // namespace

extern "C" KVX_API kvx_status kvx_decoder_create(const kvx_decoder_desc* desc, kvx_decoder** out)
{
    if (!desc || !out) return fail(KVX_ERR_INVALID_ARG, "decoder_create: NULL argument");
    *out = nullptr;
    const kvx_model_geom& g = desc->model;
    if (g.num_layers < 1 || g.num_kv_heads < 1 || desc->num_q_heads < 1)
        return fail(KVX_ERR_INVALID_ARG, "decoder_create: layer and head counts must be >= 1");
    if (g.head_dim != 64 && g.head_dim != 128 && g.head_dim != 256)
        return fail(KVX_ERR_UNSUPPORTED, "decoder_create: head_dim must be 64, 128 or 256 (got %d)", g.head_dim);
    if (desc->num_q_heads % g.num_kv_heads != 0 || desc->num_q_heads / g.num_kv_heads > 64)
        return fail(KVX_ERR_UNSUPPORTED, "decoder_create: num_q_heads must be a multiple of num_kv_heads, at most 64 times it (%d, %d)",
                    desc->num_q_heads, g.num_kv_heads);
    if (desc->dtype != KVX_BF16 && desc->dtype != KVX_FP32)
        return fail(KVX_ERR_INVALID_ARG, "decoder_create: unknown dtype %d", desc->dtype);
    if (!rope_schedule_ok(g))
        return fail(KVX_ERR_INVALID_ARG, "decoder_create: unknown rope_type, schedule parameters out of range or rotary_dim not 0 or a "
                                         "multiple of 16 in [16, head_dim]");
    const int max_pos = desc->max_position ? desc->max_position : 1 << 24;
    if (max_pos < 1 || max_pos > 1 << 30) return fail(KVX_ERR_INVALID_ARG, "decoder_create: max_position must be in [1, 1<<30]");
    if (!(desc->scale >= 0.0) || !isfinite(desc->scale) || !(desc->score_cap >= 0.0) || !isfinite(desc->score_cap))
        return fail(KVX_ERR_INVALID_ARG, "decoder_create: scale and score_cap must be finite and not negative");
    // the kernels hold them, and what a scaled score is divided by, in 32 bits
    const double scale = desc->scale > 0.0 ? desc->scale : 1.0 / sqrt((double)g.head_dim);
    auto normal = [](double x) { return x >= FLT_MIN && x <= FLT_MAX; };
    if (!normal(scale) || (desc->score_cap > 0.0 && (!normal(desc->score_cap) || !normal(1.0 / desc->score_cap) || !normal(scale / desc->score_cap))))
        return fail(KVX_ERR_INVALID_ARG, "decoder_create: scale, score_cap, 1 / score_cap and scale / score_cap must be normal numbers in 32 bits");
    kvx_decoder* d = new (std::nothrow) kvx_decoder();
    if (!d) return fail(KVX_ERR_OOM, "decoder_create: host allocation");
    d->desc = *desc;
    d->desc.scale = scale;
    d->max_position = max_pos;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&d->num_sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        delete d;
        return fail(KVX_ERR_CUDA, "decoder_create: no CUDA device");
    }
    unsigned long long turns[128] = {};
    if (g.rope_base > 0.0)
        for (int i = 0; i < rope_rot_dim(g) / 2; ++i) turns[i] = (unsigned long long)ldexp(rope_inv_freq(g, i) / (2.0 * M_PI), 64);
    const size_t rows = kAttendMaxRows;
    if (cudaMalloc(&d->turns, sizeof turns) != cudaSuccess || cudaMalloc(&d->status, sizeof(unsigned)) != cudaSuccess ||
        cudaMalloc(&d->part_o, rows * g.head_dim * sizeof(float)) != cudaSuccess ||
        cudaMalloc(&d->part_ml, rows * sizeof(float2)) != cudaSuccess ||
        cudaMalloc(&d->split, kAttendMaxCtas * sizeof(SplitItem)) != cudaSuccess ||
        cudaMalloc(&d->scores, kAttendScores * sizeof(float)) != cudaSuccess) {
        cudaGetLastError();
        free_decoder(d);
        return fail(KVX_ERR_OOM, "decoder_create: device allocation");
    }
    cudaError_t e;
    if ((e = cudaMemcpy(d->turns, turns, sizeof turns, cudaMemcpyHostToDevice)) != cudaSuccess ||
        (e = cudaMemset(d->status, 0, sizeof(unsigned))) != cudaSuccess ||
        (e = cudaDeviceSynchronize()) != cudaSuccess) {
        free_decoder(d);
        return fail(KVX_ERR_CUDA, "decoder_create: %s", cudaGetErrorString(e));
    }
    *out = d;
    return KVX_OK;
}

extern "C" KVX_API kvx_status kvx_decoder_destroy(kvx_decoder* dec)
{
    if (!dec) return KVX_OK;
    cudaDeviceSynchronize();
    free_decoder(dec);
    return KVX_OK;
}

extern "C" KVX_API kvx_status kvx_append(kvx_decoder* dec, const kvx_new_tokens* tok, const kvx_rows* q, const kvx_rows* k,
                                         const kvx_rows* v, const kvx_rows* q_out, const kvx_dst_kv* cache, int32_t layer,
                                         void* stream)
{
    if (!dec) return fail(KVX_ERR_INVALID_ARG, "append: NULL decoder");
    dec->last_launches = 0;
    kvx_status st;
    AppendParams P;
    memset(&P, 0, sizeof P);
    if ((st = check_tokens(dec, "append", tok)) || (st = check_layer(dec, "append", layer))) return st;
    if (tok->total_tokens == 0) return KVX_OK;
    if ((st = check_rows(dec, "append", "q", q)) || (st = check_rows(dec, "append", "k", k)) ||
        (st = check_rows(dec, "append", "v", v)) || (st = check_rows(dec, "append", "q_out", q_out)) ||
        (st = make_view(dec, "append", "the cache", cache, layer, 1, P.cache)))
        return st;
    const kvx_model_geom& g = dec->desc.model;
    P.T = tok->total_tokens; P.batch = tok->batch;
    P.Hq = dec->desc.num_q_heads; P.H = g.num_kv_heads; P.d = g.head_dim;
    P.rhalf = rope_rot_dim(g) / 2; P.rope = g.rope_base > 0.0; P.max_position = dec->max_position;
    P.seq_off = tok->seq_off; P.kv_len = tok->kv_len; P.pos = tok->pos;
    P.turns = dec->turns;
    P.q = q->ptr; P.q_t = q->stride_t; P.q_h = q->stride_h;
    P.k = k->ptr; P.k_t = k->stride_t; P.k_h = k->stride_h;
    P.v = v->ptr; P.v_t = v->stride_t; P.v_h = v->stride_h;
    P.q_out = q_out->ptr; P.o_t = q_out->stride_t; P.o_h = q_out->stride_h;
    P.ck = cache->k[layer]; P.cv = cache->v[layer];
    P.status = dec->status;
    const cudaError_t e = launch_append(P, dec->desc.dtype, (cudaStream_t)stream);
    if (e != cudaSuccess) return fail(KVX_ERR_CUDA, "append: launch failed: %s", cudaGetErrorString(e));
    dec->last_launches = 1;
    return KVX_OK;
}

extern "C" KVX_API kvx_status kvx_attend(kvx_decoder* dec, const kvx_new_tokens* tok, const kvx_rows* q, const kvx_dst_kv* cache,
                                         int32_t layer, const kvx_attend_opts* opts, const kvx_rows* out, void* stream)
{
    if (!dec) return fail(KVX_ERR_INVALID_ARG, "attend: NULL decoder");
    dec->last_launches = 0;
    static const kvx_attend_opts none = {};
    if (!opts) opts = &none;
    kvx_status st;
    AttendParams P;
    memset(&P, 0, sizeof P);
    if ((st = check_tokens(dec, "attend", tok)) || (st = check_layer(dec, "attend", layer))) return st;
    if (tok->total_tokens == 0) return KVX_OK;
    if ((st = check_rows(dec, "attend", "q", q)) || (st = check_rows(dec, "attend", "out", out)) ||
        (st = make_view(dec, "attend", "the cache", cache, layer, 1, P.cache)))
        return st;
    if (tok->batch > kMaxAttendBatch) return fail(KVX_ERR_UNSUPPORTED, "attend: at most %d sequences a call", kMaxAttendBatch);
    if (opts->window < 0) return fail(KVX_ERR_INVALID_ARG, "attend: window must not be negative");
    if (opts->key_weight && (!opts->lse || opts->weight_stride < 1))
        return fail(KVX_ERR_INVALID_ARG, "attend: key_weight needs lse and weight_stride >= 1");
    const kvx_model_geom& g = dec->desc.model;
    P.T = tok->total_tokens; P.batch = tok->batch;
    P.Hq = dec->desc.num_q_heads; P.H = g.num_kv_heads; P.G = P.Hq / P.H; P.d = g.head_dim;
    P.seq_off = tok->seq_off; P.kv_len = tok->kv_len;
    P.q = q->ptr; P.q_t = q->stride_t; P.q_h = q->stride_h;
    P.out = out->ptr; P.o_t = out->stride_t; P.o_h = out->stride_h;
    P.ck = cache->k[layer]; P.cv = cache->v[layer];
    P.scale = (float)dec->desc.scale; P.cap = (float)dec->desc.score_cap;
    // Slots lie in [-2^30, 2^30), those seen from zero on: a window of 2^30 hides none, and slot - window does not wrap.
    P.window = opts->window < 1 << 30 ? opts->window : 1 << 30; P.prefix_len = opts->prefix_len;
    P.lse = opts->lse; P.key_weight = opts->key_weight; P.weight_stride = opts->weight_stride;
    P.status = dec->status;
    P.part_o = dec->part_o; P.part_ml = dec->part_ml; P.split = dec->split;
    P.scores = dec->scores;
    const cudaError_t e = launch_attend(P, dec->desc.dtype, dec->num_sms, (cudaStream_t)stream, &dec->last_launches);
    if (e != cudaSuccess) return fail(KVX_ERR_CUDA, "attend: launch failed: %s", cudaGetErrorString(e));
    return KVX_OK;
}

extern "C" KVX_API kvx_status kvx_evict(kvx_decoder* dec, const kvx_evict_plan* plan, const kvx_dst_kv* src, const kvx_dst_kv* dst,
                                        void* stream)
{
    if (!dec || !plan) return fail(KVX_ERR_INVALID_ARG, "evict: NULL argument");
    dec->last_launches = 0;
    const int L = plan->num_layers;
    if (plan->batch < 1 || L < 1 || L > KVX_MAX_TARGET_LAYERS || L > dec->desc.model.num_layers)
        return fail(KVX_ERR_INVALID_ARG, "evict: batch must be >= 1 and num_layers in [1, %d], at most the model's", KVX_MAX_TARGET_LAYERS);
    // (a cache holds at most 2^30 slots; the kernels step past keep by a block's threads)
    if (plan->keep < 1 || plan->keep > 1 << 30 || plan->sinks < 0 || plan->recent < 0 || (long long)plan->sinks + plan->recent > plan->keep)
        return fail(KVX_ERR_INVALID_ARG, "evict: need keep in [1, 2^30], sinks and recent >= 0 and sinks + recent <= keep");
    if (!plan->kv_len || !plan->key_weight || !plan->kept || !plan->new_len)
        return fail(KVX_ERR_INVALID_ARG, "evict: kv_len, key_weight, kept and new_len must be set");
    if (plan->weight_stride < 1 || (plan->kept_weight && plan->kept_weight_stride < plan->keep))
        return fail(KVX_ERR_INVALID_ARG, "evict: weight_stride must be >= 1 and kept_weight_stride >= keep");
    const long long units = (long long)L * plan->batch * dec->desc.model.num_kv_heads;
    if (units > 0x7fffffffll) return fail(KVX_ERR_UNSUPPORTED, "evict: too many (layer, sequence, head) units in one call");
    if (plan->kept_weight && rows_overlap(units, plan->key_weight, plan->weight_stride, plan->kept_weight, plan->kept_weight_stride))
        return fail(KVX_ERR_INVALID_ARG, "evict: kept_weight must not overlap key_weight");
    EvictParams P;
    memset(&P, 0, sizeof P);
    kvx_status st;
    if ((st = make_view(dec, "evict", "the source cache", src, 0, L, P.src)) ||
        (st = make_view(dec, "evict", "the destination cache", dst, 0, L, P.dst)))
        return st;
    P.L = L; P.batch = plan->batch; P.H = dec->desc.model.num_kv_heads; P.d = dec->desc.model.head_dim;
    P.keep = plan->keep; P.sinks = plan->sinks; P.recent = plan->recent;
    P.kv_len = plan->kv_len; P.weight = plan->key_weight; P.weight_stride = plan->weight_stride;
    P.kept = plan->kept; P.new_len = plan->new_len; P.kept_weight = plan->kept_weight; P.kept_stride = plan->kept_weight_stride;
    P.status = dec->status;
    for (int l = 0; l < L; ++l) {
        P.sk[l] = src->k[l]; P.sv[l] = src->v[l];
        P.dk[l] = dst->k[l]; P.dv[l] = dst->v[l];
    }
    const cudaError_t e = launch_evict(P, dec->desc.dtype, dec->num_sms, (cudaStream_t)stream, &dec->last_launches);
    if (e != cudaSuccess) return fail(KVX_ERR_CUDA, "evict: launch failed: %s", cudaGetErrorString(e));
    return KVX_OK;
}

extern "C" KVX_API kvx_status kvx_decoder_status(kvx_decoder* dec, void* stream, uint32_t* bits, int32_t clear)
{
    if (!dec) return fail(KVX_ERR_INVALID_ARG, "decoder_status: NULL decoder");
    unsigned v = 0;
    cudaError_t e;
    if ((e = cudaStreamSynchronize((cudaStream_t)stream)) != cudaSuccess ||
        (e = cudaMemcpy(&v, dec->status, sizeof v, cudaMemcpyDeviceToHost)) != cudaSuccess ||
        (clear && (e = cudaMemset(dec->status, 0, sizeof v)) != cudaSuccess))
        return fail(KVX_ERR_CUDA, "decoder_status: %s", cudaGetErrorString(e));
    if (bits) *bits = v;
    if (v) return fail(KVX_ERR_DEVICE_STATUS, "device status 0x%x", v);
    return KVX_OK;
}

extern "C" KVX_API int32_t kvx_decoder_launches(const kvx_decoder* dec) { return dec ? dec->last_launches : 0; }
