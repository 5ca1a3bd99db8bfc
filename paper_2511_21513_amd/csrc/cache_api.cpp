// Host side of the operators around the paged cache (include/intattn.h): argument checks, the room that the
// context lends them, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <string>

#include "cache_params.h"
#include "context.h"
#include "work_map.h"

namespace {

constexpr int64_t MOST_SLOTS = 1ll << 30; // of a sequence
constexpr int32_t MOST_KEYS = 131071;     // of a row whose integer sums stay in 32 bits
constexpr int64_t MOST_TOKENS = (1 << 24) - 1; // of a call: up to a workgroup of 256 threads each, and a grid's threads number below 2^32

bool strides_ok(const int64_t *st, int n, int64_t multiple)
{
    for (int i = 0; i < n; ++i)
        if (st[i] < 0 || st[i] % multiple != 0) return false;
    return true;
}
// what is written must not lie over itself: a stride below a row, along an axis of more than one
bool apart(const int64_t *st, int64_t n0, int64_t n1, int64_t n2, int64_t row) { return (n0 == 1 || st[0] >= row) && (n1 == 1 || st[1] >= row) && (n2 == 1 || st[2] >= row); }
bool apart(const int64_t *st, int64_t n0, int64_t n1) { return (n0 == 1 || st[0] >= 1) && (n1 == 1 || st[1] >= 1); }
bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

int check_ctx(intattn_ctx *ctx, const void *args)
{
    if (!ctx) return INTATTN_ERR_INVALID_ARG;
    if (!args) return fail(ctx, INTATTN_ERR_INVALID_ARG, "args is NULL");
    return INTATTN_OK;
}

// after the arguments' checks, which need no device
int check_device(intattn_ctx *ctx)
{
    return ctx->device < 0 ? fail(ctx, INTATTN_ERR_UNSUPPORTED, "host-only context: no device to run on") : INTATTN_OK;
}

int check_cache(intattn_ctx *ctx, const intattn_cache *c, CacheParams *p)
{
    if (!c) return fail(ctx, INTATTN_ERR_INVALID_ARG, "cache is NULL");
    if (c->B < 1 || c->Hkv < 1 || c->n_pages < 1 || c->page_size < 1 || c->max_pages < 1)
        return fail(ctx, INTATTN_ERR_INVALID_ARG, "B, Hkv, n_pages, page_size, max_pages must be >= 1");
    if (c->d != 64 && c->d != 128) return fail(ctx, INTATTN_ERR_UNSUPPORTED, "d must be 64 or 128");
    if (c->B > 65535 || c->Hkv > 65535 || (int64_t)c->B * c->Hkv > 65535) return fail(ctx, INTATTN_ERR_UNSUPPORTED, "B * Hkv must not exceed 65535");
    if (c->page_size > 65536) return fail(ctx, INTATTN_ERR_UNSUPPORTED, "page_size must not exceed 65536");
    if ((int64_t)c->max_pages * c->page_size > MOST_SLOTS) return fail(ctx, INTATTN_ERR_UNSUPPORTED, "max_pages * page_size must not exceed 2^30");
    if (c->scale_mode != 0 && c->scale_mode != 1) return fail(ctx, INTATTN_ERR_INVALID_ARG, "the cache's scale_mode must be 0 or 1");
    if (c->reserved != 0) return fail(ctx, INTATTN_ERR_INVALID_ARG, "reserved must be 0");
    if (!c->k || !c->v || !c->table || !c->lens || !c->scale_k || !c->scale_v)
        return fail(ctx, INTATTN_ERR_INVALID_ARG, "k, v, table, lens, scale_k, scale_v must be non-NULL");
    if (!aligned(c->k, 16) || !aligned(c->v, 16)) return fail(ctx, INTATTN_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
    if (!strides_ok(c->k_stride, 3, 16) || !strides_ok(c->v_stride, 3, 16))
        return fail(ctx, INTATTN_ERR_INVALID_ARG, "strides of k and v must be non-negative multiples of 16");
    if ((c->page_size > 1 && (c->k_stride[2] < c->d || c->v_stride[2] < c->d)))
        return fail(ctx, INTATTN_ERR_INVALID_ARG, "the key strides must cover a row of d bytes");
    if (!aligned(c->table, 4) || !aligned(c->lens, 4) || !aligned(c->scale_k, 4) || !aligned(c->scale_v, 4))
        return fail(ctx, INTATTN_ERR_INVALID_ARG, "table, lens and scales must be 4-byte aligned");
    if (c->table_stride < 0 || (c->B > 1 && c->table_stride < c->max_pages))
        return fail(ctx, INTATTN_ERR_INVALID_ARG, "table_stride must be at least max_pages");
    p->k = c->k; p->v = c->v;
    for (int i = 0; i < 3; ++i) { p->ks[i] = c->k_stride[i]; p->vs[i] = c->v_stride[i]; }
    p->table = c->table; p->table_stride = c->table_stride;
    p->lens = c->lens;
    p->scale_k = c->scale_k; p->scale_v = c->scale_v;
    p->B = c->B; p->Hkv = c->Hkv;
    p->n_pages = c->n_pages; p->page_size = c->page_size;
    p->capacity = c->max_pages * c->page_size;
    p->per_head = c->scale_mode;
    p->by_page = fast_div((uint32_t)c->page_size);
    return INTATTN_OK;
}

bool writable(const intattn_cache *c) { return apart(c->k_stride, c->n_pages, c->Hkv, 1, c->d) && apart(c->v_stride, c->n_pages, c->Hkv, 1, c->d); }

// max_len of a call into the parameters' capacity
int bound_len(intattn_ctx *ctx, int32_t max_len, CacheParams *p)
{
    if (max_len < 0) return fail(ctx, INTATTN_ERR_INVALID_ARG, "max_len must be >= 0");
    if (max_len > 0) p->capacity = std::min(p->capacity, max_len);
    if (p->capacity > MOST_KEYS)
        return fail(ctx, INTATTN_ERR_UNSUPPORTED, "at most 131071 keys: give a max_len where max_pages * page_size is more");
    return INTATTN_OK;
}

// rot = 0 (allowed where `optional`): no rotation
int check_rotary(intattn_ctx *ctx, const intattn_rotary &r, int d, bool optional, RotaryParams *p)
{
    if (r.rot == 0 && optional) {
        p->rot = 0;
        return INTATTN_OK;
    }
    if (r.rot < 16 || r.rot % 16 != 0 || r.rot > d || r.rot > 256)
        return fail(ctx, INTATTN_ERR_UNSUPPORTED, "rot must be a multiple of 16, at most d and 256");
    if (r.pairing != 0 && r.pairing != 1) return fail(ctx, INTATTN_ERR_INVALID_ARG, "pairing must be 0 or 1");
    if (r.inverse != 0 && r.inverse != 1) return fail(ctx, INTATTN_ERR_INVALID_ARG, "inverse must be 0 or 1");
    if (r.n_axes < 1 || r.n_axes > 4) return fail(ctx, INTATTN_ERR_INVALID_ARG, "n_axes must be in 1..4");
    if (!r.pos || !r.freq) return fail(ctx, INTATTN_ERR_INVALID_ARG, "pos and freq must be non-NULL");
    if (!aligned(r.pos, 4) || !aligned(r.freq, 8)) return fail(ctx, INTATTN_ERR_INVALID_ARG, "pos must be 4-byte aligned and freq 8-byte aligned");
    if (!strides_ok(r.pos_stride, 3, 1)) return fail(ctx, INTATTN_ERR_INVALID_ARG, "strides of pos must be >= 0");
    std::memset(p->axis, 0, sizeof(p->axis));
    for (int i = 0; i < r.rot / 2; ++i) {
        if (r.axis[i] >= r.n_axes) return fail(ctx, INTATTN_ERR_INVALID_ARG, "an axis of a pair is not below n_axes");
        p->axis[i / 4] |= (uint32_t)r.axis[i] << (8 * (i % 4));
    }
    p->pos = r.pos; p->freq = r.freq;
    for (int i = 0; i < 3; ++i) p->ps[i] = r.pos_stride[i];
    p->rot = r.rot; p->halves = r.pairing; p->inverse = r.inverse;
    return INTATTN_OK;
}

// Room of at least `bytes` on the context.  A larger piece replaces a smaller one at least doubled, up to SCORE_ROOM, and the smaller
// stays allocated: graphs that were captured with it may be replayed.
int room(intattn_ctx *ctx, int64_t bytes, void *stream, bool may_launch, void **out)
{
    *out = ctx->d_cache_room;
    if (bytes <= 0 || (uint64_t)bytes <= ctx->cache_room_bytes) return INTATTN_OK;
    if (may_launch) {
        hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
        const hipError_t e = hipStreamIsCapturing((hipStream_t)stream, &cap);
        if (e != hipSuccess) return hip_fail(ctx, e, "hipStreamIsCapturing");
        if (cap != hipStreamCaptureStatusNone)
            return fail(ctx, INTATTN_ERR_NOMEM, "a captured call lacks room for its scores or moves: call intattn_cache_reserve before the capture");
    }
    ctx->cache_room_outgrown.reserve(ctx->cache_room_outgrown.size() + 1); // (throws before anything is allocated)
    const size_t want = std::max((size_t)bytes, std::min(2 * ctx->cache_room_bytes, (size_t)SCORE_ROOM));
    void *m = nullptr;
    size_t got = want;
    hipError_t e = hipMalloc(&m, got);
    if (e != hipSuccess && got > (size_t)bytes) {
        (void)hipGetLastError();
        got = (size_t)bytes;
        e = hipMalloc(&m, got);
    }
    if (e != hipSuccess) {
        (void)hipGetLastError();
        return fail(ctx, INTATTN_ERR_NOMEM, std::string("hipMalloc of room for scores or moves: ") + hipGetErrorString(e));
    }
    if (ctx->d_cache_room) ctx->cache_room_outgrown.push_back(ctx->d_cache_room);
    ctx->d_cache_room = m;
    ctx->cache_room_bytes = got;
    *out = m;
    return INTATTN_OK;
}

int forward_params(intattn_ctx *ctx, const intattn_cache *cache, const intattn_cache_forward_args *a, AttendParams *p)
{
    std::memset(p, 0, sizeof(*p));
    int rc = check_cache(ctx, cache, &p->c);
    if (rc) return rc;
    if (a->Hq < 1 || a->L < 1) return fail(ctx, INTATTN_ERR_INVALID_ARG, "Hq and L must be >= 1");
    if (a->Hq % cache->Hkv != 0) return fail(ctx, INTATTN_ERR_INVALID_ARG, "Hq must be a multiple of Hkv");
    if ((int64_t)(a->Hq / cache->Hkv) * a->L > 4096) return fail(ctx, INTATTN_ERR_UNSUPPORTED, "Hq / Hkv * L must not exceed 4096");
    rc = bound_len(ctx, a->max_len, &p->c);
    if (rc) return rc;
    if (a->out_type < 0 || a->out_type > 3) return fail(ctx, INTATTN_ERR_INVALID_ARG, "out_type must be 0 (fp32), 1 (fp16), 2 (bf16) or 3 (INT8)");
    if (a->scale_out_mode != 0 && a->scale_out_mode != 1) return fail(ctx, INTATTN_ERR_INVALID_ARG, "scale_out_mode must be 0 or 1");
    if (!a->q || !a->scale_q || !a->out) return fail(ctx, INTATTN_ERR_INVALID_ARG, "q, scale_q, out must be non-NULL");
    if (!aligned(a->q, 16) || !aligned(a->out, 16) || !strides_ok(a->q_stride, 3, 16) || !strides_ok(a->out_stride, 3, 16))
        return fail(ctx, INTATTN_ERR_INVALID_ARG, "q, out and their strides must be multiples of 16");
    if (!apart(a->out_stride, cache->B, a->Hq, a->L, (int64_t)cache->d * (a->out_type == 0 ? 4 : a->out_type == 3 ? 1 : 2)))
        return fail(ctx, INTATTN_ERR_INVALID_ARG, "the strides of out must cover a row");
    if (!aligned(a->scale_q, 4) || !aligned(a->scale_out, 4) || !aligned(a->n_new, 4) || !aligned(a->weight, 4) || !aligned(a->weight_out, 4))
        return fail(ctx, INTATTN_ERR_INVALID_ARG, "scales, n_new and weights must be 4-byte aligned");
    if ((a->weight == nullptr) != (a->weight_out == nullptr)) return fail(ctx, INTATTN_ERR_INVALID_ARG, "weight and weight_out go together");
    if (a->weight) {
        if (!strides_ok(a->weight_stride, 2, 1) || !strides_ok(a->weight_out_stride, 2, 1))
            return fail(ctx, INTATTN_ERR_INVALID_ARG, "strides of the weights must be >= 0");
        if (a->weight == a->weight_out && (a->weight_stride[0] != a->weight_out_stride[0] || a->weight_stride[1] != a->weight_out_stride[1]))
            return fail(ctx, INTATTN_ERR_INVALID_ARG, "weight_out is weight with other strides");
        if (!apart(a->weight_out_stride, cache->B, cache->Hkv)) return fail(ctx, INTATTN_ERR_INVALID_ARG, "planes that are written must not lie over each other");
        if (!std::isfinite(a->decay)) return fail(ctx, INTATTN_ERR_INVALID_ARG, "decay must be finite");
    }
    p->q = a->q; p->scale_q = a->scale_q; p->n_new = a->n_new;
    p->out = (uint8_t *)a->out;
    for (int i = 0; i < 3; ++i) { p->qs[i] = a->q_stride[i]; p->os[i] = a->out_stride[i]; }
    p->scale_out = a->out_type == 3 ? a->scale_out : nullptr;
    p->out_per_head = a->scale_out_mode;
    p->weight = a->weight; p->weight_out = a->weight_out;
    for (int i = 0; i < 2; ++i) { p->wst[i] = a->weight_stride[i]; p->wost[i] = a->weight_out_stride[i]; }
    p->decay = a->decay;
    p->Hq = a->Hq; p->L = a->L; p->group = a->Hq / cache->Hkv;
    p->rows = p->group * a->L; p->blocks = (p->rows + 15) / 16;
    p->out_type = a->out_type;
    p->top = (1 << ctx->lut_bits) - 1;
    p->clip = ctx->clip; p->sqrt_d = std::sqrt((double)cache->d);
    std::memcpy(p->lut, ctx->lut, 64);
    return INTATTN_OK;
}

int evict_params(intattn_ctx *ctx, const intattn_cache *cache, const intattn_evict_args *a, EvictParams *p)
{
    std::memset(p, 0, sizeof(*p));
    int rc = check_cache(ctx, cache, &p->c);
    if (rc) return rc;
    if (a->keep < 1 || a->sink < 0 || a->recent < 0) return fail(ctx, INTATTN_ERR_INVALID_ARG, "keep must be >= 1, sink and recent >= 0");
    rc = bound_len(ctx, a->max_len, &p->c);
    if (rc) return rc;
    if (!a->weight || !a->weight_out || !a->lens_out) return fail(ctx, INTATTN_ERR_INVALID_ARG, "weight, weight_out, lens_out must be non-NULL");
    if ((a->order == nullptr) != (a->order_out == nullptr)) return fail(ctx, INTATTN_ERR_INVALID_ARG, "order and order_out go together");
    if (!aligned(a->weight, 4) || !aligned(a->weight_out, 4) || !aligned(a->order, 4) || !aligned(a->order_out, 4) || !aligned(a->total, 4) || !aligned(a->lens_out, 4))
        return fail(ctx, INTATTN_ERR_INVALID_ARG, "weights, orders, total and lens_out must be 4-byte aligned");
    if (!strides_ok(a->weight_stride, 2, 1) || !strides_ok(a->weight_out_stride, 2, 1) || !strides_ok(a->order_stride, 2, 1) || !strides_ok(a->order_out_stride, 2, 1))
        return fail(ctx, INTATTN_ERR_INVALID_ARG, "strides of weights and orders must be >= 0");
    if (!apart(a->weight_out_stride, cache->B, cache->Hkv) || (a->order && !apart(a->order_out_stride, cache->B, cache->Hkv)))
        return fail(ctx, INTATTN_ERR_INVALID_ARG, "planes that are written must not lie over each other");
    if (!writable(cache)) return fail(ctx, INTATTN_ERR_INVALID_ARG, "pages and heads of a cache that is written to must not lie over each other");
    for (int i = 0; i < 2; ++i)
        if ((a->weight == a->weight_out && a->weight_stride[i] != a->weight_out_stride[i]) ||
            (a->order && a->order == a->order_out && a->order_stride[i] != a->order_out_stride[i]))
            return fail(ctx, INTATTN_ERR_INVALID_ARG, "an output that is its input has other strides");
    p->keep = a->keep; p->sink = a->sink; p->recent = a->recent;
    p->weight = a->weight; p->weight_out = a->weight_out;
    p->order = a->order; p->order_out = a->order_out;
    for (int i = 0; i < 2; ++i) {
        p->wst[i] = a->weight_stride[i]; p->wost[i] = a->weight_out_stride[i];
        p->ost[i] = a->order_stride[i]; p->oost[i] = a->order_out_stride[i];
    }
    p->total = a->total; p->lens_out = a->lens_out;
    p->d = cache->d;
    return INTATTN_OK;
}

// Nothing crosses the C boundary but return codes.
template <class F> int guarded(intattn_ctx *ctx, F f) noexcept
{
    try {
        return f();
    } catch (...) {
        if (ctx) ctx->err.clear();
        return INTATTN_ERR_NOMEM;
    }
}

} // namespace

extern "C" {

int intattn_rope(intattn_ctx *ctx, const intattn_rope_args *a, void *hip_stream)
{
    return guarded(ctx, [&]() -> int {
        int rc = check_ctx(ctx, a);
        if (rc) return rc;
        if (a->B < 1 || a->L < 1 || a->H[0] < 1 || a->H[1] < 0) return fail(ctx, INTATTN_ERR_INVALID_ARG, "B, L and H[0] must be >= 1, H[1] >= 0");
        if (a->d < 16 || a->d % 16 != 0 || a->d > 1024) return fail(ctx, INTATTN_ERR_UNSUPPORTED, "d must be a multiple of 16, at most 1024");
        if (a->dtype < 0 || a->dtype > 2) return fail(ctx, INTATTN_ERR_INVALID_ARG, "dtype must be 0 (fp32), 1 (fp16) or 2 (bf16)");
        if ((int64_t)a->H[0] + a->H[1] > 65535) return fail(ctx, INTATTN_ERR_UNSUPPORTED, "more than 65535 heads");
        if ((int64_t)a->B * a->L > MOST_TOKENS) return fail(ctx, INTATTN_ERR_UNSUPPORTED, "B * L must not exceed 2^24-1");
        RopeParams p;
        std::memset(&p, 0, sizeof(p));
        rc = check_rotary(ctx, a->rotary, a->d, false, &p.r);
        if (rc) return rc;
        const int64_t row = (int64_t)a->d * (a->dtype == 0 ? 4 : 2);
        for (int i = 0; i < (a->H[1] > 0 ? 2 : 1); ++i) {
            if (!a->src[i] || !a->dst[i]) return fail(ctx, INTATTN_ERR_INVALID_ARG, "src and dst must be non-NULL");
            if (!aligned(a->src[i], 16) || !aligned(a->dst[i], 16) || !strides_ok(a->src_stride[i], 3, 16) || !strides_ok(a->dst_stride[i], 3, 16))
                return fail(ctx, INTATTN_ERR_INVALID_ARG, "src, dst and their strides must be multiples of 16");
            if (!apart(a->dst_stride[i], a->B, a->H[i], a->L, row)) return fail(ctx, INTATTN_ERR_INVALID_ARG, "the strides of dst must cover a row");
            if (a->src[i] == a->dst[i])
                for (int s = 0; s < 3; ++s)
                    if (a->src_stride[i][s] != a->dst_stride[i][s]) return fail(ctx, INTATTN_ERR_INVALID_ARG, "dst is src with other strides");
            p.src[i] = (const uint8_t *)a->src[i];
            p.dst[i] = (uint8_t *)a->dst[i];
            for (int s = 0; s < 3; ++s) { p.ss[i][s] = a->src_stride[i][s]; p.ds[i][s] = a->dst_stride[i][s]; }
        }
        p.H0 = a->H[0]; p.H = a->H[0] + a->H[1];
        p.B = a->B; p.L = a->L; p.d = a->d;
        rc = check_device(ctx);
        if (rc) return rc;
        DeviceGuard guard(ctx->device);
        if (guard.status != hipSuccess) return hip_fail(ctx, guard.status, "hipSetDevice");
        const int herr = launch_rope(p, a->dtype, hip_stream);
        if (herr != 0) return hip_fail(ctx, (hipError_t)herr, "launch(rope)");
        ctx->err.clear();
        return INTATTN_OK;
    });
}

int intattn_cache_append(intattn_ctx *ctx, const intattn_cache *cache, const intattn_append_args *a, void *hip_stream)
{
    return guarded(ctx, [&]() -> int {
        int rc = check_ctx(ctx, a);
        if (rc) return rc;
        AppendParams p;
        std::memset(&p, 0, sizeof(p));
        rc = check_cache(ctx, cache, &p.c);
        if (rc) return rc;
        if (a->L < 1 || a->Hq < 0) return fail(ctx, INTATTN_ERR_INVALID_ARG, "L must be >= 1 and Hq >= 0");
        if (a->L > MOST_KEYS) return fail(ctx, INTATTN_ERR_UNSUPPORTED, "L must not exceed 131071");
        if (a->Hq % cache->Hkv != 0) return fail(ctx, INTATTN_ERR_INVALID_ARG, "Hq must be a multiple of Hkv");
        if ((int64_t)a->Hq + 2 * (int64_t)cache->Hkv > 2048) return fail(ctx, INTATTN_ERR_UNSUPPORTED, "Hq + 2 Hkv must not exceed 2048");
        if ((int64_t)cache->B * a->L > MOST_TOKENS) return fail(ctx, INTATTN_ERR_UNSUPPORTED, "B * L must not exceed 2^24-1");
        if (a->dtype < 0 || a->dtype > 2) return fail(ctx, INTATTN_ERR_INVALID_ARG, "dtype must be 0 (fp32), 1 (fp16) or 2 (bf16)");
        if (a->reserved != 0) return fail(ctx, INTATTN_ERR_INVALID_ARG, "reserved must be 0");
        if (!a->k || !a->v) return fail(ctx, INTATTN_ERR_INVALID_ARG, "k and v must be non-NULL");
        if (a->Hq > 0 && (!a->q || !a->q_out || !a->q_scale)) return fail(ctx, INTATTN_ERR_INVALID_ARG, "q, q_out and q_scale must be non-NULL");
        if (a->rotary.rot != 0 && a->rotary.inverse != 0) return fail(ctx, INTATTN_ERR_INVALID_ARG, "an append does not rotate backwards");
        rc = check_rotary(ctx, a->rotary, cache->d, true, &p.r);
        if (rc) return rc;
        if (!aligned(a->k, 16) || !aligned(a->v, 16) || !strides_ok(a->k_stride, 3, 16) || !strides_ok(a->v_stride, 3, 16))
            return fail(ctx, INTATTN_ERR_INVALID_ARG, "k, v and their strides must be multiples of 16");
        if (a->Hq > 0 && (!aligned(a->q, 16) || !aligned(a->q_out, 16) || !strides_ok(a->q_stride, 3, 16) || !strides_ok(a->q_out_stride, 3, 16)))
            return fail(ctx, INTATTN_ERR_INVALID_ARG, "q, q_out and their strides must be multiples of 16");
        if (a->Hq > 0 && !apart(a->q_out_stride, cache->B, a->Hq, a->L, cache->d)) return fail(ctx, INTATTN_ERR_INVALID_ARG, "the strides of q_out must cover a row");
        if (!writable(cache)) return fail(ctx, INTATTN_ERR_INVALID_ARG, "pages and heads of a cache that is written to must not lie over each other");
        if (!aligned(a->q_scale, 4) || !aligned(a->n_new, 4) || !aligned(a->weight, 4) || !aligned(a->order, 4) || !aligned(a->first, 4))
            return fail(ctx, INTATTN_ERR_INVALID_ARG, "q_scale, n_new, weight, order and first must be 4-byte aligned");
        if ((a->weight && !strides_ok(a->weight_stride, 2, 1)) || (a->order && !strides_ok(a->order_stride, 2, 1)))
            return fail(ctx, INTATTN_ERR_INVALID_ARG, "strides of weights and orders must be >= 0");
        if ((a->weight && !apart(a->weight_stride, cache->B, cache->Hkv)) || (a->order && !apart(a->order_stride, cache->B, cache->Hkv)))
            return fail(ctx, INTATTN_ERR_INVALID_ARG, "planes that are written must not lie over each other");
        const void *x[3] = {a->q, a->k, a->v};
        const int64_t *xs[3] = {a->q_stride, a->k_stride, a->v_stride};
        for (int i = 0; i < 3; ++i) {
            p.x[i] = (const uint8_t *)x[i];
            for (int s = 0; s < 3; ++s) p.xs[i][s] = xs[i][s];
        }
        p.Hq = a->Hq; p.L = a->L; p.n_new = a->n_new;
        p.q_out = a->q_out; p.q_scale = a->q_scale;
        for (int s = 0; s < 3; ++s) p.qos[s] = a->q_out_stride[s];
        p.weight = a->weight; p.order = a->order; p.first = a->first;
        for (int s = 0; s < 2; ++s) { p.wst[s] = a->weight_stride[s]; p.ost[s] = a->order_stride[s]; }
        rc = check_device(ctx);
        if (rc) return rc;
        DeviceGuard guard(ctx->device);
        if (guard.status != hipSuccess) return hip_fail(ctx, guard.status, "hipSetDevice");
        const int herr = launch_append(p, cache->d, a->dtype, hip_stream);
        if (herr != 0) return hip_fail(ctx, (hipError_t)herr, "launch(append)");
        ctx->err.clear();
        return INTATTN_OK;
    });
}

int intattn_cache_forward(intattn_ctx *ctx, const intattn_cache *cache, const intattn_cache_forward_args *a, void *hip_stream)
{
    return guarded(ctx, [&]() -> int {
        int rc = check_ctx(ctx, a);
        if (rc) return rc;
        AttendParams p;
        rc = forward_params(ctx, cache, a, &p);
        if (rc) return rc;
        rc = check_device(ctx);
        if (rc) return rc;
        DeviceGuard guard(ctx->device);
        if (guard.status != hipSuccess) return hip_fail(ctx, guard.status, "hipSetDevice");
        void *m = nullptr;
        rc = room(ctx, attend_room(p, cache->d), hip_stream, true, &m);
        if (rc) return rc;
        const int herr = launch_attend(p, cache->d, m, hip_stream);
        if (herr != 0) return hip_fail(ctx, (hipError_t)herr, "launch(attention over the cache)");
        ctx->err.clear();
        return INTATTN_OK;
    });
}

int intattn_cache_evict(intattn_ctx *ctx, const intattn_cache *cache, const intattn_evict_args *a, void *hip_stream)
{
    return guarded(ctx, [&]() -> int {
        int rc = check_ctx(ctx, a);
        if (rc) return rc;
        EvictParams p;
        rc = evict_params(ctx, cache, a, &p);
        if (rc) return rc;
        rc = check_device(ctx);
        if (rc) return rc;
        DeviceGuard guard(ctx->device);
        if (guard.status != hipSuccess) return hip_fail(ctx, guard.status, "hipSetDevice");
        void *m = nullptr;
        rc = room(ctx, evict_room(p), hip_stream, true, &m);
        if (rc) return rc;
        const int herr = launch_evict(p, m, hip_stream);
        if (herr != 0) return hip_fail(ctx, (hipError_t)herr, "launch(eviction)");
        ctx->err.clear();
        return INTATTN_OK;
    });
}

int intattn_cache_reserve(intattn_ctx *ctx, const intattn_cache *cache, int32_t rows, int32_t keep, int32_t max_len)
{
    return guarded(ctx, [&]() -> int {
        int rc = check_ctx(ctx, cache);
        if (rc) return rc;
        CacheParams c;
        rc = check_cache(ctx, cache, &c);
        if (rc) return rc;
        rc = bound_len(ctx, max_len, &c);
        if (rc) return rc;
        if (rows < 0 || rows > 4096 || keep < 0) return fail(ctx, INTATTN_ERR_INVALID_ARG, "rows must be in 0..4096, keep >= 0");
        int64_t bytes = 0;
        if (rows > 0) {
            AttendParams p;
            std::memset(&p, 0, sizeof(p));
            p.c = c;
            p.rows = rows;
            p.blocks = (rows + 15) / 16;
            bytes = std::max(bytes, attend_room_upto(p, cache->d));
        }
        if (keep > 0) {
            EvictParams p;
            std::memset(&p, 0, sizeof(p));
            p.c = c;
            p.keep = keep;
            bytes = std::max(bytes, evict_room(p));
        }
        rc = check_device(ctx);
        if (rc) return rc;
        DeviceGuard guard(ctx->device);
        if (guard.status != hipSuccess) return hip_fail(ctx, guard.status, "hipSetDevice");
        void *m = nullptr;
        rc = room(ctx, bytes, nullptr, false, &m);
        if (rc) return rc;
        ctx->err.clear();
        return INTATTN_OK;
    });
}

} // extern "C"
