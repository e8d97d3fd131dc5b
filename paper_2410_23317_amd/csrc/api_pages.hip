// C-ABI entry points of the paged prompt cache: argument validation, bookkeeping, kernel sequencing.
#include <string.h>

#include <new>

#include "internal.h"

namespace {

using vlc::fail;
using vlc::hip_fail;

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

vlc_status check_pages_shape(const vlc_pages_shape* s) {
    if (!s) return fail(VLC_ERR_INVALID_ARG, "pages shape is NULL");
    if (s->dtype != VLC_F32 && s->dtype != VLC_BF16) return fail(VLC_ERR_DTYPE, "dtype %d is neither VLC_F32 nor VLC_BF16", s->dtype);
    if (s->format != VLC_PAGES_PLAIN && s->format != VLC_PAGES_FP8 && s->format != VLC_PAGES_INT8)
        return fail(VLC_ERR_INVALID_ARG, "format %d is not a vlc_pages_format", s->format);
    if (s->format != VLC_PAGES_PLAIN && s->dtype != VLC_BF16) return fail(VLC_ERR_DTYPE, "quantised pages need bf16 storage of Q, K and V");
    if (s->L < 1 || s->Hq < 1 || s->Hkv < 1 || s->n_pages < 1) return fail(VLC_ERR_SHAPE, "L, Hq, Hkv, n_pages must be positive");
    if (s->d != 64 && s->d != 128) return fail(VLC_ERR_SHAPE, "d = %d: only 64 and 128 are built", s->d);
    if (s->Hq % s->Hkv != 0) return fail(VLC_ERR_SHAPE, "Hq = %d is not a multiple of Hkv = %d", s->Hq, s->Hkv);
    if (s->Hq / s->Hkv > 8) return fail(VLC_ERR_SHAPE, "g = Hq/Hkv = %d: at most 8 query heads per KV head", s->Hq / s->Hkv);
    if (s->L > vlc::kMaxLayers) return fail(VLC_ERR_SHAPE, "L = %d exceeds %d", s->L, vlc::kMaxLayers);
    if (s->Hkv > 65535) return fail(VLC_ERR_SHAPE, "Hkv = %d exceeds 65535", s->Hkv);
    const int ps = s->page_slots;
    if (ps != 16 && ps != 32 && ps != 64 && ps != 128 && ps != 256)
        return fail(VLC_ERR_SHAPE, "page_slots = %d is not one of 16, 32, 64, 128, 256", ps);
    if ((int64_t)s->n_pages * ps > (int64_t)1 << 30) return fail(VLC_ERR_SHAPE, "n_pages * page_slots = %lld exceeds 2^30", (long long)s->n_pages * ps);
    if ((double)s->n_pages * ps * s->d * s->Hkv * s->L > 4.0e12) return fail(VLC_ERR_SHAPE, "K pool larger than 4e12 elements");
    for (int32_t r : s->reserved)
        if (r != 0) return fail(VLC_ERR_INVALID_ARG, "pages shape: reserved fields must be 0");
    return VLC_OK;
}

void pages_layout(const vlc_pages_shape& s, vlc_pages_layout* lay) {
    const size_t rows = (size_t)s.L * s.n_pages * s.Hkv * s.page_slots;
    const bool codes = s.format != VLC_PAGES_PLAIN;
    const size_t es = codes ? 1 : (s.dtype == VLC_F32 ? 4 : 2);
    size_t off = 0;
    lay->status_off = off;     off = align_up(off + 4 * sizeof(int32_t), 256);
    lay->counters_off = off;   off = align_up(off + vlc::kMaxPagesRows * sizeof(int32_t), 256);
    lay->k_off = off;          off = align_up(off + rows * s.d * es, 256);
    lay->v_off = off;          off = align_up(off + rows * s.d * es, 256);
    lay->k_scale_off = off;
    if (codes) off = align_up(off + rows * sizeof(float), 256);
    lay->v_scale_off = off;
    if (codes) off = align_up(off + rows * sizeof(float), 256);
    lay->total_bytes = off;
}

vlc_status check_call(const char* who, const vlc_pages* pages, const vlc_chunk* c, int64_t n_layers) {
    if (!pages) return fail(VLC_ERR_INVALID_ARG, "%s: pages is NULL", who);
    if (!c) return fail(VLC_ERR_INVALID_ARG, "%s: chunk is NULL", who);
    const vlc_pages_shape& s = pages->shape;
    if (!c->table) return fail(VLC_ERR_INVALID_ARG, "%s: chunk->table is NULL", who);
    if (((uintptr_t)c->table & 3) != 0 || ((uintptr_t)c->lens & 3) != 0)
        return fail(VLC_ERR_INVALID_ARG, "%s: chunk->table and chunk->lens must be 4-byte aligned", who);
    if (c->reserved[0] != 0 || c->reserved[1] != 0) return fail(VLC_ERR_INVALID_ARG, "%s: chunk's reserved fields must be 0", who);
    if (c->B < 1 || c->max_pages < 1) return fail(VLC_ERR_SHAPE, "%s: B and max_pages must be positive", who);
    if ((int64_t)c->B * n_layers * s.Hkv > 65535)
        return fail(VLC_ERR_SHAPE, "%s: B * layers * Hkv = %lld exceeds 65535", who, (long long)c->B * n_layers * s.Hkv);
    if (c->max_new < 1 || c->max_new > c->max_len || c->max_len > (int64_t)c->max_pages * s.page_slots || c->max_len > 1 << 25)
        return fail(VLC_ERR_SHAPE, "%s: 1 <= max_new = %d <= max_len = %d <= max_pages * page_slots = %lld (and 2^25) does not hold", who,
                    c->max_new, c->max_len, (long long)c->max_pages * s.page_slots);
    if ((int64_t)c->B * n_layers * s.Hkv * (c->max_len / 1024 + 1) > 1 << 23)
        return fail(VLC_ERR_SHAPE, "%s: B * layers * Hkv * (max_len / 1024 + 1) exceeds 2^23", who);
    return VLC_OK;
}

// What an attention call takes of query rows: with it and the limit above, its grids have fewer than 2^24 blocks.
vlc_status check_queries(const char* who, const vlc_pages* pages, const vlc_chunk* c, int64_t n_layers) {
    const vlc_pages_shape& s = pages->shape;
    if ((int64_t)c->B * n_layers * s.Hq * c->max_new > (int64_t)1 << 30) return fail(VLC_ERR_SHAPE, "%s: B * layers * Hq * max_new exceeds 2^30", who);
    if ((int64_t)c->max_new * s.Hq > 1 << 26) return fail(VLC_ERR_SHAPE, "%s: max_new * Hq = %lld exceeds 2^26", who, (long long)c->max_new * s.Hq);
    return VLC_OK;
}

// Rows that a launch of the writer or the reader moves per (layer, request): at most 2^23 blocks along x.
vlc_status check_moved(const char* who, const vlc_pages* pages, const char* name, int rows) {
    const int64_t n = (int64_t)rows * pages->shape.Hkv;
    if (n > 1 << 26) return fail(VLC_ERR_SHAPE, "%s: %s * Hkv = %lld exceeds 2^26", who, name, (long long)n);
    return VLC_OK;
}

vlc_status check_layers(const char* who, const vlc_pages* pages, int lb, int le) {
    if (!pages) return fail(VLC_ERR_INVALID_ARG, "%s: pages is NULL", who);
    if (lb < 0 || le > pages->shape.L || lb >= le)
        return fail(VLC_ERR_INVALID_ARG, "%s: layer range [%d, %d) is outside [0, %d)", who, lb, le, pages->shape.L);
    return VLC_OK;
}

// extent: how many of each stride the call takes; a written tensor may not fold a dimension of more than one onto itself
vlc_status check_rows(const char* who, const char* name, const vlc_rows* r, int dtype, bool written, int64_t layers, int64_t reqs, int64_t heads, int64_t rows) {
    if (!r || !r->data) return fail(VLC_ERR_INVALID_ARG, "%s: %s must not be NULL", who, name);
    if (((uintptr_t)r->data & 15) != 0) return fail(VLC_ERR_INVALID_ARG, "%s: %s must be 16-byte aligned", who, name);
    const int64_t piece = dtype == VLC_F32 ? 4 : 8;
    const int64_t stride[4] = {r->layer, r->request, r->head, r->row}, extent[4] = {layers, reqs, heads, rows};
    for (int x = 0; x < 4; ++x) {
        if (extent[x] <= 1) continue;
        if (stride[x] < 0 || stride[x] % piece != 0 || stride[x] > (int64_t)1 << 42)
            return fail(VLC_ERR_INVALID_ARG, "%s: stride %lld of %s is negative, too large or no multiple of 16 bytes", who, (long long)stride[x], name);
        if (written && stride[x] == 0) return fail(VLC_ERR_INVALID_ARG, "%s: a stride of 0 in %s, which is written", who, name);
    }
    return VLC_OK;
}

vlc_status check_cleared(const char* who, const vlc_pages* pages) {
    if (!pages->cleared) return fail(VLC_ERR_INVALID_ARG, "%s: vlc_pages_clear has not been called on these pages", who);
    return VLC_OK;
}

vlc::PagesCall pages_call(const vlc_pages* pages, const vlc_chunk* c, int lb, int le, vlc_stream st) {
    vlc::PagesCall a;
    a.s = pages->shape; a.dev = pages->dev; a.chunk = *c;
    a.layer_begin = lb; a.n_layers = le - lb; a.stream = (hipStream_t)st;
    return a;
}

}  // namespace

extern "C" {

size_t vlc_pages_bytes(const vlc_pages_shape* shape) {
    if (check_pages_shape(shape) != VLC_OK) return 0;
    vlc_pages_layout lay;
    pages_layout(*shape, &lay);
    return lay.total_bytes;
}

vlc_status vlc_pages_create(const vlc_pages_shape* shape, void* arena, size_t arena_bytes, vlc_pages** out) {
    if (!out) return fail(VLC_ERR_INVALID_ARG, "vlc_pages_create: out is NULL");
    *out = nullptr;
    if (vlc_status st = check_pages_shape(shape)) return st;
    if (!arena) return fail(VLC_ERR_INVALID_ARG, "vlc_pages_create: arena is NULL");
    if (((uintptr_t)arena & 255) != 0) return fail(VLC_ERR_INVALID_ARG, "vlc_pages_create: arena must be 256-byte aligned");
    vlc_pages_layout lay;
    pages_layout(*shape, &lay);
    if (arena_bytes < lay.total_bytes)
        return fail(VLC_ERR_CAPACITY, "vlc_pages_create: arena of %zu bytes, %zu needed", arena_bytes, lay.total_bytes);
    vlc_pages* p = new (std::nothrow) vlc_pages;
    if (!p) return fail(VLC_ERR_INVALID_ARG, "vlc_pages_create: out of host memory");
    char* base = (char*)arena;
    p->shape = *shape;
    p->layout = lay;
    p->dev.status = (int32_t*)(base + lay.status_off);
    p->dev.counters = (int32_t*)(base + lay.counters_off);
    p->dev.k = base + lay.k_off;
    p->dev.v = base + lay.v_off;
    p->dev.k_scale = (float*)(base + lay.k_scale_off);
    p->dev.v_scale = (float*)(base + lay.v_scale_off);
    p->cleared = false;
    *out = p;
    return VLC_OK;
}

void vlc_pages_destroy(vlc_pages* pages) { delete pages; }

vlc_status vlc_pages_get_layout(const vlc_pages* pages, vlc_pages_layout* out) {
    if (!pages || !out) return fail(VLC_ERR_INVALID_ARG, "vlc_pages_get_layout: NULL argument");
    *out = pages->layout;
    return VLC_OK;
}

vlc_status vlc_pages_clear(vlc_pages* pages, vlc_stream stream) {
    if (!pages) return fail(VLC_ERR_INVALID_ARG, "vlc_pages_clear: pages is NULL");
    const hipError_t e = vlc::launch_pages_clear(pages->dev, (hipStream_t)stream);
    if (e != hipSuccess) return hip_fail(e, "vlc_pages_clear");
    pages->cleared = true;
    return VLC_OK;
}

vlc_status vlc_pages_status(vlc_pages* pages, vlc_stream stream) {
    if (!pages) return fail(VLC_ERR_INVALID_ARG, "vlc_pages_status: pages is NULL");
    if (vlc_status st = check_cleared("vlc_pages_status", pages)) return st;
    int32_t st[4] = {0, 0, 0, 0};
    hipError_t e = hipMemcpyAsync(st, pages->dev.status, sizeof(st), hipMemcpyDeviceToHost, (hipStream_t)stream);
    if (e == hipSuccess) e = hipStreamSynchronize((hipStream_t)stream);
    if (e != hipSuccess) return hip_fail(e, "vlc_pages_status");
    if (st[0] == VLC_OK) return VLC_OK;
    if (st[2] == -2)
        return fail(VLC_ERR_INVALID_ARG, "request %d: lengths (n_b = %d) break 0 <= c_b <= max_new, c_b <= n_b <= max_len", st[1], st[3]);
    return fail((vlc_status)st[0], "request %d: page %d of its table is outside [0, %d)", st[1], st[3], pages->shape.n_pages);
}

vlc_status vlc_pages_write(vlc_pages* pages, const vlc_chunk* chunk, int32_t layer_begin, int32_t layer_end,
                           const vlc_rows* k_new, const vlc_rows* v_new, vlc_stream stream) {
    static const char who[] = "vlc_pages_write";
    if (vlc_status st = check_layers(who, pages, layer_begin, layer_end)) return st;
    const int64_t nl = layer_end - layer_begin;
    if (vlc_status st = check_call(who, pages, chunk, nl)) return st;
    if (vlc_status st = check_moved(who, pages, "max_new", chunk->max_new)) return st;
    const vlc_pages_shape& s = pages->shape;
    if (vlc_status st = check_rows(who, "k_new", k_new, s.dtype, false, nl, chunk->B, s.Hkv, chunk->max_new)) return st;
    if (vlc_status st = check_rows(who, "v_new", v_new, s.dtype, false, nl, chunk->B, s.Hkv, chunk->max_new)) return st;
    if (vlc_status st = check_cleared(who, pages)) return st;
    const hipError_t e = vlc::launch_pages_write(pages_call(pages, chunk, layer_begin, layer_end, stream), *k_new, *v_new);
    if (e != hipSuccess) return hip_fail(e, who);
    return VLC_OK;
}

vlc_status vlc_pages_read(vlc_pages* pages, const vlc_chunk* chunk, int32_t layer_begin, int32_t layer_end, int32_t first,
                          int32_t count, const vlc_rows* k_out, const vlc_rows* v_out, vlc_stream stream) {
    static const char who[] = "vlc_pages_read";
    if (vlc_status st = check_layers(who, pages, layer_begin, layer_end)) return st;
    const int64_t nl = layer_end - layer_begin;
    if (vlc_status st = check_call(who, pages, chunk, nl)) return st;
    if (first < 0 || count < 1) return fail(VLC_ERR_INVALID_ARG, "%s: first = %d, count = %d", who, first, count);
    const vlc_pages_shape& s = pages->shape;
    if (vlc_status st = check_rows(who, "k_out", k_out, s.dtype, true, nl, chunk->B, s.Hkv, count)) return st;
    if (vlc_status st = check_rows(who, "v_out", v_out, s.dtype, true, nl, chunk->B, s.Hkv, count)) return st;
    if (first >= chunk->max_len) return VLC_OK;               // no request holds such a position
    if (count > chunk->max_len - first) count = chunk->max_len - first;
    if (vlc_status st = check_moved(who, pages, "count", count)) return st;
    if (vlc_status st = check_cleared(who, pages)) return st;
    const hipError_t e = vlc::launch_pages_read(pages_call(pages, chunk, layer_begin, layer_end, stream), first, count, *k_out, *v_out);
    if (e != hipSuccess) return hip_fail(e, who);
    return VLC_OK;
}

vlc_status vlc_pages_attn_workspace_bytes(const vlc_pages* pages, const vlc_chunk* chunk, int32_t n_layers, size_t* bytes_out) {
    static const char who[] = "vlc_pages_attn_workspace_bytes";
    if (!bytes_out) return fail(VLC_ERR_INVALID_ARG, "%s: bytes_out is NULL", who);
    *bytes_out = 0;
    if (vlc_status st = check_layers(who, pages, 0, n_layers)) return st;
    if (vlc_status st = check_call(who, pages, chunk, n_layers)) return st;
    if (vlc_status st = check_queries(who, pages, chunk, n_layers)) return st;
    const vlc::PagesCall c = pages_call(pages, chunk, 0, n_layers, nullptr);
    *bytes_out = vlc::pages_few_supported(c) ? vlc::pages_few_workspace_bytes(c)
                 : c.s.dtype == VLC_F32        ? vlc::pages_rows_f32_workspace_bytes(c)
                                               : vlc::pages_rows_workspace_bytes(c);
    return VLC_OK;
}

vlc_status vlc_pages_attn(vlc_pages* pages, const vlc_chunk* chunk, int32_t layer_begin, int32_t layer_end, const vlc_rows* q,
                          const vlc_rows* k_new, const vlc_rows* v_new, const float* sm_scale, const vlc_rows* out,
                          const vlc_row_stats* stats, void* workspace, size_t workspace_bytes, vlc_stream stream) {
    static const char who[] = "vlc_pages_attn";
    if (vlc_status st = check_layers(who, pages, layer_begin, layer_end)) return st;
    const int64_t nl = layer_end - layer_begin;
    if (vlc_status st = check_call(who, pages, chunk, nl)) return st;
    if (vlc_status st = check_queries(who, pages, chunk, nl)) return st;
    const vlc_pages_shape& s = pages->shape;
    if (vlc_status st = check_rows(who, "q", q, s.dtype, false, nl, chunk->B, s.Hq, chunk->max_new)) return st;
    if (vlc_status st = check_rows(who, "out", out, s.dtype, true, nl, chunk->B, s.Hq, chunk->max_new)) return st;
    if ((k_new == nullptr) != (v_new == nullptr))
        return fail(VLC_ERR_INVALID_ARG, "%s: k_new and v_new must both be given or both be NULL", who);
    if (k_new) {
        if (vlc_status st = check_rows(who, "k_new", k_new, s.dtype, false, nl, chunk->B, s.Hkv, chunk->max_new)) return st;
        if (vlc_status st = check_rows(who, "v_new", v_new, s.dtype, false, nl, chunk->B, s.Hkv, chunk->max_new)) return st;
    }
    if (((uintptr_t)sm_scale & 3) != 0) return fail(VLC_ERR_INVALID_ARG, "%s: sm_scale must be 4-byte aligned", who);
    if (stats) {
        if ((((uintptr_t)stats->row_max | (uintptr_t)stats->row_sum) & 3) != 0) return fail(VLC_ERR_INVALID_ARG, "%s: row_max and row_sum must be 4-byte aligned", who);
        if (!stats->row_max || !stats->row_sum) return fail(VLC_ERR_INVALID_ARG, "%s: stats without row_max or row_sum", who);
        const int64_t stride[3] = {stats->layer, stats->request, stats->head}, extent[3] = {nl, chunk->B, s.Hq};
        for (int x = 0; x < 3; ++x)
            if (extent[x] > 1 && (stride[x] < chunk->max_new || stride[x] > (int64_t)1 << 42))
                return fail(VLC_ERR_INVALID_ARG, "%s: stride %lld of stats is below max_new = %d or too large", who, (long long)stride[x], chunk->max_new);
    }
    size_t need = 0;
    if (vlc_status st = vlc_pages_attn_workspace_bytes(pages, chunk, (int32_t)nl, &need)) return st;
    if (need && !workspace) return fail(VLC_ERR_INVALID_ARG, "%s: workspace must not be NULL for this call", who);
    if (workspace_bytes < need) return fail(VLC_ERR_CAPACITY, "%s: workspace of %zu bytes, %zu needed", who, workspace_bytes, need);
    if (need && ((uintptr_t)workspace & 15) != 0) return fail(VLC_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", who);
    if (vlc_status st = check_cleared(who, pages)) return st;
    vlc::PagesAttn a;
    a.c = pages_call(pages, chunk, layer_begin, layer_end, stream);
    a.q = *q; a.out = *out; a.sm_scale = sm_scale; a.workspace = workspace;
    memset(&a.stats, 0, sizeof(a.stats));
    if (stats) a.stats = *stats;
    memset(&a.k_new, 0, sizeof(a.k_new));
    a.v_new = a.k_new;
    if (k_new) { a.k_new = *k_new; a.v_new = *v_new; }
    if (vlc::pages_few_supported(a.c)) {
        const hipError_t e = vlc::launch_pages_few(a);
        if (e != hipSuccess) return hip_fail(e, who);
        return VLC_OK;
    }
    if (k_new) {
        const hipError_t e = vlc::launch_pages_write(a.c, *k_new, *v_new);
        if (e != hipSuccess) return hip_fail(e, who);
    }
    const hipError_t e = a.c.s.dtype == VLC_F32 ? vlc::launch_pages_rows_f32(a) : vlc::launch_pages_rows(a);
    if (e != hipSuccess) return hip_fail(e, who);
    return VLC_OK;
}

}  // extern "C"
