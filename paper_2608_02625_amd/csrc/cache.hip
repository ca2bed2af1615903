// C entry points of the rotary positions, the paged cache and the verification of
// drafted tokens (see include/dlm.h): argument checks, sizes, launches.
#include <math.h>

#include <algorithm>
#include <string>

#include "cache.h"
#include "status.h"
#include "verify.h"

namespace {

dlm_status fail(dlm_status s, const std::string& msg) { return dlm_internal_fail(s, msg); }

dlm_status launched(hipError_t e, const char* what) {
    if (e == hipSuccess) return DLM_OK;
    return fail(e == hipErrorInvalidValue ? DLM_ERR_INVALID_ARG : DLM_ERR_HIP,
                std::string(what) + ": " + hipGetErrorString(e));
}

bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }
int64_t capacity(const dlm_cache& c) { return (int64_t)c.max_pages * c.page_len; }

// Shape of a cache; "" if it is sound.
std::string check_shape(const dlm_cache* c) {
    if (!c) return "cache is NULL";
    if (c->dtype != DLM_BF16 && c->dtype != DLM_F16) return "the cache's dtype must be DLM_BF16 or DLM_F16";
    if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
    if (c->page_len != 16 && c->page_len != 32 && c->page_len != 64 && c->page_len != 128)
        return "page_len must be 16, 32, 64 or 128";
    if (c->n_layers < 1 || c->n_layers > 4096) return "n_layers must be in [1, 4096]";
    if (c->n_pages < 1 || c->n_pages > kCacheMaxPages) return "n_pages must be in [1, 2^20]";
    if (c->n_kv_heads < 1 || c->n_kv_heads > kCacheMaxKvHeads) return "n_kv_heads must be in [1, 128]";
    if (c->n_seqs < 1 || c->n_seqs > kCacheMaxSeqs) return "n_seqs must be in [1, 1024]";
    if (c->max_pages < 1 || capacity(*c) > (1 << 26)) return "max_pages * page_len must be in [1, 2^26]";
    return "";
}
dlm_status check_cache(const dlm_cache* c) {
    const std::string e = check_shape(c);
    if (!e.empty()) return fail(DLM_ERR_INVALID_ARG, e);
    if (!c->d_k || !c->d_v || !c->d_ref || !c->d_len || !c->d_table)
        return fail(DLM_ERR_INVALID_ARG, "a buffer of the cache is NULL");
    if (!aligned(c->d_k, 256) || !aligned(c->d_v, 256))
        return fail(DLM_ERR_INVALID_ARG, "d_k and d_v must be 256-byte aligned");
    if (!aligned(c->d_ref, 4) || !aligned(c->d_len, 4) || !aligned(c->d_table, 4))
        return fail(DLM_ERR_INVALID_ARG, "d_ref, d_len and d_table must be 4-byte aligned");
    return DLM_OK;
}
dlm_status check_workspace(const void* ws, size_t have, size_t need) {
    if (!ws) return fail(DLM_ERR_INVALID_ARG, "workspace is NULL");
    if (!aligned(ws, 256)) return fail(DLM_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (have < need)
        return fail(DLM_ERR_WORKSPACE, "workspace too small: need " + std::to_string(need) + " bytes, got " +
                                           std::to_string(have));
    return DLM_OK;
}
dlm_status check_rows(const int32_t* row_start, int total_rows, int max_rows) {
    if (!row_start) return fail(DLM_ERR_INVALID_ARG, "row_start is NULL");
    if (total_rows < 0 || max_rows < 0) return fail(DLM_ERR_INVALID_ARG, "total_rows and max_rows must be >= 0");
    if (total_rows > 0 && max_rows == 0) return fail(DLM_ERR_INVALID_ARG, "max_rows is 0 but there are rows");
    if (total_rows > (1 << 24)) return fail(DLM_ERR_INVALID_ARG, "total_rows must be at most 2^24");
    return DLM_OK;
}
dlm_status check_rope(const dlm_rope* r) {
    if (r->head_dim < 2 || r->head_dim > 2 * DLM_ROPE_MAX_PAIRS || r->rot_dim < 2 || r->rot_dim > r->head_dim ||
        r->rot_dim % 2 || !(r->scale > 0.f) || !isfinite(r->scale))
        return fail(DLM_ERR_INVALID_ARG, "rope was not filled by dlm_rope_init");
    return DLM_OK;
}
#define TRY(expr)                        \
    do {                                 \
        dlm_status _s = (expr);          \
        if (_s != DLM_OK) return _s;     \
    } while (0)

// Results must not overlap: heads inside a row, or rows inside a head.
bool overlaps(int64_t rows, int64_t heads, int64_t row_stride, int64_t head_stride, int64_t hd) {
    const int64_t h = heads > 1 ? head_stride : 0, r = rows > 1 ? row_stride : 0;
    const bool rows_outer = (rows == 1 || r >= (__int128)(heads - 1) * h + hd) && (heads == 1 || h >= hd);
    const bool heads_outer = (heads == 1 || h >= (__int128)(rows - 1) * r + hd) && (rows == 1 || r >= hd);
    return !rows_outer && !heads_outer;
}
bool same_layout(int64_t rows, int64_t heads, int64_t a_row, int64_t a_head, int64_t b_row, int64_t b_head) {
    return (rows <= 1 || a_row == b_row) && (heads <= 1 || a_head == b_head);
}

dlm_status check_eps(float eps) {
    if (!(eps > 0.f) || !std::isfinite(eps)) return fail(DLM_ERR_INVALID_ARG, "eps must be finite and > 0");
    return DLM_OK;
}
dlm_status check_gain(int dtype, int gain_dtype, const void* gain, const void* dgain) {
    if (gain_dtype != dtype && gain_dtype != DLM_F32)
        return fail(DLM_ERR_INVALID_ARG, "gain_dtype must be the rows' dtype or DLM_F32");
    const size_t size = gain_dtype == DLM_F32 ? 4 : 2;
    if (!aligned(gain, size) || !aligned(dgain, size)) return fail(DLM_ERR_INVALID_ARG, "gains must be aligned to their elements");
    return DLM_OK;
}
// A set of heads of dlm_rope_norm or, with `grad`, of its gradient.
dlm_status check_norm_set(const dlm_norm_heads* s, const dlm_norm_grads* g, bool grad, int dtype, int64_t rows, int64_t hd) {
    if (!s) return DLM_OK;
    if (s->n_heads == 0) return grad && g && g->d_dgain ? check_gain(dtype, s->gain_dtype, nullptr, g->d_dgain) : DLM_OK;
    if (s->n_heads < 0 || s->n_heads > (1 << 24)) return fail(DLM_ERR_INVALID_ARG, "n_heads must be in [0, 2^24]");
    if (grad && !g) return fail(DLM_ERR_INVALID_ARG, "a set of heads without its gradients");
    TRY(check_gain(dtype, s->gain_dtype, s->d_gain, grad ? g->d_dgain : nullptr));
    if (rows == 0) return DLM_OK;
    const size_t size = dtype == DLM_F32 ? 4 : 2;
    const int64_t n = s->n_heads;
    const void* out = grad ? g->d_dx : s->d_y;
    const int64_t out_row = grad ? g->dx_row_stride : s->y_row_stride, out_head = grad ? g->dx_head_stride : s->y_head_stride;
    if (!s->d_x || !out || (grad && !g->d_dy)) return fail(DLM_ERR_INVALID_ARG, grad ? "x, dy or dx is NULL" : "x or y is NULL");
    if (!aligned(s->d_x, size) || !aligned(out, size) || (grad && !aligned(g->d_dy, size)))
        return fail(DLM_ERR_INVALID_ARG, "rows must be aligned to their elements");
    if (s->x_row_stride < 0 || s->x_head_stride < 0 || out_row < 0 || out_head < 0 ||
        (grad && (g->dy_row_stride < 0 || g->dy_head_stride < 0)))
        return fail(DLM_ERR_INVALID_ARG, "strides must be >= 0");
    if (overlaps(rows, n, out_row, out_head, hd)) return fail(DLM_ERR_INVALID_ARG, "rows or heads of the result overlap");
    if ((s->d_x == out && !same_layout(rows, n, s->x_row_stride, s->x_head_stride, out_row, out_head)) ||
        (grad && g->d_dy == out && !same_layout(rows, n, g->dy_row_stride, g->dy_head_stride, out_row, out_head)))
        return fail(DLM_ERR_INVALID_ARG, "in place, rows and results must have the same strides");
    return DLM_OK;
}
dlm_status check_norm(const dlm_rope* rope, int dtype, int rows, float eps, const dlm_norm_heads* q, const dlm_norm_heads* k,
                      const int32_t* pos) {
    if (!rope) return fail(DLM_ERR_INVALID_ARG, "rope is NULL");
    TRY(check_rope(rope));
    if (dtype != DLM_BF16 && dtype != DLM_F16 && dtype != DLM_F32) return fail(DLM_ERR_INVALID_ARG, "unknown dtype");
    if (rows < 0) return fail(DLM_ERR_INVALID_ARG, "rows must be >= 0");
    TRY(check_eps(eps));
    if (!q) return fail(DLM_ERR_INVALID_ARG, "q is NULL");
    const bool any = q->n_heads != 0 || (k && k->n_heads != 0);
    if (rows > 0 && any && (!pos || !aligned(pos, 4))) return fail(DLM_ERR_INVALID_ARG, "pos must not be NULL and be 4-byte aligned");
    return DLM_OK;
}
bool norm_idle(int rows, const dlm_norm_heads* q, const dlm_norm_heads* k) {
    return rows == 0 || (q->n_heads == 0 && (!k || k->n_heads == 0));
}

// What the two forms of append ask for; *nothing: no rows.
dlm_status check_append(const dlm_cache* cache, int layer, const int32_t* d_row_start, int total_rows, int max_rows,
                        int src_dtype, const void* d_k, int64_t k_stride, const void* d_v, int64_t v_stride,
                        const dlm_rope* rope, int n_heads, const void* d_q, int64_t q_stride, const void* d_q_out,
                        int64_t q_out_stride, bool* nothing) {
    TRY(check_cache(cache));
    if (layer < 0 || layer >= cache->n_layers) return fail(DLM_ERR_INVALID_ARG, "layer out of range");
    TRY(check_rows(d_row_start, total_rows, max_rows));
    if (src_dtype != cache->dtype && src_dtype != DLM_F32)
        return fail(DLM_ERR_INVALID_ARG, "src_dtype must be the cache's dtype or DLM_F32");
    if (rope) {
        TRY(check_rope(rope));
        if (rope->head_dim != cache->head_dim) return fail(DLM_ERR_INVALID_ARG, "rope and cache differ in head_dim");
    }
    *nothing = total_rows == 0;
    if (*nothing) return DLM_OK;
    if (!d_k || !d_v) return fail(DLM_ERR_INVALID_ARG, "k or v is NULL");
    const int64_t kv_width = (int64_t)cache->n_kv_heads * cache->head_dim;
    if (k_stride < kv_width || v_stride < kv_width) return fail(DLM_ERR_INVALID_ARG, "k_stride or v_stride below a row");
    const size_t size = src_dtype == DLM_F32 ? 4 : 2;
    if (!aligned(d_k, size) || !aligned(d_v, size)) return fail(DLM_ERR_INVALID_ARG, "k and v must be aligned to their elements");
    if (d_q) {
        if (n_heads < 1 || n_heads > (1 << 16)) return fail(DLM_ERR_INVALID_ARG, "n_heads must be in [1, 65536]");
        if (!d_q_out) return fail(DLM_ERR_INVALID_ARG, "q_out is NULL");
        const int64_t width = (int64_t)n_heads * cache->head_dim;
        if (q_stride < width || q_out_stride < width) return fail(DLM_ERR_INVALID_ARG, "q_stride or q_out_stride below a row");
        if (!aligned(d_q, size) || !aligned(d_q_out, 2)) return fail(DLM_ERR_INVALID_ARG, "q and q_out must be aligned to their elements");
        if (d_q == d_q_out && (src_dtype != cache->dtype || q_stride != q_out_stride))
            return fail(DLM_ERR_INVALID_ARG, "in place, q and q_out must have the same type and stride");
    }
    if ((int64_t)cache->n_seqs * std::max(d_q ? n_heads : 0, cache->n_kv_heads) * std::min(max_rows, total_rows) > ((int64_t)1 << 33))
        return fail(DLM_ERR_INVALID_ARG, "n_seqs * n_heads * max_rows must be at most 2^33");
    return DLM_OK;
}

// What the two forms of attend ask for; *nothing: no rows.
dlm_status check_attend(const dlm_cache* cache, int layer, const int32_t* d_row_start, int total_rows, int max_rows,
                        int max_keys, int n_heads, const void* d_q, int64_t q_stride, const uint32_t* d_mask, int mask_words,
                        float scale, const void* d_o, int64_t o_stride, const float* d_lse, bool* nothing) {
    TRY(check_cache(cache));
    if (layer < 0 || layer >= cache->n_layers) return fail(DLM_ERR_INVALID_ARG, "layer out of range");
    TRY(check_rows(d_row_start, total_rows, max_rows));
    if (n_heads < 1 || n_heads % cache->n_kv_heads) return fail(DLM_ERR_INVALID_ARG, "n_heads must be a positive multiple of n_kv_heads");
    if (max_keys < 0) return fail(DLM_ERR_INVALID_ARG, "max_keys must be >= 0");
    if (!(scale >= 0.f) || !std::isfinite(scale)) return fail(DLM_ERR_INVALID_ARG, "scale must be finite and >= 0");
    *nothing = total_rows == 0;
    if (*nothing) return DLM_OK;
    if (!d_q || !d_o) return fail(DLM_ERR_INVALID_ARG, "q or o is NULL");
    const int rows = std::min(max_rows, total_rows);
    const int64_t width = (int64_t)n_heads * cache->head_dim;
    if (q_stride < width || o_stride < width) return fail(DLM_ERR_INVALID_ARG, "q_stride or o_stride below a row");
    if (!aligned(d_q, 16) || !aligned(d_o, 16) || q_stride % 8 || o_stride % 8)
        return fail(DLM_ERR_INVALID_ARG, "q and o must be 16-byte aligned, with strides that are multiples of 8");
    if (d_q == d_o && q_stride != o_stride) return fail(DLM_ERR_INVALID_ARG, "in place, q and o must have the same stride");
    if (d_mask && (!aligned(d_mask, 4) || (int64_t)mask_words * 32 < rows))
        return fail(DLM_ERR_INVALID_ARG, "mask must be 4-byte aligned and hold max_rows bits per row");
    if (d_lse && !aligned(d_lse, 4)) return fail(DLM_ERR_INVALID_ARG, "lse must be 4-byte aligned");
    const std::string bad = dlm_internal_check_windows(*cache, n_heads, rows);
    if (!bad.empty()) return fail(DLM_ERR_INVALID_ARG, bad);
    return DLM_OK;
}

dlm_status check_share(const dlm_cache& c, int total_rows, int max_group_rows, const void* share, size_t bytes) {
    if (max_group_rows < 0) return fail(DLM_ERR_INVALID_ARG, "max_group_rows must be >= 0");
    if (!share || !aligned(share, 256)) return fail(DLM_ERR_INVALID_ARG, "share must not be NULL and be 256-byte aligned");
    const size_t need = share_bytes(c.n_seqs, total_rows);
    if (bytes < need)
        return fail(DLM_ERR_WORKSPACE, "share too small: need " + std::to_string(need) + " bytes, got " + std::to_string(bytes));
    return DLM_OK;
}

std::string check_verify_sizes(int n_seqs, int total_rows, int vocab) {
    if (n_seqs < 1 || n_seqs > 65535) return "n_seqs must be in [1, 65535]";
    if (total_rows < 0 || total_rows > (1 << 20)) return "total_rows must be in [0, 2^20]";
    if (vocab < 1 || vocab > (1 << 24)) return "vocab must be in [1, 2^24]";
    if (verify_workgroups(total_rows, vocab) > kVerifyMaxWorkgroups) return "total_rows * (vocab / 8192 + 2) must be below 2^31";
    return "";
}

}  // namespace

dlm_status dlm_internal_check_cache(const dlm_cache* cache) { return check_cache(cache); }

std::string dlm_internal_check_windows(const dlm_cache& cache, int n_heads, int64_t rows) {
    if (rows * (n_heads / cache.n_kv_heads) > (1 << 28)) return "max_rows times query heads per key head too large";
    if (cache.n_seqs * (int64_t)std::max(n_heads, cache.n_kv_heads) * rows > ((int64_t)1 << 33))
        return "n_seqs * n_heads * max_rows must be at most 2^33";
    return "";
}

extern "C" {

dlm_status dlm_rope_init(const dlm_rope_spec* s, dlm_rope* out) {
    try {
        if (!s || !out) return fail(DLM_ERR_INVALID_ARG, "NULL argument");
        if (s->head_dim < 2 || s->head_dim > 2 * DLM_ROPE_MAX_PAIRS)
            return fail(DLM_ERR_INVALID_ARG, "head_dim must be in [2, 256]");
        if (s->rot_dim < 2 || s->rot_dim > s->head_dim || s->rot_dim % 2)
            return fail(DLM_ERR_INVALID_ARG, "rot_dim must be even and in [2, head_dim]");
        if (s->scaling < DLM_ROPE_PLAIN || s->scaling > DLM_ROPE_YARN) return fail(DLM_ERR_INVALID_ARG, "unknown scaling");
        if (!(s->theta > 0.) || !std::isfinite(s->theta)) return fail(DLM_ERR_INVALID_ARG, "theta must be finite and > 0");
        if (!(s->scale >= 0.f) || !std::isfinite(s->scale)) return fail(DLM_ERR_INVALID_ARG, "scale must be finite and >= 0");
        const bool scaled = s->scaling != DLM_ROPE_PLAIN;
        if (scaled && (!(s->factor >= 1.) || !std::isfinite(s->factor)))
            return fail(DLM_ERR_INVALID_ARG, "factor must be finite and >= 1");
        if (s->scaling == DLM_ROPE_NTK && s->rot_dim < 4) return fail(DLM_ERR_INVALID_ARG, "this scaling needs rot_dim >= 4");
        if (s->scaling == DLM_ROPE_YARN) {
            if (s->original_len <= 0) return fail(DLM_ERR_INVALID_ARG, "original_len must be > 0");
            if (!(s->beta_slow >= 0.) || !(s->beta_fast > s->beta_slow) || !std::isfinite(s->beta_fast))
                return fail(DLM_ERR_INVALID_ARG, "beta_slow and beta_fast must satisfy 0 <= beta_slow < beta_fast");
        }
        dlm_rope r{};
        r.head_dim = s->head_dim;
        r.rot_dim = s->rot_dim;
        r.interleaved = s->interleaved != 0;
        r.scale = s->scale > 0.f ? s->scale : s->scaling == DLM_ROPE_YARN ? (float)(0.1 * log(s->factor) + 1.) : 1.f;
        const long double two_pi = 6.283185307179586476925286766559005768L;
        long double theta = s->theta;
        const long double f = scaled ? (long double)s->factor : 1.0L;
        if (s->scaling == DLM_ROPE_NTK) theta *= powl(f, (long double)s->rot_dim / (s->rot_dim - 2));
        for (int i = 0; i < s->rot_dim / 2; ++i) {
            long double w = powl(theta, -2.0L * i / s->rot_dim);
            if (s->scaling == DLM_ROPE_LINEAR) w /= f;
            if (s->scaling == DLM_ROPE_YARN) {
                const long double turns = s->original_len * w / two_pi;
                long double g = (turns - s->beta_slow) / (s->beta_fast - s->beta_slow);
                g = std::min(1.0L, std::max(0.0L, g));
                w = g * w + (1.0L - g) * w / f;
            }
            long double part = w / two_pi;
            part -= floorl(part);
            r.phase[i] = part < 1.0L ? (uint64_t)ldexpl(part, 64) : 0;
        }
        *out = r;
        return DLM_OK;
    } catch (...) {
        return dlm_internal_caught();
    }
}

dlm_status dlm_rope_apply(const dlm_rope* rope, int32_t dtype, int32_t rows, int32_t heads, const void* d_x,
                          int64_t x_row_stride, int64_t x_head_stride, void* d_y, int64_t y_row_stride,
                          int64_t y_head_stride, const int32_t* d_pos, int32_t transpose, void* hip_stream) {
    try {
        if (!rope) return fail(DLM_ERR_INVALID_ARG, "rope is NULL");
        TRY(check_rope(rope));
        if (dtype != DLM_BF16 && dtype != DLM_F16 && dtype != DLM_F32) return fail(DLM_ERR_INVALID_ARG, "unknown dtype");
        if (rows < 0 || heads < 0) return fail(DLM_ERR_INVALID_ARG, "rows and heads must be >= 0");
        if (rows == 0 || heads == 0) return DLM_OK;
        if (!d_x || !d_y || !d_pos) return fail(DLM_ERR_INVALID_ARG, "x, y or pos is NULL");
        const size_t size = dtype == DLM_F32 ? 4 : 2;
        if (!aligned(d_x, size) || !aligned(d_y, size) || !aligned(d_pos, 4))
            return fail(DLM_ERR_INVALID_ARG, "x, y and pos must be aligned to their elements");
        if (x_row_stride < 0 || x_head_stride < 0 || y_row_stride < 0 || y_head_stride < 0)
            return fail(DLM_ERR_INVALID_ARG, "strides must be >= 0");
        if (overlaps(rows, heads, y_row_stride, y_head_stride, rope->head_dim))
            return fail(DLM_ERR_INVALID_ARG, "rows or heads of y overlap");
        if (d_x == d_y && !same_layout(rows, heads, x_row_stride, x_head_stride, y_row_stride, y_head_stride))
            return fail(DLM_ERR_INVALID_ARG, "in place, x and y must have the same strides");
        return launched(launch_rope(*rope, dtype, rows, heads, d_x, x_row_stride, x_head_stride, d_y, y_row_stride,
                                    y_head_stride, d_pos, transpose != 0, (hipStream_t)hip_stream), "rope");
    } catch (...) {
        return dlm_internal_caught();
    }
}

dlm_status dlm_rope_norm(const dlm_rope* rope, int32_t dtype, int32_t rows, const dlm_norm_heads* q,
                         const dlm_norm_heads* k, float eps, const int32_t* d_pos, void* hip_stream) {
    try {
        TRY(check_norm(rope, dtype, rows, eps, q, k, d_pos));
        TRY(check_norm_set(q, nullptr, false, dtype, rows, rope->head_dim));
        TRY(check_norm_set(k, nullptr, false, dtype, rows, rope->head_dim));
        if (norm_idle(rows, q, k)) return DLM_OK;
        if (k && q->n_heads && k->n_heads && q->d_y == k->d_y) return fail(DLM_ERR_INVALID_ARG, "the sets' results overlap");
        return launched(launch_rope_norm(*rope, dtype, rows, q, k, eps, d_pos, (hipStream_t)hip_stream), "rope_norm");
    } catch (...) {
        return dlm_internal_caught();
    }
}

size_t dlm_rope_norm_grad_workspace_bytes(const dlm_rope* rope) {
    try {
        if (!rope || check_rope(rope) != DLM_OK) return 0;
        return norm_grad_workspace_bytes(rope->head_dim);
    } catch (...) {
        dlm_internal_caught();
        return 0;
    }
}

dlm_status dlm_rope_norm_grad(const dlm_rope* rope, int32_t dtype, int32_t rows, const dlm_norm_heads* q,
                              const dlm_norm_heads* k, const dlm_norm_grads* dq, const dlm_norm_grads* dk, float eps,
                              const int32_t* d_pos, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    try {
        TRY(check_norm(rope, dtype, rows, eps, q, k, d_pos));
        TRY(check_norm_set(q, dq, true, dtype, rows, rope->head_dim));
        TRY(check_norm_set(k, dk, true, dtype, rows, rope->head_dim));
        if (!norm_idle(rows, q, k) && k && q->n_heads && k->n_heads && dq->d_dx == dk->d_dx)
            return fail(DLM_ERR_INVALID_ARG, "the sets' results overlap");
        if (dq && k && dk && dq->d_dgain && dq->d_dgain == dk->d_dgain)
            return fail(DLM_ERR_INVALID_ARG, "the gains' gradients overlap");
        TRY(check_workspace(d_workspace, workspace_bytes, norm_grad_workspace_bytes(rope->head_dim)));
        return launched(launch_rope_norm_grad(*rope, dtype, rows, q, k, dq, dk, eps, d_pos, d_workspace,
                                              (hipStream_t)hip_stream), "rope_norm_grad");
    } catch (...) {
        return dlm_internal_caught();
    }
}

size_t dlm_cache_workspace_bytes(const dlm_cache* c, int32_t total_rows, int32_t max_rows, int32_t n_heads) {
    try {
        if (!check_shape(c).empty() || total_rows < 0 || max_rows < 0 || n_heads < 0 || n_heads % c->n_kv_heads) return 0;
        const size_t pages = pages_workspace_bytes(c->n_seqs, c->n_pages);
        if (total_rows == 0 || max_rows == 0 || n_heads == 0) return pages;
        return std::max(pages, attend_workspace_bytes(c->n_seqs, c->n_kv_heads, c->head_dim, total_rows, max_rows,
                                                      n_heads / c->n_kv_heads));
    } catch (...) {
        dlm_internal_caught();
        return 0;
    }
}

dlm_status dlm_cache_reset(const dlm_cache* cache, void* hip_stream) {
    try {
        TRY(check_cache(cache));
        return launched(launch_cache_reset(cache_args(*cache), (hipStream_t)hip_stream), "cache_reset");
    } catch (...) {
        return dlm_internal_caught();
    }
}

dlm_status dlm_cache_reserve(const dlm_cache* cache, const int32_t* d_row_start, int32_t total_rows, int32_t* d_ok,
                             void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    try {
        TRY(check_cache(cache));
        TRY(check_rows(d_row_start, total_rows, total_rows));
        TRY(check_workspace(d_workspace, workspace_bytes, pages_workspace_bytes(cache->n_seqs, cache->n_pages)));
        return launched(launch_reserve(cache_args(*cache), d_row_start, total_rows, d_ok, d_workspace,
                                       (hipStream_t)hip_stream), "cache_reserve");
    } catch (...) {
        return dlm_internal_caught();
    }
}

dlm_status dlm_cache_append(const dlm_cache* cache, int32_t layer, const int32_t* d_row_start, int32_t total_rows,
                            int32_t max_rows, int32_t src_dtype, const void* d_k, int64_t k_stride, const void* d_v,
                            int64_t v_stride, const dlm_rope* rope, const int32_t* d_pos, int32_t n_heads,
                            const void* d_q, int64_t q_stride, void* d_q_out, int64_t q_out_stride, void* hip_stream) {
    try {
        bool nothing;
        TRY(check_append(cache, layer, d_row_start, total_rows, max_rows, src_dtype, d_k, k_stride, d_v, v_stride, rope,
                         n_heads, d_q, q_stride, d_q_out, q_out_stride, &nothing));
        if (nothing) return DLM_OK;
        return launched(launch_append(cache_args(*cache), cache->dtype, layer, d_row_start, total_rows,
                                      std::min(max_rows, total_rows), src_dtype, d_k, k_stride, d_v, v_stride, rope, d_pos,
                                      d_q ? n_heads : 0, d_q, q_stride, d_q_out, q_out_stride, (hipStream_t)hip_stream),
                        "cache_append");
    } catch (...) {
        return dlm_internal_caught();
    }
}

dlm_status dlm_cache_append_norm(const dlm_cache* cache, int32_t layer, const int32_t* d_row_start, int32_t total_rows,
                                 int32_t max_rows, int32_t src_dtype, const void* d_k, int64_t k_stride, const void* d_v,
                                 int64_t v_stride, const dlm_rope* rope, const int32_t* d_pos, int32_t n_heads,
                                 const void* d_q, int64_t q_stride, void* d_q_out, int64_t q_out_stride,
                                 int32_t gain_dtype, const void* d_q_gain, const void* d_k_gain, float eps,
                                 void* hip_stream) {
    try {
        TRY(check_eps(eps));
        bool nothing;
        TRY(check_append(cache, layer, d_row_start, total_rows, max_rows, src_dtype, d_k, k_stride, d_v, v_stride, rope,
                         n_heads, d_q, q_stride, d_q_out, q_out_stride, &nothing));
        TRY(check_gain(src_dtype, gain_dtype, d_q_gain, d_k_gain));
        if (nothing) return DLM_OK;
        return launched(launch_append_norm(cache_args(*cache), cache->dtype, layer, d_row_start, total_rows,
                                           std::min(max_rows, total_rows), src_dtype, d_k, k_stride, d_v, v_stride, rope,
                                           d_pos, d_q ? n_heads : 0, d_q, q_stride, d_q_out, q_out_stride, gain_dtype,
                                           d_q_gain, d_k_gain, eps, (hipStream_t)hip_stream), "cache_append_norm");
    } catch (...) {
        return dlm_internal_caught();
    }
}

dlm_status dlm_cache_attend(const dlm_cache* cache, int32_t layer, const int32_t* d_row_start, int32_t total_rows,
                            int32_t max_rows, int32_t max_keys, int32_t n_heads, const void* d_q, int64_t q_stride,
                            const uint32_t* d_mask, int32_t mask_words, float scale, void* d_o, int64_t o_stride,
                            float* d_lse, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    try {
        bool nothing;
        TRY(check_attend(cache, layer, d_row_start, total_rows, max_rows, max_keys, n_heads, d_q, q_stride, d_mask, mask_words,
                         scale, d_o, o_stride, d_lse, &nothing));
        if (nothing) return DLM_OK;
        const int rows = std::min(max_rows, total_rows), group = n_heads / cache->n_kv_heads;
        TRY(check_workspace(d_workspace, workspace_bytes,
                            attend_workspace_bytes(cache->n_seqs, cache->n_kv_heads, cache->head_dim, total_rows, rows, group)));
        const int keys = (int)std::min<int64_t>(max_keys ? max_keys : capacity(*cache), capacity(*cache));
        return launched(launch_attend(cache_args(*cache), cache->dtype, layer, d_row_start, total_rows, rows, keys, n_heads,
                                      d_q, q_stride, d_mask, d_mask ? mask_words : 0,
                                      scale > 0.f ? scale : 1.f / sqrtf((float)cache->head_dim), d_o, o_stride, d_lse,
                                      d_workspace, (hipStream_t)hip_stream), "cache_attend");
    } catch (...) {
        return dlm_internal_caught();
    }
}

size_t dlm_cache_share_bytes(const dlm_cache* cache, int32_t total_rows) {
    try {
        if (!check_shape(cache).empty() || total_rows < 0 || total_rows > (1 << 24)) return 0;
        return share_bytes(cache->n_seqs, total_rows);
    } catch (...) {
        dlm_internal_caught();
        return 0;
    }
}

dlm_status dlm_cache_share(const dlm_cache* cache, const int32_t* d_row_start, int32_t total_rows, int32_t max_rows,
                           const int32_t* d_group, int32_t max_group_rows, void* d_share, size_t bytes, void* hip_stream) {
    try {
        TRY(check_cache(cache));
        TRY(check_rows(d_row_start, total_rows, max_rows));
        TRY(check_share(*cache, total_rows, max_group_rows, d_share, bytes));
        if (!d_group || !aligned(d_group, 4)) return fail(DLM_ERR_INVALID_ARG, "group must not be NULL and be 4-byte aligned");
        return launched(launch_share(cache_args(*cache), d_row_start, total_rows, std::min(max_rows, total_rows), d_group,
                                     std::min(max_group_rows, total_rows), (int32_t*)d_share, (hipStream_t)hip_stream),
                        "cache_share");
    } catch (...) {
        return dlm_internal_caught();
    }
}

size_t dlm_cache_shared_workspace_bytes(const dlm_cache* c, int32_t total_rows, int32_t max_rows, int32_t max_group_rows,
                                        int32_t n_heads) {
    try {
        if (max_group_rows < 0 || dlm_cache_workspace_bytes(c, total_rows, max_rows, n_heads) == 0) return 0;
        const size_t pages = pages_workspace_bytes(c->n_seqs, c->n_pages);
        if (total_rows == 0 || max_rows == 0 || n_heads == 0) return pages;
        return std::max(pages, attend_shared_workspace_bytes(c->n_seqs, c->n_kv_heads, c->head_dim, total_rows,
                                                             std::min(max_rows, total_rows),
                                                             std::min(max_group_rows, total_rows), n_heads / c->n_kv_heads));
    } catch (...) {
        dlm_internal_caught();
        return 0;
    }
}

dlm_status dlm_cache_attend_shared(const dlm_cache* cache, int32_t layer, const int32_t* d_row_start, int32_t total_rows,
                                   int32_t max_rows, int32_t max_group_rows, int32_t max_keys, const void* d_share,
                                   size_t bytes, int32_t n_heads, const void* d_q, int64_t q_stride, const uint32_t* d_mask,
                                   int32_t mask_words, float scale, void* d_o, int64_t o_stride, float* d_lse,
                                   void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    try {
        bool nothing;
        TRY(check_attend(cache, layer, d_row_start, total_rows, max_rows, max_keys, n_heads, d_q, q_stride, d_mask, mask_words,
                         scale, d_o, o_stride, d_lse, &nothing));
        if (nothing) return DLM_OK;
        const int rows = std::min(max_rows, total_rows), group = n_heads / cache->n_kv_heads;
        TRY(check_share(*cache, total_rows, max_group_rows, d_share, bytes));
        const int group_rows = std::min(max_group_rows, total_rows);
        // A group's rows are counted together where they could share: as a window of so many.
        const std::string bad = attend_may_share(rows, group_rows, group)
                                    ? dlm_internal_check_windows(*cache, n_heads, group_rows) : "";
        if (!bad.empty()) return fail(DLM_ERR_INVALID_ARG, bad);
        TRY(check_workspace(d_workspace, workspace_bytes,
                            attend_shared_workspace_bytes(cache->n_seqs, cache->n_kv_heads, cache->head_dim, total_rows, rows,
                                                          group_rows, group)));
        const int keys = (int)std::min<int64_t>(max_keys ? max_keys : capacity(*cache), capacity(*cache));
        return launched(launch_attend_shared(cache_args(*cache), cache->dtype, layer, d_row_start, total_rows, rows, group_rows,
                                             keys, (const int32_t*)d_share, n_heads, d_q, q_stride, d_mask,
                                             d_mask ? mask_words : 0, scale > 0.f ? scale : 1.f / sqrtf((float)cache->head_dim),
                                             d_o, o_stride, d_lse, d_workspace, (hipStream_t)hip_stream), "cache_attend_shared");
    } catch (...) {
        return dlm_internal_caught();
    }
}

dlm_status dlm_cache_commit(const dlm_cache* cache, const int32_t* d_row_start, int32_t total_rows,
                            const int32_t* d_keep, const int32_t* d_keep_start, int32_t total_keep, int32_t* d_ok,
                            void* hip_stream) {
    try {
        TRY(check_cache(cache));
        TRY(check_rows(d_row_start, total_rows, total_rows));
        if (!d_keep != !d_keep_start) return fail(DLM_ERR_INVALID_ARG, "keep and keep_start go together");
        if (total_keep < 0) return fail(DLM_ERR_INVALID_ARG, "total_keep must be >= 0");
        return launched(launch_commit(cache_args(*cache), d_row_start, total_rows, d_keep, d_keep_start, total_keep, d_ok,
                                      (hipStream_t)hip_stream), "cache_commit");
    } catch (...) {
        return dlm_internal_caught();
    }
}

dlm_status dlm_cache_fork(const dlm_cache* cache, int32_t n_pairs, const int32_t* d_src, const int32_t* d_dst,
                          int32_t* d_ok, void* hip_stream) {
    try {
        TRY(check_cache(cache));
        if (n_pairs < 0 || n_pairs > kCacheMaxSeqs) return fail(DLM_ERR_INVALID_ARG, "n_pairs must be in [0, 1024]");
        if (n_pairs > 0 && (!d_src || !d_dst)) return fail(DLM_ERR_INVALID_ARG, "src or dst is NULL");
        return launched(launch_fork(cache_args(*cache), n_pairs, d_src, d_dst, d_ok, (hipStream_t)hip_stream), "cache_fork");
    } catch (...) {
        return dlm_internal_caught();
    }
}

dlm_status dlm_cache_truncate(const dlm_cache* cache, const int32_t* d_new_len, void* hip_stream) {
    try {
        TRY(check_cache(cache));
        return launched(launch_truncate(cache_args(*cache), d_new_len, (hipStream_t)hip_stream), "cache_truncate");
    } catch (...) {
        return dlm_internal_caught();
    }
}

dlm_status dlm_cache_compact(const dlm_cache* cache, int32_t* d_n_used, void* d_workspace, size_t workspace_bytes,
                             void* hip_stream) {
    try {
        TRY(check_cache(cache));
        TRY(check_workspace(d_workspace, workspace_bytes, pages_workspace_bytes(cache->n_seqs, cache->n_pages)));
        return launched(launch_compact(cache_args(*cache), d_n_used, d_workspace, (hipStream_t)hip_stream), "cache_compact");
    } catch (...) {
        return dlm_internal_caught();
    }
}

size_t dlm_verify_workspace_bytes(int32_t n_seqs, int32_t total_rows, int32_t vocab, int32_t with_draft) {
    try {
        if (!check_verify_sizes(n_seqs, total_rows, vocab).empty()) return 0;
        return verify_workspace_bytes(n_seqs, total_rows, vocab, with_draft != 0);
    } catch (...) {
        dlm_internal_caught();
        return 0;
    }
}

dlm_status dlm_verify(int32_t n_seqs, const int32_t* d_row_start, int32_t total_rows, int32_t max_rows,
                      const int32_t* d_tokens, const int32_t* d_parent, int32_t dtype, int32_t vocab, const void* d_target,
                      int64_t target_stride, const void* d_draft, int64_t draft_stride, double temperature,
                      const float* d_u, const float* d_u_next, int32_t* d_next, int32_t* d_keep, int32_t* d_keep_start,
                      void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    try {
        const std::string bad = check_verify_sizes(n_seqs, total_rows, vocab);
        if (!bad.empty()) return fail(DLM_ERR_INVALID_ARG, bad);
        TRY(check_rows(d_row_start, total_rows, max_rows));
        const int rows = std::min(max_rows, total_rows);
        if (rows > kVerifyMaxRows) return fail(DLM_ERR_INVALID_ARG, "max_rows must be at most 1024");
        if (dtype != DLM_BF16 && dtype != DLM_F16 && dtype != DLM_F32) return fail(DLM_ERR_INVALID_ARG, "unknown dtype");
        // float32 holds log2(e) / temperature, and its product with an infinity is one.
        if (!(temperature == 0. || (temperature >= 1e-30 && temperature <= 1e30)))
            return fail(DLM_ERR_INVALID_ARG, "temperature must be 0 or from 1e-30 to 1e30");
        if (d_draft && d_parent) return fail(DLM_ERR_INVALID_ARG, "with the draft's logits windows are chains: parent must be NULL");
        if (!d_next || !d_keep_start || !d_u_next) return fail(DLM_ERR_INVALID_ARG, "next, keep_start or u_next is NULL");
        if (total_rows > 0 && (!d_tokens || !d_target || !d_u || !d_keep))
            return fail(DLM_ERR_INVALID_ARG, "tokens, target, u or keep is NULL");
        const size_t size = dtype == DLM_F32 ? 4 : 2;
        if (!aligned(d_target, size) || !aligned(d_draft, size) || !aligned(d_row_start, 4) || !aligned(d_tokens, 4) ||
            !aligned(d_parent, 4) || !aligned(d_u, 4) || !aligned(d_u_next, 4) || !aligned(d_next, 4) || !aligned(d_keep, 4) ||
            !aligned(d_keep_start, 4))
            return fail(DLM_ERR_INVALID_ARG, "buffers must be aligned to their elements");
        if (total_rows > 0 && ((total_rows > 1 && target_stride < vocab) || (d_draft && total_rows > 1 && draft_stride < vocab)))
            return fail(DLM_ERR_INVALID_ARG, "target_stride or draft_stride below a row");
        const bool drafts = d_draft && temperature > 0.;
        TRY(check_workspace(d_workspace, workspace_bytes, verify_workspace_bytes(n_seqs, total_rows, vocab, drafts)));
        VerifyArgs a{};
        a.n_seqs = n_seqs;
        a.total_rows = total_rows;
        a.max_rows = rows;
        a.vocab = vocab;
        a.row_start = d_row_start;
        a.tokens = d_tokens;
        a.parent = d_parent;
        a.target = d_target;
        a.draft = drafts ? d_draft : nullptr;
        a.target_stride = target_stride;
        a.draft_stride = draft_stride;
        a.c = temperature > 0. ? 1.4426950408889634 / temperature : 0.;
        a.u = d_u;
        a.u_next = d_u_next;
        a.next = d_next;
        a.keep = d_keep;
        a.keep_start = d_keep_start;
        return launched(launch_verify(a, dtype, d_workspace, (hipStream_t)hip_stream), "verify");
    } catch (...) {
        return dlm_internal_caught();
    }
}

}  // extern "C"
