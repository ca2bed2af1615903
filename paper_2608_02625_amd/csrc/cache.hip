// C entry points of the rotary positions and of the paged cache (see
// include/dlm.h): argument checks, sizes, launches.
#include <math.h>

#include <algorithm>
#include <string>

#include "cache.h"
#include "status.h"

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
        // Results must not overlap: heads inside a row, or rows inside a head.
        const int64_t hd = rope->head_dim;
        const int64_t h = heads > 1 ? y_head_stride : 0, r = rows > 1 ? y_row_stride : 0;
        const bool rows_outer = (rows == 1 || r >= (__int128)(heads - 1) * h + hd) && (heads == 1 || h >= hd);
        const bool heads_outer = (heads == 1 || h >= (__int128)(rows - 1) * r + hd) && (rows == 1 || r >= hd);
        if (!rows_outer && !heads_outer) return fail(DLM_ERR_INVALID_ARG, "rows or heads of y overlap");
        if (d_x == d_y && ((rows > 1 && x_row_stride != y_row_stride) || (heads > 1 && x_head_stride != y_head_stride)))
            return fail(DLM_ERR_INVALID_ARG, "in place, x and y must have the same strides");
        return launched(launch_rope(*rope, dtype, rows, heads, d_x, x_row_stride, x_head_stride, d_y, y_row_stride,
                                    y_head_stride, d_pos, transpose != 0, (hipStream_t)hip_stream), "rope");
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
        TRY(check_cache(cache));
        if (layer < 0 || layer >= cache->n_layers) return fail(DLM_ERR_INVALID_ARG, "layer out of range");
        TRY(check_rows(d_row_start, total_rows, max_rows));
        if (src_dtype != cache->dtype && src_dtype != DLM_F32)
            return fail(DLM_ERR_INVALID_ARG, "src_dtype must be the cache's dtype or DLM_F32");
        if (rope) {
            TRY(check_rope(rope));
            if (rope->head_dim != cache->head_dim) return fail(DLM_ERR_INVALID_ARG, "rope and cache differ in head_dim");
        }
        if (total_rows == 0) return DLM_OK;
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
        return launched(launch_append(cache_args(*cache), cache->dtype, layer, d_row_start, total_rows,
                                      std::min(max_rows, total_rows), src_dtype, d_k, k_stride, d_v, v_stride, rope, d_pos,
                                      d_q ? n_heads : 0, d_q, q_stride, d_q_out, q_out_stride, (hipStream_t)hip_stream),
                        "cache_append");
    } catch (...) {
        return dlm_internal_caught();
    }
}

dlm_status dlm_cache_attend(const dlm_cache* cache, int32_t layer, const int32_t* d_row_start, int32_t total_rows,
                            int32_t max_rows, int32_t max_keys, int32_t n_heads, const void* d_q, int64_t q_stride,
                            const uint32_t* d_mask, int32_t mask_words, float scale, void* d_o, int64_t o_stride,
                            float* d_lse, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    try {
        TRY(check_cache(cache));
        if (layer < 0 || layer >= cache->n_layers) return fail(DLM_ERR_INVALID_ARG, "layer out of range");
        TRY(check_rows(d_row_start, total_rows, max_rows));
        if (n_heads < 1 || n_heads % cache->n_kv_heads) return fail(DLM_ERR_INVALID_ARG, "n_heads must be a positive multiple of n_kv_heads");
        if (max_keys < 0) return fail(DLM_ERR_INVALID_ARG, "max_keys must be >= 0");
        if (!(scale >= 0.f) || !std::isfinite(scale)) return fail(DLM_ERR_INVALID_ARG, "scale must be finite and >= 0");
        if (total_rows == 0) return DLM_OK;
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
        const int group = n_heads / cache->n_kv_heads;
        const std::string bad = dlm_internal_check_windows(*cache, n_heads, rows);
        if (!bad.empty()) return fail(DLM_ERR_INVALID_ARG, bad);
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

}  // extern "C"
