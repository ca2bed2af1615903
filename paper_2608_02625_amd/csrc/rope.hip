// Rotary positions: a kernel that rotates rows (dlm_rope_apply), and one that
// rotates the keys and queries of a window while it puts keys and values into
// their pages (dlm_cache_append).
//
// A pair (a, b) at position p turns by the angle p w: a' = s (a cos - b sin), b'
// = s (b cos + a sin).  The host passes w / (2 pi) as a fraction of 2^64, so p
// times it, modulo 2^64, is the fraction of a turn: integer arithmetic that is
// exact for every position, where the float32 product p w is off by 2^-24 p w
// (0.03 rad at a position of 2^20).  The top bits give the quadrant, the rest an
// angle within +-1/8 turn for sinpi / cospi.
//
// Bound by the bytes of the rows: a thread takes one vector of pairs of a row,
// computes its sines and cosines once and walks heads with them.  32768 rows of 20
// heads of 128 (336 MB): 63 us, 5.3 TB/s; 32 prompts of up to 1024 rows, float32 to
// pages of bf16 (378 MB): 66 us, 5.7 TB/s; one row of each of 32 sequences: 5.4 us,
// four loads that need each other (the page's references among them, beside the sines).
#include <algorithm>

#include "rotary.h"

namespace {

// V pairs of a head: from src to dst (rotated by (c, s) where `rotate`), the
// pairs being values at offsets o .. o + V - 1 and o + half .. (INTER: at 2 o ..
// 2 (o + V) - 1).
template <typename S, typename D, int V, bool INTER, bool STREAM>
__device__ __forceinline__ void turn_pairs(const S* src, D* dst, int o, int half, const float (&c)[V],
                                           const float (&s)[V], bool rotate) {
    float a[V], b[V];
    if constexpr (INTER) {
        const auto x = load<STREAM, Pairs<S, V>>(src + 2 * o);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            a[i] = to_f32(x.v[2 * i]);
            b[i] = to_f32(x.v[2 * i + 1]);
        }
    } else {
        const auto x = load<STREAM, Vec<S, V>>(src + o), y = load<STREAM, Vec<S, V>>(src + o + half);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            a[i] = to_f32(x.v[i]);
            b[i] = to_f32(y.v[i]);
        }
    }
    if (rotate) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float t = a[i] * c[i] - b[i] * s[i];
            b[i] = b[i] * c[i] + a[i] * s[i];
            a[i] = t;
        }
    }
    if constexpr (INTER) {
        Pairs<D, V> x;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x.v[2 * i] = (D)a[i];
            x.v[2 * i + 1] = (D)b[i];
        }
        store<STREAM>(dst + 2 * o, x);
    } else {
        Vec<D, V> x, y;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x.v[i] = (D)a[i];
            y.v[i] = (D)b[i];
        }
        store<STREAM>(dst + o, x);
        store<STREAM>(dst + o + half, y);
    }
}
template <typename S, typename D, int V, bool STREAM>
__device__ __forceinline__ void pass_values(const S* src, D* dst) {
    const auto x = load<STREAM, Vec<S, V>>(src);
    Vec<D, V> y;
#pragma unroll
    for (int i = 0; i < V; ++i) y.v[i] = (D)to_f32(x.v[i]);
    store<STREAM>(dst, y);
}

// How a workgroup's threads are laid over a head, the heads and the rows:
// `turn` lanes with V pairs each and `pass` lanes with V values behind the
// rotated ones, for each of `slots` heads at a time, for each of `rows` rows.
struct Lanes {
    int turn, pass, slots, rows;
};

template <typename T, int V, bool INTER, bool STREAM>
__global__ __launch_bounds__(256) void rope_kernel(const dlm_rope rope, const T* x, int64_t x_row, int64_t x_head, T* y,
                                                   int64_t y_row, int64_t y_head, const int32_t* __restrict__ pos,
                                                   int rows, int heads, Lanes ln, bool back) {
    const int lanes = ln.turn + ln.pass;
    const int lane = threadIdx.x % lanes, slot = threadIdx.x / lanes;
    const int64_t r = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * ln.rows + slot / ln.slots;
    const uint32_t h0 = slot % ln.slots;                      // unsigned: heads up to 2^31 - 1 and a step more
    if (slot >= ln.slots * ln.rows || r >= rows) return;
    x += r * x_row;
    y += r * y_row;
    if (lane < ln.turn) {
        float c[V], s[V];
        angles<V>(rope.phase, rope.scale, pos[r], lane * V, back, c, s);
#pragma unroll 4
        for (uint32_t h = h0; h < (uint32_t)heads; h += ln.slots)
            turn_pairs<T, T, V, INTER, STREAM>(x + h * x_head, y + h * y_head, lane * V, rope.rot_dim / 2, c, s, true);
    } else {
        const int o = rope.rot_dim + (lane - ln.turn) * V;
#pragma unroll 2
        for (uint32_t h = h0; h < (uint32_t)heads; h += ln.slots) pass_values<T, T, V, STREAM>(x + h * x_head + o, y + h * y_head + o);
    }
}

// Keys, values and queries of the rows of sequence blockIdx.y.  Head indexes run
// over the keys, the values, then the queries.  Values take the keys' lanes
// without a rotation.
template <typename S, typename D, int V, bool INTER, bool STREAM>
__global__ __launch_bounds__(256) void append_kernel(const dlm_rope rope, CacheArgs c, int64_t layer_base,
                                                     const int32_t* __restrict__ row_start, int total_rows,
                                                     int max_rows, const S* k, int64_t k_stride, const S* v,
                                                     int64_t v_stride, const int32_t* __restrict__ pos, int n_heads,
                                                     const S* q, int64_t q_stride, D* q_out, int64_t q_out_stride,
                                                     Lanes ln) {
    const int b = blockIdx.y;
    const int lanes = ln.turn + ln.pass;
    const int lane = threadIdx.x % lanes, slot = threadIdx.x / lanes;
    const int i = (int)(blockIdx.z * gridDim.x + blockIdx.x) * ln.rows + slot / ln.slots;    // max_rows <= 2^24
    const int h0 = slot % ln.slots;
    const int start = row_start[b], end = min(row_start[b + 1], total_rows), len = c.len[b];
    if (slot >= ln.slots * ln.rows || start < 0 || i >= max_rows || start >= end || i >= end - start) return;
    const int64_t r = (int64_t)start + i;
    const int64_t t = (int64_t)len + i;                       // the row's token
    const int64_t entry = t >> c.page_log2;
    int page = -1;
    if (len >= 0 && entry < c.max_pages) page = c.table[(int64_t)b * c.max_pages + entry];
    bool held = page >= 0 && page < c.n_pages;                // else the row's keys and values are dropped
    const int refs = held ? c.ref[page] : 0;
    const int hd = c.head_dim;
    const int64_t head_stride = (int64_t)c.page_len * hd;     // within a page
    const int64_t base = layer_base + (int64_t)(held ? page : 0) * c.n_kv * head_stride + (t & (c.page_len - 1)) * hd;
    const int n_all = 2 * c.n_kv + (q ? n_heads : 0);
    const bool turns = lane < ln.turn;
    const int o = turns ? lane * V : rope.rot_dim + (lane - ln.turn) * V;
    float co[V], si[V];
    const bool rotate = rope.scale != 0.f;                    // 0: no rotation asked for
    if (turns && rotate) angles<V>(rope.phase, rope.scale, pos ? pos[r] : t, o, false, co, si);
    // Only a window without room of its own gets here with a page of others (or one forked
    // since it was reserved).
    if (refs > 1 && counted_elsewhere(c, b, t, page)) held = false;
#pragma unroll 4
    for (int h = h0; h < n_all; h += ln.slots) {
        const S* src;
        D* dst;
        if (h < c.n_kv) {
            src = k + r * k_stride + h * hd;
            dst = reinterpret_cast<D*>(c.k) + base + h * head_stride;
        } else if (h < 2 * c.n_kv) {
            src = v + r * v_stride + (h - c.n_kv) * hd;
            dst = reinterpret_cast<D*>(c.v) + base + (h - c.n_kv) * head_stride;
        } else {
            src = q + r * q_stride + (h - 2 * c.n_kv) * hd;
            dst = q_out + r * q_out_stride + (h - 2 * c.n_kv) * hd;
        }
        if (h < 2 * c.n_kv && !held) continue;
        if (turns)
            turn_pairs<S, D, V, INTER, STREAM>(src, dst, o, rope.rot_dim / 2, co, si, rotate && (h < c.n_kv || h >= 2 * c.n_kv));
        else
            pass_values<S, D, V, STREAM>(src + o, dst + o);
    }
}

// A thread walks heads with its sines and cosines.  How many heads a workgroup takes at
// a time: the number that leaves the fewest threads and turns idle, the largest of
// those (4099 rows of 16 heads of 20 lanes: 9.0 us, where 8 heads of one row leave a
// third of the workgroup idle, 11.0; 20000 rows of 24 heads of 16 lanes: 8 heads of 2
// rows 65 us, 2 heads of 8 rows 78).
Lanes lay_out(const dlm_rope& r, int V, int64_t rows, int heads) {
    const int turn = r.rot_dim / 2 / V, pass = (r.head_dim - r.rot_dim) / V;
    const int most = 256 / (turn + pass);
    Lanes best{turn, pass, 1, 1};
    double best_use = 0.;
    for (int s = 1; s <= heads && s <= most; ++s) {
        const int rows_at_once = (int)std::min<int64_t>(most / s, rows);
        const double use = (double)(s * rows_at_once) / most * heads / (s * (((int64_t)heads + s - 1) / s));
        if (use >= best_use) {
            best_use = use;
            best.slots = s;
            best.rows = rows_at_once;
        }
    }
    return best;
}

template <typename T, int V, bool STREAM = false>
hipError_t rope_layout(const dlm_rope& r, int rows, int heads, const void* x, int64_t xr, int64_t xh, void* y,
                       int64_t yr, int64_t yh, const int32_t* pos, bool back, hipStream_t st) {
    const Lanes ln = lay_out(r, V, rows, heads);
    const int64_t wgs = ((int64_t)rows + ln.rows - 1) / ln.rows;
    const dim3 grid((unsigned)std::min(wgs, kWgsAcross), (unsigned)((wgs + kWgsAcross - 1) / kWgsAcross));
    if (r.interleaved)
        hipLaunchKernelGGL((rope_kernel<T, V, true, STREAM>), grid, dim3(256), 0, st, r, (const T*)x, xr, xh, (T*)y, yr, yh, pos,
                           rows, heads, ln, back);
    else
        hipLaunchKernelGGL((rope_kernel<T, V, false, STREAM>), grid, dim3(256), 0, st, r, (const T*)x, xr, xh, (T*)y, yr, yh, pos,
                           rows, heads, ln, back);
    return hipGetLastError();
}
template <typename T>
hipError_t rope_type(const dlm_rope& r, int rows, int heads, const void* x, int64_t xr, int64_t xh, void* y, int64_t yr,
                     int64_t yh, const int32_t* pos, bool back, hipStream_t st) {
    const int V = pairs_per_access(r, sizeof(T), [&](int n) {
        return fits(x, sizeof(T), n, xr) && fits(x, sizeof(T), n, xh) && fits(y, sizeof(T), n, yr) &&
               fits(y, sizeof(T), n, yh);
    });
    // Widest accesses: 8 pairs of two bytes, 4 of four; interleaved ones half as many.
    constexpr int W = 16 / sizeof(T);
    const bool stream = streams(2 * (int64_t)rows * heads * r.head_dim * sizeof(T));
    if (V == W && stream) return rope_layout<T, W, true>(r, rows, heads, x, xr, xh, y, yr, yh, pos, back, st);
    if (r.interleaved && V == W / 2 && stream)
        return rope_layout<T, W / 2, true>(r, rows, heads, x, xr, xh, y, yr, yh, pos, back, st);
    if constexpr (sizeof(T) == 2)
        if (V == 8) return rope_layout<T, 8>(r, rows, heads, x, xr, xh, y, yr, yh, pos, back, st);
    if (V == 4) return rope_layout<T, 4>(r, rows, heads, x, xr, xh, y, yr, yh, pos, back, st);
    if (V == 2) return rope_layout<T, 2>(r, rows, heads, x, xr, xh, y, yr, yh, pos, back, st);
    return rope_layout<T, 1>(r, rows, heads, x, xr, xh, y, yr, yh, pos, back, st);
}

struct AppendCall {
    const CacheArgs& c;
    int layer;
    const int32_t* row_start;
    int total_rows, max_rows;
    const void *k, *v, *q;
    int64_t k_stride, v_stride, q_stride;
    const dlm_rope& rope;
    const int32_t* pos;
    int n_heads;
    void* q_out;
    int64_t q_out_stride;
    hipStream_t st;
};
template <typename S, typename D, int V, bool STREAM = false>
hipError_t append_layout(const AppendCall& a) {
    const int n_all = 2 * a.c.n_kv + (a.q ? a.n_heads : 0);
    const Lanes ln = lay_out(a.rope, V, a.max_rows, n_all);
    const int64_t wgs = ((int64_t)a.max_rows + ln.rows - 1) / ln.rows;
    const dim3 grid((unsigned)std::min(wgs, kWgsAcross), a.c.n_seqs, (unsigned)((wgs + kWgsAcross - 1) / kWgsAcross));
    const int64_t layer_base = (int64_t)a.layer * a.c.n_pages * a.c.n_kv * a.c.page_len * a.c.head_dim;
    if (a.rope.interleaved)
        hipLaunchKernelGGL((append_kernel<S, D, V, true, STREAM>), grid, dim3(256), 0, a.st, a.rope, a.c, layer_base,
                           a.row_start, a.total_rows, a.max_rows, (const S*)a.k, a.k_stride, (const S*)a.v, a.v_stride,
                           a.pos, a.n_heads, (const S*)a.q, a.q_stride, (D*)a.q_out, a.q_out_stride, ln);
    else
        hipLaunchKernelGGL((append_kernel<S, D, V, false, STREAM>), grid, dim3(256), 0, a.st, a.rope, a.c, layer_base,
                           a.row_start, a.total_rows, a.max_rows, (const S*)a.k, a.k_stride, (const S*)a.v, a.v_stride,
                           a.pos, a.n_heads, (const S*)a.q, a.q_stride, (D*)a.q_out, a.q_out_stride, ln);
    return hipGetLastError();
}
template <typename S, typename D>
hipError_t append_type(const AppendCall& a) {
    const int V = pairs_per_access(a.rope, sizeof(S), [&](int n) {
        return fits(a.k, sizeof(S), n, a.k_stride) && fits(a.v, sizeof(S), n, a.v_stride) &&
               (!a.q || (fits(a.q, sizeof(S), n, a.q_stride) && fits(a.q_out, sizeof(D), n, a.q_out_stride)));
    });
    constexpr int W = 16 / sizeof(S);
    const int64_t width = (int64_t)(2 * a.c.n_kv + (a.q ? a.n_heads : 0)) * a.c.head_dim;
    const bool stream = streams(a.total_rows * width * (int64_t)(sizeof(S) + sizeof(D)));
    if (V == W && stream) return append_layout<S, D, W, true>(a);
    if (a.rope.interleaved && V == W / 2 && stream) return append_layout<S, D, W / 2, true>(a);
    if constexpr (sizeof(S) == 2)
        if (V == 8) return append_layout<S, D, 8>(a);
    if (V == 4) return append_layout<S, D, 4>(a);
    if (V == 2) return append_layout<S, D, 2>(a);
    return append_layout<S, D, 1>(a);
}

}  // namespace

hipError_t launch_rope(const dlm_rope& rope, int dtype, int rows, int heads, const void* x, int64_t x_row,
                       int64_t x_head, void* y, int64_t y_row, int64_t y_head, const int32_t* pos, bool transpose,
                       hipStream_t st) {
    if (heads == 1) x_head = y_head = 0;
    if (dtype == DLM_BF16) return rope_type<__bf16>(rope, rows, heads, x, x_row, x_head, y, y_row, y_head, pos, transpose, st);
    if (dtype == DLM_F16) return rope_type<_Float16>(rope, rows, heads, x, x_row, x_head, y, y_row, y_head, pos, transpose, st);
    return rope_type<float>(rope, rows, heads, x, x_row, x_head, y, y_row, y_head, pos, transpose, st);
}

hipError_t launch_append(const CacheArgs& c, int dtype, int layer, const int32_t* row_start, int total_rows,
                         int max_rows, int src_dtype, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                         const dlm_rope* rope, const int32_t* pos, int n_heads, const void* q, int64_t q_stride,
                         void* q_out, int64_t q_out_stride, hipStream_t st) {
    dlm_rope none{};
    none.head_dim = none.rot_dim = c.head_dim;                // scale 0: values pass through
    const AppendCall a{c, layer, row_start, total_rows, max_rows, k, v, q, k_stride, v_stride, q_stride,
                       rope ? *rope : none, pos, n_heads, q_out, q_out_stride, st};
    if (dtype == DLM_BF16)
        return src_dtype == DLM_F32 ? append_type<float, __bf16>(a) : append_type<__bf16, __bf16>(a);
    return src_dtype == DLM_F32 ? append_type<float, _Float16>(a) : append_type<_Float16, _Float16>(a);
}
