// Norms of queries and keys for each head with the rotation in the same pass
// (dlm_rope_norm), their gradient (dlm_rope_norm_grad), and the form that puts keys
// and values into their pages (dlm_cache_append_norm).
//
// A head's row x of n values becomes y = R (g x r), r = 1 / sqrt(mean(x^2) + eps), R
// the rotation at the row's position.  Given dy, with u = R^T dy and h = g u: dg = the
// sum of u x r over rows and heads, dx = r (h - x r mean(h x r)).
//
// A head belongs to a run of lanes of one wave, a power of two of them, each with one
// vector of pairs (or of values behind the rotated ones): the sums over a head are a few
// lane moves, and a head is read once, kept in registers and written once.  The lanes walk
// heads with a row's sines and cosines, the next head's loads in flight; what hides the
// loads beyond that is waves, so few registers count for more than loads per wave (32
// prompts into pages: four heads in flight 90 us, one 80).
//
// Bound by the bytes.  32768 rows of 20 heads of 128, bf16 (336 MB): 64 us, 5.25 TB/s, as
// the rotation alone.  32 prompts of up to 1024 rows, float32 to pages of bf16 (377 MB): 65
// us, 5.8 TB/s.  The vector units are busy 73 % of the time in the norms.  Gradient of 16384
// rows of 20 heads, bf16 (252 MB): 52 us, 4.9 TB/s; there they are busy 85 % of it, and are
// what bounds it.  A row of each of 32 sequences: 5.9 us, four loads that need each other.
#include <algorithm>
#include <type_traits>

#include "rotary.h"

namespace {

// How a workgroup's threads are laid over a head, the heads and the rows: runs of
// `run` lanes (a power of two), of which `turn` chunks hold V pairs each and `pass`
// chunks the values behind the rotated ones; `slots` heads at a time of `rows` rows.
struct NormLanes {
    int turn, pass, run, slots, rows;
};
// Values of a chunk behind the rotated ones: as many bytes as the accesses of a pair's.
template <int V, bool INTER>
constexpr int kPass = INTER && V > 1 ? 2 * V : V;

// Sum over the run of lanes that this one belongs to.
__device__ __forceinline__ float run_sum(float v, int run) {
    if (run >= 2) v += dpp_f<0xB1>(v);                        // quad_perm [1,0,3,2]
    if (run >= 4) v += dpp_f<0x4E>(v);                        // quad_perm [2,3,0,1]
    if (run >= 8) v += dpp_f<0x141>(v);                       // row_half_mirror
    if (run >= 16) v += dpp_f<0x140>(v);                      // row_mirror
    if (run >= 32) v += __shfl_xor(v, 16, 64);
    if (run >= 64) v += __shfl_xor(v, 32, 64);
    return v;
}

// A chunk of a head as it is loaded (whole registers: an array of values would be put
// into memory), and in float32: V pairs (a[i], a[V + i]), or kPass values and zeros.
template <int BYTES>
struct Bits;
template <>
struct Bits<16> { typedef u32x4 type; };
template <>
struct Bits<8> { typedef u32x2 type; };
template <>
struct Bits<4> { typedef uint32_t type; };
template <>
struct Bits<2> { typedef uint16_t type; };

template <typename S, int V, bool INTER>
struct Raw {
    typedef typename Bits<(INTER ? 2 : 1) * V * sizeof(S)>::type X;
    typedef typename Bits<V * sizeof(S)>::type Y;
    X x;                                                      // pairs, their first values, or values
    Y y;                                                      // half layout: the pairs' second values
};
template <typename S, int V, bool INTER, bool STREAM>
__device__ __forceinline__ Raw<S, V, INTER> load_chunk(const S* src, int c, const NormLanes& ln, int rot_dim) {
    constexpr int P = kPass<V, INTER>;
    Raw<S, V, INTER> r{};
    if (c < ln.turn) {
        if constexpr (INTER) {
            if constexpr (V == 1) r.x = __builtin_bit_cast(typename Raw<S, V, INTER>::X, load<STREAM, Pairs<S, V>>(src + 2 * V * c));
            else r.x = load<STREAM, typename Raw<S, V, INTER>::X>(src + 2 * V * c);
        } else {
            r.x = load<STREAM, typename Raw<S, V, INTER>::X>(src + V * c);
            r.y = load<STREAM, typename Raw<S, V, INTER>::Y>(src + V * c + rot_dim / 2);
        }
    } else if (c < ln.turn + ln.pass) {
        if constexpr (INTER && V == 1) r.y = load<false, typename Raw<S, V, INTER>::Y>(src + rot_dim + (c - ln.turn) * P);
        else r.x = load<STREAM, typename Raw<S, V, INTER>::X>(src + rot_dim + (c - ln.turn) * P);
    }
    return r;
}
template <typename S, int V, bool INTER>
__device__ __forceinline__ void widen_chunk(const Raw<S, V, INTER>& r, int c, const NormLanes& ln, float (&a)[2 * V]) {
    const bool turns = c < ln.turn;
    const auto x = __builtin_bit_cast(Vec<S, (INTER ? 2 : 1) * V>, r.x);
    const auto y = __builtin_bit_cast(Vec<S, V>, r.y);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (!INTER) {
            a[i] = to_f32(x.v[i]);
            a[V + i] = to_f32(y.v[i]);
        } else if constexpr (V == 1) {                        // a single value behind the rotated ones
            a[0] = turns ? to_f32(x.v[0]) : to_f32(y.v[0]);
            a[1] = to_f32(x.v[1]);
        } else {                                              // pairs side by side, values in their order
            a[i] = turns ? to_f32(x.v[2 * i]) : to_f32(x.v[i]);
            a[V + i] = turns ? to_f32(x.v[2 * i + 1]) : to_f32(x.v[V + i]);
        }
    }
}
template <typename D, int V, bool INTER, bool STREAM>
__device__ __forceinline__ void store_chunk(D* dst, int c, const NormLanes& ln, int rot_dim, const float (&a)[2 * V]) {
    constexpr int P = kPass<V, INTER>;
    if (c < ln.turn) {
        if constexpr (INTER) {
            Pairs<D, V> x;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x.v[2 * i] = (D)a[i];
                x.v[2 * i + 1] = (D)a[V + i];
            }
            store<STREAM>(dst + 2 * V * c, x);
        } else {
            Vec<D, V> x, y;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x.v[i] = (D)a[i];
                y.v[i] = (D)a[V + i];
            }
            store<STREAM>(dst + V * c, x);
            store<STREAM>(dst + V * c + rot_dim / 2, y);
        }
    } else if (c < ln.turn + ln.pass) {
        Vec<D, P> x;
#pragma unroll
        for (int i = 0; i < P; ++i) x.v[i] = (D)a[i];
        store<STREAM>(dst + rot_dim + (c - ln.turn) * P, x);
    }
}
// Offset in the head of value i of a chunk in float32; -1: none.
template <int V, bool INTER>
__device__ __forceinline__ int value_at(int c, int i, const NormLanes& ln, int rot_dim) {
    constexpr int P = kPass<V, INTER>;
    if (c < ln.turn) {
        if constexpr (INTER) return 2 * (V * c + (i < V ? i : i - V)) + (i < V ? 0 : 1);
        else return i < V ? V * c + i : V * c + i - V + rot_dim / 2;
    }
    return i < P && c < ln.turn + ln.pass ? rot_dim + (c - ln.turn) * P + i : -1;
}

// A row's cosines and sines; 1 and 0 for the values behind the rotated ones, so that
// every lane turns what it holds.
template <int V>
__device__ __forceinline__ void chunk_angles(const dlm_rope& rope, int64_t pos, int c, const NormLanes& ln, bool back,
                                             float (&co)[V], float (&si)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        co[i] = 1.f;
        si[i] = 0.f;
    }
    if (c < ln.turn) angles<V>(rope.phase, rope.scale, pos, c * V, back, co, si);
}
// Cosines and sines of a workgroup's rows: worked out once, a pair per thread, into LDS
// ([rows][pairs]; `pos` tells the position of a row), and from there to the lanes; 1 and 0
// for the values behind the rotated ones, so that every lane turns what it holds.  For
// append, whose workgroups take many heads of few rows (80 -> 70 us); where lanes walk
// several heads of a row they work their own out (norms 67 us, through LDS 69.5).
template <int N>
struct Angles {
    float co[N], si[N];
};
template <int N, typename F>
__device__ __forceinline__ void stage_angles(Angles<N>& lds, const dlm_rope& rope, int rows, bool back, F pos) {
    const int half = rope.rot_dim / 2;
    for (int x = threadIdx.x; x < rows * half; x += blockDim.x) {
        const int row = x / half, i = x - row * half;
        float c[1], s[1];
        angles<1>(rope.phase, rope.scale, pos(row), i, back, c, s);
        lds.co[x] = c[0];
        lds.si[x] = s[0];
    }
}
template <int V, int N>
__device__ __forceinline__ void read_angles(const Angles<N>& lds, int row, int half, int c, bool turns, float (&co)[V],
                                            float (&si)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        co[i] = turns ? lds.co[row * half + (turns ? c * V + i : 0)] : 1.f;
        si[i] = turns ? lds.si[row * half + (turns ? c * V + i : 0)] : 0.f;
    }
}
template <int V>
__device__ __forceinline__ void turn(float (&a)[2 * V], const float (&co)[V], const float (&si)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float t = a[i] * co[i] - a[V + i] * si[i];
        a[V + i] = a[V + i] * co[i] + a[i] * si[i];
        a[i] = t;
    }
}

__device__ __forceinline__ float gain_value(const void* gain, int dtype, int i) {
    if (!gain) return 1.f;
    if (dtype == DLM_F32) return reinterpret_cast<const float*>(gain)[i];
    if (dtype == DLM_BF16) return (float)reinterpret_cast<const __bf16*>(gain)[i];
    return (float)reinterpret_cast<const _Float16*>(gain)[i];
}
// A gain in LDS in the order of the chunks: chunk c's at [c][2 V].
template <int V, bool INTER>
__device__ __forceinline__ void stage_gain(float* lds, int width, const void* gain, int type, const NormLanes& ln, int rot_dim) {
    for (int x = threadIdx.x; x < width; x += blockDim.x) {
        const int at = value_at<V, INTER>(x / (2 * V), x % (2 * V), ln, rot_dim);
        lds[x] = at < 0 ? 0.f : gain_value(gain, type, at);
    }
}
// Chunks of a head, a lane's unused ones included, times their values: 256 chunks of V = 1
// hold 512 values, 64 of V = 4 or 32 of V = 8 as many.
constexpr int kGainWords = 512;

template <int V>
__device__ __forceinline__ float sum_squares(const float (&a)[2 * V]) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) s = fmaf(a[i], a[i], s);
    return s;
}

struct NormSet {
    int heads, gain_dtype;
    const void* gain;
    const void* x;
    int64_t x_row, x_head;
    void* y;
    int64_t y_row, y_head;
};

// Pairs of a workgroup's rows: its lanes hold V per chunk.
template <int V, int CH>
constexpr int kRowPairs = 256 * V * CH;

// A lane asks for its next head before it works on the one at hand.
template <typename T, int V, bool INTER, bool STREAM, int CH>
__global__ __launch_bounds__(256) void norm_kernel(const dlm_rope rope, const NormSet q, const NormSet k, float eps,
                                                   const int32_t* __restrict__ pos, int rows, NormLanes ln) {
    __shared__ __attribute__((aligned(16))) float gains[2 * kGainWords];
    const int width = CH * ln.run * 2 * V;
    const int64_t r0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * ln.rows;
    stage_gain<V, INTER>(gains, width, q.gain, q.gain_dtype, ln, rope.rot_dim);
    stage_gain<V, INTER>(gains + width, width, k.gain, k.gain_dtype, ln, rope.rot_dim);
    __syncthreads();
    const int lane = threadIdx.x & (ln.run - 1), slot = threadIdx.x / ln.run, row = slot / ln.slots;
    const int64_t r = r0 + row;
    if (slot >= ln.slots * ln.rows || r >= rows) return;      // whole runs
    const T *xq = (const T*)q.x + r * q.x_row, *xk = (const T*)k.x + r * k.x_row;
    T *yq = (T*)q.y + r * q.y_row, *yk = (T*)k.y + r * k.y_row;
    const float inv_n = 1.f / (float)rope.head_dim;
    const uint32_t n_all = (uint32_t)q.heads + (uint32_t)k.heads;
    float co[CH][V], si[CH][V];
    const int64_t p = pos[r];
#pragma unroll
    for (int j = 0; j < CH; ++j) chunk_angles<V>(rope, p, lane + j * ln.run, ln, false, co[j], si[j]);
    Raw<T, V, INTER> raw[CH];
    auto ask = [&](uint32_t h) {
        const T* src = h < (uint32_t)q.heads ? xq + h * q.x_head : xk + (h - q.heads) * k.x_head;
#pragma unroll
        for (int j = 0; j < CH; ++j) raw[j] = load_chunk<T, V, INTER, STREAM>(src, lane + j * ln.run, ln, rope.rot_dim);
    };
    uint32_t h = slot % ln.slots;
    if (h < n_all) ask(h);
    while (h < n_all) {
        const bool is_q = h < (uint32_t)q.heads;
        T* dst = is_q ? yq + h * q.y_head : yk + (h - q.heads) * k.y_head;
        float a[CH][2 * V], ss = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            widen_chunk<T, V, INTER>(raw[j], lane + j * ln.run, ln, a[j]);
            ss += sum_squares<V>(a[j]);
        }
        h += ln.slots;
        if (h < n_all) ask(h);
        const float rs = rsqrtf(run_sum(ss, ln.run) * inv_n + eps);
        const float* g = gains + (is_q ? 0 : width);
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const float* gc = g + (lane + j * ln.run) * 2 * V;
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) a[j][i] *= rs * gc[i];
            turn<V>(a[j], co[j], si[j]);
            store_chunk<T, V, INTER, STREAM>(dst, lane + j * ln.run, ln, rope.rot_dim, a[j]);
        }
    }
}

// ------------------------------------------------------------------ gradient

struct NormGrad {
    const void* dy;
    int64_t dy_row, dy_head;
    void* dx;
    int64_t dx_row, dx_head;
};
// Pairs of a lane in the gradient, and its workgroups, each with a part of one gain's
// gradient: as many as the chip holds at once (5 per CU at 86 VGPRs), so that the parts are
// few and no second turn of workgroups runs half empty.  16384 rows of 20 heads of 128, bf16:
// 8 pairs (146 VGPRs) and 768 workgroups 65 us, 1024 83; 4 pairs and 768, 1024, 1280, 1536
// workgroups 63, 61, 54, 67.
constexpr int kGradPairs = 4;
constexpr int kGradWgs = 1280;

// The first q_wgs workgroups take the queries, the others the keys, each every q_wgs-th (or
// other) group of rows.  A lane asks for its next head before it works on the one at hand.
// The gain's sums stay in registers over all of them, are added over the workgroup's runs in
// order, in float64, and leave one part per workgroup; the second kernel adds the parts in order.
template <typename T, int V, bool INTER, bool STREAM, int CH>
__global__ __launch_bounds__(256) void norm_grad_kernel(const dlm_rope rope, const NormSet q, const NormSet k,
                                                        const NormGrad gq, const NormGrad gk, float eps,
                                                        const int32_t* __restrict__ pos, int rows, NormLanes lq,
                                                        NormLanes lk, int q_wgs, double* __restrict__ parts) {
    __shared__ __attribute__((aligned(16))) float gain[kGainWords];
    __shared__ float sums[256];
    const bool is_q = (int)blockIdx.x < q_wgs;
    const NormSet s = is_q ? q : k;
    const NormGrad g = is_q ? gq : gk;
    const NormLanes ln = is_q ? lq : lk;
    const int wg = is_q ? blockIdx.x : blockIdx.x - q_wgs, wgs = is_q ? q_wgs : gridDim.x - q_wgs;
    stage_gain<V, INTER>(gain, CH * ln.run * 2 * V, s.gain, s.gain_dtype, ln, rope.rot_dim);
    __syncthreads();
    const int lane = threadIdx.x & (ln.run - 1), slot = threadIdx.x / ln.run;
    const float inv_n = 1.f / (float)rope.head_dim;
    float acc[CH][2 * V];
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) acc[j][i] = 0.f;
    int64_t r = (int64_t)wg * ln.rows + slot / ln.slots;
    const int64_t stride = (int64_t)wgs * ln.rows;
    if (slot >= ln.slots * ln.rows) r = rows;
    const int h0 = slot % ln.slots;
    int h = h0;
    Raw<T, V, INTER> nx[CH], ny[CH];
    auto ask = [&](int64_t row, int head) {
        const T *x = (const T*)s.x + row * s.x_row + head * s.x_head, *y = (const T*)g.dy + row * g.dy_row + head * g.dy_head;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            nx[j] = load_chunk<T, V, INTER, STREAM>(x, lane + j * ln.run, ln, rope.rot_dim);
            ny[j] = load_chunk<T, V, INTER, STREAM>(y, lane + j * ln.run, ln, rope.rot_dim);
        }
    };
    int p = 0;
    if (r < rows) {
        p = pos[r];
        ask(r, h);
    }
    float co[CH][V], si[CH][V];
    while (r < rows) {
        float a[CH][2 * V], b[CH][2 * V];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            widen_chunk<T, V, INTER>(nx[j], lane + j * ln.run, ln, a[j]);
            widen_chunk<T, V, INTER>(ny[j], lane + j * ln.run, ln, b[j]);
        }
        if (h == h0) {
#pragma unroll
            for (int j = 0; j < CH; ++j) chunk_angles<V>(rope, p, lane + j * ln.run, ln, true, co[j], si[j]);
            if (r + stride < rows) p = pos[r + stride];
        }
        T* dst = (T*)g.dx + r * g.dx_row + h * g.dx_head;
        h += ln.slots;
        if (h >= s.heads) {
            h = h0;
            r += stride;
        }
        if (r < rows) ask(r, h);
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            turn<V>(b[j], co[j], si[j]);                      // u = R^T dy
            ss += sum_squares<V>(a[j]);
        }
        const float rs = rsqrtf(run_sum(ss, ln.run) * inv_n + eps);
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const float* gc = gain + (lane + j * ln.run) * 2 * V;
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) {
                a[j][i] *= rs;                                // x r
                const float t = b[j][i] * a[j][i];
                acc[j][i] += t;
                dot = fmaf(t, gc[i], dot);
            }
        }
        dot = run_sum(dot, ln.run) * inv_n;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const float* gc = gain + (lane + j * ln.run) * 2 * V;
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) a[j][i] = rs * (b[j][i] * gc[i] - a[j][i] * dot);
            store_chunk<T, V, INTER, STREAM>(dst, lane + j * ln.run, ln, rope.rot_dim, a[j]);
        }
    }
    if (!parts) return;
    // Over the runs of the workgroup, value by value.
    const int runs = ln.slots * ln.rows;
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) {
            __syncthreads();
            sums[threadIdx.x] = acc[j][i];
            __syncthreads();
            if ((int)threadIdx.x < ln.run) {
                double t = 0.0;
                for (int x = 0; x < runs; ++x) t += sums[x * ln.run + threadIdx.x];
                const int at = value_at<V, INTER>(threadIdx.x + j * ln.run, i, ln, rope.rot_dim);
                if (at >= 0) parts[(int64_t)blockIdx.x * rope.head_dim + at] = t;
            }
        }
}

// The parts added in order: blockIdx.x takes 16 values of one gain, 64 runs of parts each.
__global__ __launch_bounds__(1024) void gain_sum_kernel(const double* __restrict__ parts, int q_parts, int k_parts,
                                                        int head_dim, void* out_q, int type_q, void* out_k, int type_k) {
    __shared__ double run[64][17];
    const int v = threadIdx.x & 15, at = threadIdx.x >> 4;
    const int per = (head_dim + 15) / 16, set = blockIdx.x / per, i = blockIdx.x % per * 16 + v;
    const int n = set ? k_parts : q_parts, first = set ? q_parts : 0;
    const int each = (n + 63) / 64, p1 = min(n, (at + 1) * each);
    double t = 0.0;
    if (i < head_dim)
#pragma unroll 16
        for (int p = at * each; p < p1; ++p) t += parts[(int64_t)(first + p) * head_dim + i];
    run[at][v] = t;
    __syncthreads();
    void* out = set ? out_k : out_q;
    if (at || i >= head_dim || !out) return;
#pragma unroll 16
    for (int x = 1; x < 64; ++x) t += run[x][v];
    const int type = set ? type_k : type_q;
    if (type == DLM_F32) reinterpret_cast<float*>(out)[i] = (float)t;
    else if (type == DLM_BF16) reinterpret_cast<__bf16*>(out)[i] = (__bf16)(float)t;
    else reinterpret_cast<_Float16*>(out)[i] = (_Float16)(float)t;
}

// ------------------------------------------------------------------ into pages

// As append_kernel of rope.hip, keys and queries normalised.  Head indexes run over the
// keys, the values, then the queries.
template <typename S, typename D, int V, bool INTER, bool STREAM, int CH>
__global__ __launch_bounds__(256) void append_norm_kernel(const dlm_rope rope, CacheArgs c, int64_t layer_base,
                                                          const int32_t* __restrict__ row_start, int total_rows,
                                                          int max_rows, const NormSet q, const NormSet k, const S* v,
                                                          int64_t v_stride, float eps, const int32_t* __restrict__ pos,
                                                          NormLanes ln) {
    __shared__ __attribute__((aligned(16))) float gains[2 * kGainWords];
    __shared__ __attribute__((aligned(16))) Angles<kRowPairs<V, CH>> ang;
    const int width = CH * ln.run * 2 * V;
    const int b = blockIdx.y;
    const int lane = threadIdx.x & (ln.run - 1), slot = threadIdx.x / ln.run, row = slot / ln.slots;
    const int i0 = (int)(blockIdx.z * gridDim.x + blockIdx.x) * ln.rows, i = i0 + row;       // max_rows <= 2^24
    const int start = row_start[b], end = min(row_start[b + 1], total_rows), len = c.len[b];
    if (start < 0 || start >= end || i0 >= max_rows || i0 >= end - start) return;            // the whole workgroup
    const bool rotate = rope.scale != 0.f;                    // 0: no rotation asked for
    if (rotate)
        stage_angles(ang, rope, ln.rows, false, [&](int x) {
            const int64_t at = min((int64_t)start + i0 + x, (int64_t)end - 1);
            return pos ? (int64_t)pos[at] : (int64_t)len + i0 + x;
        });
    stage_gain<V, INTER>(gains, width, q.gain, q.gain_dtype, ln, rope.rot_dim);
    stage_gain<V, INTER>(gains + width, width, k.gain, k.gain_dtype, ln, rope.rot_dim);
    const int64_t r = (int64_t)start + i;
    const int64_t t = (int64_t)len + i;                       // the row's token
    const bool mine = slot < ln.slots * ln.rows && i < max_rows && i < end - start;
    const int64_t entry = t >> c.page_log2;
    int page = -1;
    if (mine && len >= 0 && entry < c.max_pages) page = c.table[(int64_t)b * c.max_pages + entry];
    bool held = page >= 0 && page < c.n_pages;                // else the row's keys and values are dropped
    const int refs = held ? c.ref[page] : 0;
    __syncthreads();
    if (!mine) return;                                        // whole runs
    const int hd = c.head_dim, n_all = 2 * c.n_kv + q.heads;
    const int64_t head_stride = (int64_t)c.page_len * hd;     // within a page
    const int64_t base = layer_base + (int64_t)(held ? page : 0) * c.n_kv * head_stride + (t & (c.page_len - 1)) * hd;
    Raw<S, V, INTER> raw[CH];
    auto ask = [&](int h) {
        const S* src = h < c.n_kv       ? (const S*)k.x + r * k.x_row + h * hd
                       : h < 2 * c.n_kv ? v + r * v_stride + (h - c.n_kv) * hd
                                        : (const S*)q.x + r * q.x_row + (h - 2 * c.n_kv) * hd;
#pragma unroll
        for (int j = 0; j < CH; ++j) raw[j] = load_chunk<S, V, INTER, STREAM>(src, lane + j * ln.run, ln, rope.rot_dim);
    };
    int h = slot % ln.slots;
    if (h < n_all) ask(h);
    float co[CH][V], si[CH][V];
#pragma unroll
    for (int j = 0; j < CH; ++j)
        read_angles<V>(ang, row, rope.rot_dim / 2, lane + j * ln.run, rotate && lane + j * ln.run < ln.turn, co[j], si[j]);
    if (refs > 1 && counted_elsewhere(c, b, t, page)) held = false;
    const float inv_n = 1.f / (float)hd;
    while (h < n_all) {
        const bool is_k = h < c.n_kv, is_v = !is_k && h < 2 * c.n_kv, drop = h < 2 * c.n_kv && !held;
        D* dst = is_k   ? reinterpret_cast<D*>(c.k) + base + h * head_stride
                 : is_v ? reinterpret_cast<D*>(c.v) + base + (h - c.n_kv) * head_stride
                        : (D*)q.y + r * q.y_row + (h - 2 * c.n_kv) * hd;
        float a[CH][2 * V], ss = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            widen_chunk<S, V, INTER>(raw[j], lane + j * ln.run, ln, a[j]);
            ss += sum_squares<V>(a[j]);
        }
        h += ln.slots;
        if (h < n_all) ask(h);
        if (drop) continue;
        if (!is_v) {
            const float rs = rsqrtf(run_sum(ss, ln.run) * inv_n + eps);
            const float* g = gains + (is_k ? width : 0);
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const float* gc = g + (lane + j * ln.run) * 2 * V;
#pragma unroll
                for (int x = 0; x < 2 * V; ++x) a[j][x] *= rs * gc[x];
                turn<V>(a[j], co[j], si[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < CH; ++j)
            store_chunk<D, V, INTER, STREAM>(dst, lane + j * ln.run, ln, rope.rot_dim, a[j]);
    }
}

// ------------------------------------------------------------------ launches

// Runs of a power of two of lanes; how many heads a workgroup takes at a time: the number
// that leaves the fewest lanes and turns idle, the largest of those.
NormLanes lay_out(const dlm_rope& r, int V, int64_t rows, int64_t heads, int64_t most_slots = 256) {
    const int pass = r.interleaved && V > 1 ? 2 * V : V;
    NormLanes ln{r.rot_dim / 2 / V, (r.head_dim - r.rot_dim) / pass, 1, 1, 1};
    while (ln.run < ln.turn + ln.pass && ln.run < 64) ln.run *= 2;
    const int most = 256 / ln.run;
    double best_use = 0.;
    for (int s = 1; s <= heads && s <= most && s <= most_slots; ++s) {
        const int at_once = (int)std::min<int64_t>(most / s, rows);
        const double use = (double)(s * at_once) / most * heads / (s * ((heads + s - 1) / s));
        if (use >= best_use) {
            best_use = use;
            ln.slots = s;
            ln.rows = at_once;
        }
    }
    return ln;
}

// pairs_per_access, with values behind the rotated ones in accesses as wide as a pair's.
template <typename F>
int pairs_per_chunk(const dlm_rope& r, int elem, F aligned) {
    int V = pairs_per_access(r, elem, aligned);
    if (r.interleaved)
        while (V > 1 && (r.head_dim - r.rot_dim) % (2 * V)) V /= 2;
    return V;
}
// Chunks of a lane: more than one only where a head of up to 256 values is taken in
// pieces so small that a wave has too few lanes for it.
template <int V, typename S, typename F>
hipError_t with_chunks(const dlm_rope& r, const NormLanes& ln, F launch) {
    auto with_layout = [&](auto ch) {
        if constexpr (2 * V * sizeof(S) <= 16)                // pairs_per_access
            if (r.interleaved) return launch(ch, std::true_type{});
        return launch(ch, std::false_type{});
    };
    if constexpr (V <= 2)
        if (ln.turn + ln.pass > 64) return with_layout(std::integral_constant<int, V == 2 ? 2 : 4>{});
    return with_layout(std::integral_constant<int, 1>{});
}

// Heads of a row that a run of lanes walks in the gradient at most, so that its angles, as much
// arithmetic as a head, are worked out once for them: a training step of 16384 rows of 20 heads
// with 2, 4 and 8 of them 107, 95, 97 us.  Fewer where that would leave workgroups idle
// (grad_layout): a row of 20 heads with 1 and 4 of them 9.7 and 11.3 us, 256 rows of 40 heads
// 12.3 and 13.3; 1024 rows of 20 heads, float32, 17.3 and 16.5.
constexpr int kWalk = 4;

struct NormCall {
    const dlm_rope& rope;
    int rows;
    NormSet q, k;
    float eps;
    const int32_t* pos;
    hipStream_t st;
    const NormGrad *gq = nullptr, *gk = nullptr;
    double* parts = nullptr;
    int* q_parts = nullptr;
    int* k_parts = nullptr;
};
template <typename T, int V, bool STREAM = false>
hipError_t grad_layout(const NormCall& a) {
    // Workgroups by the heads of the two sets, at least one for a set that has heads.
    const int64_t all = (int64_t)a.q.heads + a.k.heads;
    // Times that half of the workgroups are full with a head per run.
    const int64_t full = (int64_t)a.rows * all / (kGradWgs / 2 * (256 / lay_out(a.rope, V, 1, 1, 1).run));
    const int walk = (int)std::clamp<int64_t>(full, 1, kWalk);
    const NormLanes lq = lay_out(a.rope, V, a.rows, a.q.heads, std::max(a.q.heads / walk, 1)),
                    lk = lay_out(a.rope, V, a.rows, a.k.heads, std::max(a.k.heads / walk, 1));
    auto groups = [&](const NormLanes& ln, int heads, int64_t most) {
        return heads ? (int)std::min<int64_t>(((int64_t)a.rows + ln.rows - 1) / ln.rows, std::max<int64_t>(most, 1)) : 0;
    };
    const int nk = groups(lk, a.k.heads, kGradWgs * (int64_t)a.k.heads / all);
    const int nq = groups(lq, a.q.heads, kGradWgs - nk);
    *a.q_parts = nq;
    *a.k_parts = nk;
    return with_chunks<V, T>(a.rope, a.q.heads ? lq : lk, [&](auto ch, auto inter) {
        hipLaunchKernelGGL((norm_grad_kernel<T, V, decltype(inter)::value, STREAM, decltype(ch)::value>), dim3((unsigned)(nq + nk)), dim3(256), 0, a.st, a.rope, a.q, a.k, *a.gq, *a.gk, a.eps,
                           a.pos, a.rows, lq, lk, nq, a.parts);
        return hipGetLastError();
    });
}
template <typename T, int V, bool STREAM = false>
hipError_t norm_layout(const NormCall& a) {
    const NormLanes ln = lay_out(a.rope, V, a.rows, (int64_t)a.q.heads + a.k.heads);
    const int64_t wgs = ((int64_t)a.rows + ln.rows - 1) / ln.rows;
    const dim3 grid((unsigned)std::min(wgs, kWgsAcross), (unsigned)((wgs + kWgsAcross - 1) / kWgsAcross));
    return with_chunks<V, T>(a.rope, ln, [&](auto ch, auto inter) {
        hipLaunchKernelGGL((norm_kernel<T, V, decltype(inter)::value, STREAM, decltype(ch)::value>), grid, dim3(256), 0, a.st, a.rope, a.q, a.k, a.eps, a.pos, a.rows, ln);
        return hipGetLastError();
    });
}
template <typename T>
hipError_t norm_type(const NormCall& a) {
    auto set_fits = [&](const NormSet& s, const NormGrad* g, int n) {
        if (s.heads == 0) return true;
        constexpr int e = sizeof(T);
        auto one = [&](const void* p, int64_t row, int64_t head) { return fits(p, e, n, row) && fits(p, e, n, head); };
        if (!one(s.x, s.x_row, s.x_head)) return false;
        return g ? one(g->dy, g->dy_row, g->dy_head) && one(g->dx, g->dx_row, g->dx_head) : one(s.y, s.y_row, s.y_head);
    };
    const int V = pairs_per_chunk(a.rope, sizeof(T), [&](int n) { return set_fits(a.q, a.gq, n) && set_fits(a.k, a.gk, n); });
    constexpr int W = 16 / sizeof(T);
    const bool stream = streams((a.gq ? 3 : 2) * (int64_t)a.rows * ((int64_t)a.q.heads + a.k.heads) * a.rope.head_dim * sizeof(T));
    if (a.gq) {
        if (V >= kGradPairs) return stream ? grad_layout<T, kGradPairs, true>(a) : grad_layout<T, kGradPairs>(a);
        if constexpr (sizeof(T) == 4)
            if (a.rope.interleaved && V == W / 2 && stream) return grad_layout<T, W / 2, true>(a);
        if (V == 2) return grad_layout<T, 2>(a);
        return grad_layout<T, 1>(a);
    }
    if (V == W && stream) return norm_layout<T, W, true>(a);
    if (a.rope.interleaved && V == W / 2 && stream) return norm_layout<T, W / 2, true>(a);
    if constexpr (sizeof(T) == 2)
        if (V == 8) return norm_layout<T, 8>(a);
    if (V == 4) return norm_layout<T, 4>(a);
    if (V == 2) return norm_layout<T, 2>(a);
    return norm_layout<T, 1>(a);
}
hipError_t norm_any(const NormCall& a, int dtype) {
    if (dtype == DLM_BF16) return norm_type<__bf16>(a);
    if (dtype == DLM_F16) return norm_type<_Float16>(a);
    return norm_type<float>(a);
}
NormSet norm_set(const dlm_norm_heads* h) {
    if (!h || h->n_heads == 0) return NormSet{};
    NormSet s{h->n_heads, h->gain_dtype, h->d_gain, h->d_x, h->x_row_stride, h->x_head_stride,
              h->d_y, h->y_row_stride, h->y_head_stride};
    if (s.heads == 1) s.x_head = s.y_head = 0;
    return s;
}
NormGrad norm_grad(const dlm_norm_heads* h, const dlm_norm_grads* g) {
    if (!h || h->n_heads == 0) return NormGrad{};
    NormGrad s{g->d_dy, g->dy_row_stride, g->dy_head_stride, g->d_dx, g->dx_row_stride, g->dx_head_stride};
    if (h->n_heads == 1) s.dy_head = s.dx_head = 0;
    return s;
}

struct AppendNormCall {
    const CacheArgs& c;
    int layer;
    const int32_t* row_start;
    int total_rows, max_rows;
    NormSet q, k;
    const void* v;
    int64_t v_stride;
    const dlm_rope& rope;
    const int32_t* pos;
    float eps;
    hipStream_t st;
};
template <typename S, typename D, int V, bool STREAM = false>
hipError_t append_layout(const AppendNormCall& a) {
    const NormLanes ln = lay_out(a.rope, V, a.max_rows, 2 * a.c.n_kv + a.q.heads);
    const int64_t wgs = ((int64_t)a.max_rows + ln.rows - 1) / ln.rows;
    const dim3 grid((unsigned)std::min(wgs, kWgsAcross), a.c.n_seqs, (unsigned)((wgs + kWgsAcross - 1) / kWgsAcross));
    const int64_t layer_base = (int64_t)a.layer * a.c.n_pages * a.c.n_kv * a.c.page_len * a.c.head_dim;
    return with_chunks<V, S>(a.rope, ln, [&](auto ch, auto inter) {
        hipLaunchKernelGGL((append_norm_kernel<S, D, V, decltype(inter)::value, STREAM, decltype(ch)::value>), grid, dim3(256), 0, a.st, a.rope, a.c, layer_base, a.row_start, a.total_rows, a.max_rows,
                           a.q, a.k, (const S*)a.v, a.v_stride, a.eps, a.pos, ln);
        return hipGetLastError();
    });
}
template <typename S, typename D>
hipError_t append_type(const AppendNormCall& a) {
    const int V = pairs_per_chunk(a.rope, sizeof(S), [&](int n) {
        return fits(a.k.x, sizeof(S), n, a.k.x_row) && fits(a.v, sizeof(S), n, a.v_stride) &&
               (!a.q.heads || (fits(a.q.x, sizeof(S), n, a.q.x_row) && fits(a.q.y, sizeof(D), n, a.q.y_row)));
    });
    constexpr int W = 16 / sizeof(S);
    const int64_t width = (int64_t)(2 * a.c.n_kv + a.q.heads) * a.c.head_dim;
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

hipError_t launch_rope_norm(const dlm_rope& rope, int dtype, int rows, const dlm_norm_heads* q, const dlm_norm_heads* k,
                            float eps, const int32_t* pos, hipStream_t st) {
    return norm_any(NormCall{rope, rows, norm_set(q), norm_set(k), eps, pos, st}, dtype);
}

size_t norm_grad_workspace_bytes(int head_dim) { return (size_t)kGradWgs * head_dim * sizeof(double); }

hipError_t launch_rope_norm_grad(const dlm_rope& rope, int dtype, int rows, const dlm_norm_heads* q,
                                 const dlm_norm_heads* k, const dlm_norm_grads* dq, const dlm_norm_grads* dk, float eps,
                                 const int32_t* pos, void* ws, hipStream_t st) {
    NormCall a{rope, rows, norm_set(q), norm_set(k), eps, pos, st};
    const NormGrad gq = norm_grad(q, dq), gk = norm_grad(k, dk);
    int q_parts = 0, k_parts = 0;
    // A set without heads leaves no parts, and a gain's gradient of zeros.
    void* out_q = q && dq ? dq->d_dgain : nullptr;
    void* out_k = k && dk ? dk->d_dgain : nullptr;
    a.gq = &gq;
    a.gk = &gk;
    a.parts = out_q || out_k ? (double*)ws : nullptr;
    a.q_parts = &q_parts;
    a.k_parts = &k_parts;
    if (rows > 0 && a.q.heads + (int64_t)a.k.heads > 0) {
        const hipError_t e = norm_any(a, dtype);
        if (e != hipSuccess) return e;
    }
    if (!a.parts) return hipSuccess;
    hipLaunchKernelGGL(gain_sum_kernel, dim3(2 * ((rope.head_dim + 15) / 16)), dim3(1024), 0, st, a.parts, q_parts, k_parts,
                       rope.head_dim, out_q, q ? q->gain_dtype : 0, out_k, k ? k->gain_dtype : 0);
    return hipGetLastError();
}

hipError_t launch_append_norm(const CacheArgs& c, int dtype, int layer, const int32_t* row_start, int total_rows,
                              int max_rows, int src_dtype, const void* k, int64_t k_stride, const void* v,
                              int64_t v_stride, const dlm_rope* rope, const int32_t* pos, int n_heads, const void* q,
                              int64_t q_stride, void* q_out, int64_t q_out_stride, int gain_dtype, const void* q_gain,
                              const void* k_gain, float eps, hipStream_t st) {
    dlm_rope none{};
    none.head_dim = none.rot_dim = c.head_dim;                // scale 0: values are not rotated
    const NormSet qs{q ? n_heads : 0, gain_dtype, q_gain, q, q_stride, 0, q_out, q_out_stride, 0};
    const NormSet ks{c.n_kv, gain_dtype, k_gain, k, k_stride, 0, nullptr, 0, 0};
    const AppendNormCall a{c, layer, row_start, total_rows, max_rows, qs, ks, v, v_stride, rope ? *rope : none, pos, eps, st};
    if (dtype == DLM_BF16)
        return src_dtype == DLM_F32 ? append_type<float, __bf16>(a) : append_type<__bf16, __bf16>(a);
    return src_dtype == DLM_F32 ? append_type<float, _Float16>(a) : append_type<_Float16, _Float16>(a);
}
