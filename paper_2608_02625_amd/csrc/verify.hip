// Verification of drafted tokens against the target's logits (dlm_verify).
//
// Row r of the logits says p(v) = 2^(c (z_v - max z)) / sum, c = log2(e) / temperature.
// A drafted token x below the node at hand is accepted when u q(x) < p(x); when it is
// not, what is left of p is max(p - q, 0) (a certain draft: p without x), and the next
// token is the first whose running sum of that passes u' times the whole.
//
//   stats    every row of target and draft in chunks of kChunk tokens, a wave each:
//            maximum and float32 sum
//   walk     a workgroup per sequence: rows' totals, drafted tokens' p and q, the path (kept and
//            rejected rows as bits of the sequence: windows may lie over each other)
//   sums     float64 sums by chunk of the rows that the next token is drawn from
//   rest     with a draft: float64 sums of max(p - q, 0) by chunk, where one was rejected
//   pick     a workgroup per sequence: the next token from chunk sums and one chunk; the
//            kept rows packed
//
// A token is drawn where a running sum over the vocabulary passes a border, and float32
// sums over 157184 tokens move the borders by more than many tokens weigh: so the sums of
// the one row (or pair) that a sequence draws from are float64, of float64 powers (2^t
// reduced to half around the nearest integer, its series to the 11th power, off by at most 9e-15
// of it).
// Whether a drafted token is kept is a single comparison, which float32 sums decide but
// for one in 10^5: when both sides are that near the walk works the row's sum out in
// float64 itself.  Float64 for every row would be bound by its arithmetic (32 chains of up
// to 7 tokens of 157184, bf16: 51 us where the bytes take 18).
//
// `stats` reads the logits once: 190 MB of 16 trees of up to 32 tokens, float32, 31 us (6.1
// TB/s); 94 MB of those chains 21 us (4.5), where a value is half as many bytes.  The others are launches that wait for each other:
// 3.5 to 6 us each for one chain over 32768 tokens, 7 + 12 + 12 + 6 for the 32 chains (sums
// and rest: 10 M float64 powers each, vector units busy 71 and 76 %).
#include <float.h>

#include <algorithm>

#include "common.h"
#include "verify.h"

namespace {

constexpr int kThreads = kVerifyThreads, kWaves = kThreads / 64;
constexpr int kChunk = 2048;                      // tokens of a chunk: 32 per lane of a wave, 8 per thread of a workgroup
constexpr int kPer = kChunk / 64;

// Maximum and sum of 2^(c (z - max)) of a chunk of a row; greedy: the first place of the
// maximum (-1: nothing in it).
struct Part {
    float m, s;
    int32_t at, unused;
};
// What `walk` found for a sequence.
struct Verdict {
    float mp, mq;                                 // maxima of the node's rows; mp -inf: nothing to draw from
    int32_t count, node, best;                    // kept rows; node; greedy's token
    int32_t rest;                                 // its child was rejected, with a draft
    int32_t unused[2];
};

template <typename T>
struct Elems {
    static constexpr int N = 16 / sizeof(T);
};

__device__ __forceinline__ float clean(float z) {
    return z != z ? -INFINITY : fminf(z, FLT_MAX);
}
// A random number in [0, 1).
__device__ __forceinline__ double unit(float u) { return (double)fminf(fmaxf(u, 0.f), 0x1.fffffep-1f); }
template <typename T>
__device__ __forceinline__ float logit(const T* row, int64_t v) { return clean((float)row[v]); }

// 2^t for t <= 0, 0 below 2^-1070.
__device__ __forceinline__ double pow2(double t) {
    t = fmax(t, -1100.0);                         // NaN: -1100
    const double n = __builtin_rint(t), f = t - n;
    // ln(2)^k / k!
    double p = 4.44553827187081e-10;
    p = fma(p, f, 7.054911620801121e-09);
    p = fma(p, f, 1.0178086009239696e-07);
    p = fma(p, f, 1.3215486790144305e-06);
    p = fma(p, f, 1.5252733804059838e-05);
    p = fma(p, f, 0.00015403530393381606);
    p = fma(p, f, 0.0013333558146428441);
    p = fma(p, f, 0.009618129107628477);
    p = fma(p, f, 0.055504108664821576);
    p = fma(p, f, 0.2402265069591007);
    p = fma(p, f, 0.6931471805599453);
    p = fma(p, f, 1.0);
    return ldexp(p, (int)n);
}
__device__ __forceinline__ double weight(float z, float m, double c) { return pow2(((double)z - (double)m) * c); }

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// ------------------------------------------------------------------ chunks

// Chunk ch of a row starts ch * kChunk tokens behind the 16-byte border at or before the
// row's first token, `off` tokens ahead of it, whatever the stride, so that its vectors are
// aligned; the vectors that reach past the row's ends are read token by token.
template <typename T>
__device__ __forceinline__ int row_offset(const T* row) { return (int)(((uintptr_t)row & 15) / sizeof(T)); }

template <typename T, bool ONCE>
__device__ __forceinline__ void load_vector(const T* row, int v, int vocab, float* z) {
    constexpr int E = Elems<T>::N;
    if (v >= 0 && v + E <= vocab) {
        typedef T VT __attribute__((ext_vector_type(E)));
        const VT x = ONCE ? __builtin_nontemporal_load((const VT*)(row + v)) : *(const VT*)(row + v);
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] = (float)x[e];
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] = v + e >= 0 && v + e < vocab ? (float)row[v + e] : -INFINITY;
    }
}
// A wave's chunk from token v0 on: lane's tokens v0 + (k * 64 + lane) * E + e.
template <typename T, bool ONCE>
__device__ __forceinline__ void load_chunk(const T* row, int v0, int vocab, float (&z)[kPer]) {
    constexpr int E = Elems<T>::N;
#pragma unroll
    for (int k = 0; k < kPer / E; ++k) load_vector<T, ONCE>(row, v0 + (k * 64 + (int)(threadIdx.x & 63)) * E, vocab, z + k * E);
}
__device__ __forceinline__ void clean_chunk(float (&z)[kPer]) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) z[i] = clean(z[i]);
}
__device__ __forceinline__ float chunk_max(const float (&z)[kPer]) {
    float m = z[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) m = fmaxf(m, z[i]);
    return wave_max_dpp(m);
}
template <typename T>
__device__ __forceinline__ int chunk_token(int v0, int i) {
    constexpr int E = Elems<T>::N;
    return v0 + (i / E * 64 + (int)(threadIdx.x & 63)) * E + i % E;
}

// ------------------------------------------------------------------ stats

// The exponents of a chunk's tokens that float32 can take as z c - m c in one step, m c
// rounded: all of them are then off by the same, which the sum is corrected for.  A larger
// m c would leave more than 2^(1/16) to correct.
constexpr float kPlainExponent = 0x1p20f;

// Four chunks of a row, a wave each (verify_grid); blockIdx.z: target or draft.
// A chunk is first taken as if its logits were ordinary.  A NaN among them makes the sum
// one, +infinity the maximum, and then they are cleaned and summed again; -infinity needs
// nothing (94 MB of bf16: 24.7 us where every value is cleaned first, 21.2 so).
template <typename T, bool GREEDY>
__global__ __launch_bounds__(kThreads) void stats_kernel(const VerifyArgs a, int chunks, int groups) {
    const bool draft = blockIdx.z;
    const unsigned wg = blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t r = wg / (unsigned)groups;
    const int ch = uniform((int)(wg % (unsigned)groups) * kWaves + (int)(threadIdx.x >> 6));
    if (ch >= chunks || r >= a.total_rows) return;
    const T* row = (const T*)(draft ? a.draft : a.target) + r * (draft ? a.draft_stride : a.target_stride);
    const int v0 = ch * kChunk - row_offset(row);
    float z[kPer];
    load_chunk<T, true>(row, v0, a.vocab, z);
    if constexpr (GREEDY) clean_chunk(z);
    float m = chunk_max(z), s = 0.f;
    int at = 0x7fffffff;
    if constexpr (GREEDY) {
        if (m > -INFINITY) {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (z[i] == m) at = min(at, chunk_token<T>(v0, i));
            for (int o = 32; o; o >>= 1) at = min(at, __shfl_xor(at, o, 64));
        }
    } else if (m != -INFINITY) {
        const float mc = m * a.cf;
        if (fabsf(mc) < kPlainExponent) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) s += __builtin_amdgcn_exp2f(fmaf(z[i], a.cf, -mc));
            s = wave_sum_dpp(s) * __builtin_amdgcn_exp2f(-fmaf(m, a.cf, -mc));
        } else {
            s = NAN;
        }
        if (s != s) {
            clean_chunk(z);
            m = chunk_max(z);
            s = 0.f;
            if (m > -INFINITY) {
#pragma unroll
                for (int i = 0; i < kPer; ++i) s += __builtin_amdgcn_exp2f((z[i] - m) * a.cf);
                s = wave_sum_dpp(s);
            }
        }
    }
    if ((threadIdx.x & 63) == 0)
        ((Part*)a.parts)[((int64_t)draft * a.total_rows + r) * chunks + ch] = Part{m, s, at == 0x7fffffff ? -1 : at, 0};
}

// ------------------------------------------------------------------ walk

struct Window {
    int start, n;
};
__device__ __forceinline__ Window window(const VerifyArgs& a, int b) {
    Window w{a.row_start[b], 0};
    const int end = min(a.row_start[b + 1], a.total_rows);
    if (w.start >= 0 && end > w.start) w.n = min(end - w.start, a.max_rows);
    else w.start = 0;
    return w;
}

// How near, relative to what is compared, float32 sums may leave a comparison: a power is
// off by 2^-24 of its exponent, at most 20 or so where it counts, and by its own rounding.
constexpr double kNear = 1e-5;

// Rows' totals take a wave each, so many waves; the path itself is one wave's work.
constexpr int kWalkThreads = 1024, kWalkWaves = kWalkThreads / 64;

template <typename T>
__global__ __launch_bounds__(kWalkThreads) void walk_kernel(const VerifyArgs a, int chunks) {
    __shared__ double sum[2][kVerifyMaxRows], p[kVerifyMaxRows], q[kVerifyMaxRows];
    __shared__ float top[2][kVerifyMaxRows], zp[kVerifyMaxRows], zq[kVerifyMaxRows];
    __shared__ int best[kVerifyMaxRows], parent[kVerifyMaxRows], token[kVerifyMaxRows];
    __shared__ double lds[kWalkWaves];
    __shared__ int doubt;                         // the row at which the walk waits for exact sums (-1: it is done)
    __shared__ int last;                          // the node that it has come to
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const Window w = window(a, b);
    const bool greedy = a.c == 0.0;
    Verdict* out = (Verdict*)a.verdicts + b;
    if (w.n == 0) {
        if (tid == 0) *out = Verdict{-INFINITY, 0.f, 0, 0, -1, 0, {}};
        return;
    }
    const T *target = (const T*)a.target + (int64_t)w.start * a.target_stride;
    const T *draft = (const T*)a.draft + (int64_t)w.start * a.draft_stride;
    // Drafted tokens and their logits: loads that need no total.
    if (tid < w.n) {
        int up = tid - 1;
        if (tid > 0 && a.parent) up = a.parent[w.start + tid];
        if (up >= tid || up < 0) up = -1;
        const int x = a.tokens[w.start + tid];
        const bool known = up >= 0 && (unsigned)x < (unsigned)a.vocab;
        parent[tid] = up;
        token[tid] = x;
        zp[tid] = known ? logit(target + (int64_t)up * a.target_stride, x) : -INFINITY;
        zq[tid] = known && a.draft ? logit(draft + (int64_t)up * a.draft_stride, x) : -INFINITY;
    }
    const int sets = a.draft ? 2 : 1;
    for (int x = wave; x < sets * w.n; x += kWalkWaves) {
        const int d = x >= w.n, i = d ? x - w.n : x;
        const Part* part = (const Part*)a.parts + ((int64_t)d * a.total_rows + w.start + i) * chunks;
        const Part none{-INFINITY, 0.f, -1, 0};
        const Part y0 = lane < chunks ? part[lane] : none, y1 = lane + 64 < chunks ? part[lane + 64] : none;
        float m = fmaxf(y0.m, y1.m);
        for (int ch = lane + 128; ch < chunks; ch += 64) m = fmaxf(m, part[ch].m);
        m = wave_max_dpp(m);
        double s = 0.0;
        int at = 0x7fffffff;
        auto add = [&](const Part& y) {
            if (y.m > -INFINITY) s += (double)y.s * weight(y.m, m, a.c);
            if (y.at >= 0 && y.m == m) at = min(at, y.at);
        };
        add(y0);
        add(y1);
        for (int ch = lane + 128; ch < chunks; ch += 64) add(part[ch]);
        s = wave_sum64(s);
        if (greedy)
            for (int o = 32; o; o >>= 1) at = min(at, __shfl_xor(at, o, 64));
        if (lane == 0) {
            sum[d][i] = s;
            top[d][i] = m;
            if (!d) best[i] = at == 0x7fffffff ? -1 : at;
        }
    }
    __syncthreads();
    // p and q of the drafted tokens below row `only` (-1: of all).
    auto chances = [&](int only) {
        const int i = tid, up = i < w.n ? parent[i] : -1;
        if (i < w.n && (only < 0 || up == only)) {
            const int x = token[i];
            double pi = 0.0, qi = a.draft ? 0.0 : 1.0;
            if (up >= 0 && greedy) pi = x == best[up] && x >= 0 ? 1.0 : 0.0;
            if (up >= 0 && !greedy) {
                if (sum[0][up] > 0.0) pi = weight(zp[i], top[0][up], a.c) / sum[0][up];
                if (a.draft && sum[1][up] > 0.0) qi = weight(zq[i], top[1][up], a.c) / sum[1][up];
                // A sibling before it with the same token: nothing is left of it.
                if (a.parent)
                    for (int j = up + 1; j < i; ++j)
                        if (parent[j] == up && token[j] == x) pi = 0.0;
            }
            p[i] = pi;
            q[i] = qi;
        }
        __syncthreads();
    };
    chances(-1);
    // The first wave walks, a lane per row, 64 rows at a time: of the rows below the node at
    // hand the next one is tried, until there is none.
    int at = 0, count = 1, rejected = 0, exact = -1, from = 1;     // exact: the node of float64 sums
    double mass = 1.0;                            // what is left of the node's p
    uint32_t kept = tid == 0;                     // of rows 32 lane .. 32 lane + 31, row 0 among them
    bool done = false;
    for (;;) {
        if (wave == 0) {
            int stop = -1;
            for (int i0 = from & ~63; i0 < w.n && !done && stop < 0; i0 += 64) {
                const int i = i0 + lane;
                const bool here = i < w.n;
                const int up = here ? parent[i] : -2;
                const double x = here ? unit(a.u[w.start + i]) * q[i] : 0.0, r = here ? p[i] : 0.0;
                for (;;) {
                    const uint64_t kids = __ballot(up == at && i >= from);
                    if (!kids) break;
                    const int l = __builtin_ctzll(kids);
                    const double lhs = x * mass;
                    const bool near = !greedy && exact != at && r > 0.0 && fabs(lhs - r) <= kNear * (x + r);
                    if ((__ballot(near) >> l) & 1) {
                        stop = i0 + l;
                        break;
                    }
                    from = i0 + l + 1;
                    if ((__ballot(lhs < r) >> l) & 1) {
                        at = i0 + l;
                        kept |= lane == at >> 5 ? 1u << (at & 31) : 0u;
                        ++count;
                        rejected = 0;
                        mass = 1.0;
                        continue;
                    }
                    rejected = 1;
                    if (a.draft) {                // a chain: no other child
                        done = true;
                        break;
                    }
                    mass = fmax(mass - __shfl(r, l, 64), 0.0);
                }
                from = max(from, i0 + 64 < w.n && stop < 0 && !done ? i0 + 64 : from);
            }
            if (lane == 0) {
                doubt = stop;
                last = at;
            }
            if (stop >= 0) from = stop;
        }
        __syncthreads();
        const int row = doubt;
        if (row < 0) break;
        const int node = parent[row];
        for (int d = 0; d < sets; ++d) {
            const T* z = d ? draft + (int64_t)node * a.draft_stride : target + (int64_t)node * a.target_stride;
            double s = 0.0;
            for (int v = tid; v < a.vocab; v += kWalkThreads) s += weight(logit(z, v), top[d][node], a.c);
            s = wave_sum64(s);
            __syncthreads();
            if (lane == 0) lds[wave] = s;
            __syncthreads();
            if (tid == 0) {
                s = lds[0];
                for (int i = 1; i < kWalkWaves; ++i) s += lds[i];
                sum[d][node] = s;
            }
        }
        __syncthreads();
        chances(node);
        exact = node;                             // the first wave's `at`
        if (wave == 0) {                          // the children rejected before it
            mass = 1.0;
            for (int i = node + 1; i < row; ++i)
                if (parent[i] == node) mass = fmax(mass - p[i], 0.0);
        }
    }
    if (!a.draft) {                               // every child of the last node has been rejected
        const uint64_t gone = __ballot(tid < w.n && parent[tid] == last && (unsigned)token[tid] < (unsigned)a.vocab);
        if (wave * 64 < w.n && lane < 2) a.removed[b * kVerifyRowWords + 2 * wave + lane] = (uint32_t)(gone >> (32 * lane));
    }
    if (tid * 32 < w.n) a.kept[b * kVerifyRowWords + tid] = kept;
    if (tid) return;
    const bool any = sum[0][at] > 0.0;
    *out = Verdict{any ? top[0][at] : -INFINITY, a.draft ? top[1][at] : 0.f, count, at, best[at], a.draft && rejected, {}};
}

// ------------------------------------------------------------------ sums, rest

// The node's row of a sequence in target or draft.
template <typename T>
__device__ __forceinline__ const T* node_row(const VerifyArgs& a, const Verdict& d, int start, bool draft) {
    const int64_t r = (int64_t)start + d.node;
    return (const T*)(draft ? a.draft : a.target) + r * (draft ? a.draft_stride : a.target_stride);
}
// A workgroup's thread of a chunk: kDraw tokens from v on, those that are gone at -infinity.
constexpr int kDraw = kChunk / kThreads;
template <typename T>
__device__ __forceinline__ void load_target(const VerifyArgs& a, int b, const Window& w, const T* row, int v,
                                            float (&z)[kDraw]) {
    constexpr int E = Elems<T>::N;
#pragma unroll
    for (int k = 0; k < kDraw / E; ++k) load_vector<T, false>(row, v + k * E, a.vocab, z + k * E);
#pragma unroll
    for (int i = 0; i < kDraw; ++i) z[i] = clean(z[i]);
    for (int j = 0; !a.draft && j < w.n; j += 32)
        for (uint32_t bits = a.removed[b * kVerifyRowWords + (j >> 5)]; bits; bits &= bits - 1) {
            const int x = a.tokens[w.start + j + __builtin_ctz(bits)];
#pragma unroll
            for (int i = 0; i < kDraw; ++i)
                if (v + i == x) z[i] = -INFINITY;
        }
}
// The same tokens of the draft's row, whose vectors may lie otherwise.
template <typename T>
__device__ __forceinline__ void load_draft(const VerifyArgs& a, const T* row, int v, float (&z)[kDraw]) {
    constexpr int E = Elems<T>::N;
    if ((uintptr_t)(row + v) % 16 == 0) {
#pragma unroll
        for (int k = 0; k < kDraw / E; ++k) load_vector<T, false>(row, v + k * E, a.vocab, z + k * E);
    } else {
#pragma unroll
        for (int i = 0; i < kDraw; ++i) z[i] = v + i >= 0 && v + i < a.vocab ? (float)row[v + i] : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < kDraw; ++i) z[i] = clean(z[i]);
}
// Sum over the workgroup, in its first thread.
__device__ __forceinline__ double first_sum(double v, double* lds) {
    v = wave_sum64(v);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// A workgroup per chunk.  Sums [2][n_seqs][chunks]: blockIdx.z: target or draft.
template <typename T>
__global__ __launch_bounds__(kThreads) void sums_kernel(const VerifyArgs a, int chunks) {
    __shared__ double lds[kWaves];
    const int ch = blockIdx.x, b = blockIdx.y, set = blockIdx.z;
    const Window w = window(a, b);
    const Verdict d = ((const Verdict*)a.verdicts)[b];
    if (d.count == 0 || !(d.mp > -INFINITY) || (set && !d.rest)) return;
    const T* row = node_row<T>(a, d, w.start, set);
    const int v = ch * kChunk - row_offset(row) + (int)threadIdx.x * kDraw;
    const float m = set ? d.mq : d.mp;
    double s = 0.0;
    if (m > -INFINITY) {
        float z[kDraw];
        load_target(a, b, w, row, v, z);            // with a draft nothing is gone
#pragma unroll
        for (int i = 0; i < kDraw; ++i) s += weight(z[i], m, a.c);
    }
    s = first_sum(s, lds);
    if (threadIdx.x == 0) a.sums[((int64_t)set * a.n_seqs + b) * chunks + ch] = s;
}
// 1 over the sum of a row's chunks; 0 if there is none.
__device__ __forceinline__ double wave_inverse(const double* sums, int chunks) {
    const int lane = threadIdx.x & 63;
    double s = 0.0;
    for (int ch = lane; ch < chunks; ch += 64) s += sums[ch];
    s = wave_sum64(s);
    return s > 0.0 ? 1.0 / s : 0.0;
}
// Chunks of the target's row: max(p - q, 0).
template <typename T>
__global__ __launch_bounds__(kThreads) void rest_kernel(const VerifyArgs a, int chunks) {
    __shared__ double lds[kWaves];
    const int ch = blockIdx.x, b = blockIdx.y;
    const Window w = window(a, b);
    const Verdict d = ((const Verdict*)a.verdicts)[b];
    if (!d.rest || !(d.mp > -INFINITY)) return;
    const T* prow = node_row<T>(a, d, w.start, false);
    const int v = ch * kChunk - row_offset(prow) + (int)threadIdx.x * kDraw;
    float z[kDraw], y[kDraw];
    load_target(a, b, w, prow, v, z);
    load_draft(a, node_row<T>(a, d, w.start, true), v, y);
    const double ip = wave_inverse(a.sums + (int64_t)b * chunks, chunks);
    const double iq = wave_inverse(a.sums + ((int64_t)a.n_seqs + b) * chunks, chunks);
    if (ch == 0 && threadIdx.x == 0) {
        a.inverse[2 * b] = ip;
        a.inverse[2 * b + 1] = iq;
    }
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kDraw; ++i) {
        const double x = weight(z[i], d.mp, a.c) * ip;
        s += iq > 0.0 ? fmax(x - weight(y[i], d.mq, a.c) * iq, 0.0) : x;
    }
    s = first_sum(s, lds);
    if (threadIdx.x == 0) a.rest[(int64_t)b * chunks + ch] = s;
}

// ------------------------------------------------------------------ pick

// Sums of v of the threads before this one; *total: of all.
__device__ __forceinline__ double block_scan(double v, double* lds, double* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    double before = 0.0, t = 0.0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        if (i < wave) before += lds[i];
        t += lds[i];
    }
    *total = t;
    return before + (x - v);
}
// The first thread of a workgroup with `hit` (-1: none).
__device__ __forceinline__ int first_thread(bool hit, int* lds) {
    const uint64_t votes = __ballot(hit);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = votes ? __builtin_ctzll(votes) : -1;
    __syncthreads();
    int at = -1;
#pragma unroll
    for (int i = kWaves - 1; i >= 0; --i) at = lds[i] >= 0 ? i * 64 + lds[i] : at;
    return at;
}
__device__ __forceinline__ int last_thread(bool hit, int* lds) {
    const uint64_t votes = __ballot(hit);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = votes ? 63 - __builtin_clzll(votes) : -1;
    __syncthreads();
    int at = -1;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) at = lds[i] >= 0 ? i * 64 + lds[i] : at;
    return at;
}

// Of max(p - q, 0) in all: what equal rows may leave by the rounding of their sums and
// products (a few 2^-53 of p each), with room to spare.
constexpr double kNothing = 0x1p-43;

template <typename T>
__global__ __launch_bounds__(kThreads) void pick_kernel(const VerifyArgs a, int chunks) {
    __shared__ double scan[2][kWaves], part_total[kWaves], chosen_before;
    __shared__ int first[4][kWaves], counts[2][kWaves], chosen;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Verdict* verdicts = (const Verdict*)a.verdicts;
    const Verdict d = verdicts[b];
    const Window w = window(a, b);
    const bool draws = d.count > 0 && a.c != 0.0 && d.mp > -INFINITY;
    // A thread's run of chunks: what they weigh, of p and of max(p - q, 0).
    const double* sums = a.sums + (int64_t)b * chunks;
    const int per = (chunks + kThreads - 1) / kThreads;
    const int c0 = min(tid * per, chunks), c1 = min(c0 + per, chunks);
    double own = 0.0, own_rest = 0.0, ip = 1.0, iq = 0.0;
    if (draws) {
        for (int ch = c0; ch < c1; ++ch) {
            own += sums[ch];
            if (d.rest) own_rest += a.rest[(int64_t)b * chunks + ch];
        }
        if (d.rest) {
            ip = a.inverse[2 * b];
            iq = a.inverse[2 * b + 1];
        }
    }
    const double u = draws ? unit(a.u_next[b]) : 0.0;

    // The kept rows behind those of the sequences before.
    int mine = 0, all = 0;
    for (int s = tid; s < a.n_seqs; s += kThreads) {
        const int n = verdicts[s].count;
        all += n;
        if (s < b) mine += n;
    }
    for (int o = 32; o; o >>= 1) {
        mine += __shfl_xor(mine, o, 64);
        all += __shfl_xor(all, o, 64);
    }
    const double rest_all = wave_sum64(own_rest);
    if (lane == 0) {
        counts[0][wave] = mine;
        counts[1][wave] = all;
        part_total[wave] = rest_all;
    }
    __syncthreads();
    int base = 0, total_keep = 0;
    double rest_total = 0.0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        base += counts[0][i];
        total_keep += counts[1][i];
        rest_total += part_total[i];
    }
    total_keep = min(total_keep, a.total_rows);
    for (int i = tid; i < w.n; i += kThreads) {           // a kept row behind those before it
        const uint32_t* kept = a.kept + b * kVerifyRowWords;
        const uint32_t bits = kept[i >> 5];
        if (!((bits >> (i & 31)) & 1)) continue;
        int at = base + __popc(bits & ((1u << (i & 31)) - 1));
        for (int x = 0; x < i >> 5; ++x) at += __popc(kept[x]);
        if (at < a.total_rows) a.keep[at] = i;
    }
    for (int64_t i = total_keep + (int64_t)b * kThreads + tid; i < a.total_rows; i += (int64_t)a.n_seqs * kThreads) a.keep[i] = -1;
    if (tid == 0) {
        a.keep_start[b] = min(base, a.total_rows);
        if (b == a.n_seqs - 1) a.keep_start[a.n_seqs] = total_keep;
        if (!draws) a.next[b] = d.count && a.c == 0.0 ? d.best : -1;
    }
    if (!draws) return;

    const T *prow = node_row<T>(a, d, w.start, false), *qrow = nullptr;
    if (d.rest && rest_total > kNothing) {        // else p = q but for rounding: then from p
        sums = a.rest + (int64_t)b * chunks;
        own = own_rest;
        if (iq > 0.0) qrow = node_row<T>(a, d, w.start, true);
    } else {
        ip = 1.0;
    }
    // The first chunk at which the running sum passes the border; rounding may leave none:
    // then the last of positive weight, and its last such token.
    double total;
    double run = block_scan(own, scan[0], &total);
    const double border = u * total;
    const int t = first_thread(run + own > border && own > 0.0, first[0]);
    const int back = t >= 0 ? t : last_thread(own > 0.0, first[1]);
    if (tid == (back >= 0 ? back : 0)) {
        int ch = -1;
        double before = 0.0;
        for (int i = c0; i < c1; ++i) {
            const double x = sums[i];
            if (x > 0.0) {
                ch = i;
                before = run;
                if (t >= 0 && run + x > border) break;
            }
            run += x;
        }
        chosen = ch;
        chosen_before = before;
    }
    __syncthreads();
    int ch = chosen, token = -1;
    const double before = chosen_before;
    for (int tries = 0; ch >= 0 && token < 0 && tries < chunks; ++tries, ch = ch + 1 == chunks ? 0 : ch + 1) {
        const int v = ch * kChunk - row_offset(prow) + tid * kDraw;
        float z[kDraw], y[kDraw];
        load_target(a, b, w, prow, v, z);
        if (qrow) load_draft(a, qrow, v, y);
        double x[kDraw];
        own = 0.0;
#pragma unroll
        for (int i = 0; i < kDraw; ++i) {
            x[i] = weight(z[i], d.mp, a.c) * ip;
            if (qrow) x[i] = fmax(x[i] - weight(y[i], d.mq, a.c) * iq, 0.0);
            own += x[i];
        }
        // The first token that passes the border; by rounding none: the last that weighs
        // anything.  No such token (sums that were rounding alone): the first of the next chunks.
        run = block_scan(own, scan[1], &total) + before;
        const double past = tries ? -1.0 : border;
        const int t1 = first_thread(own > 0.0 && (tries || run + own > past), first[2]);
        const int t2 = t1 >= 0 ? t1 : last_thread(own > 0.0, first[3]);
        if (tid == (t2 >= 0 ? t2 : 0)) {
            int hit = -1;
#pragma unroll
            for (int i = 0; i < kDraw; ++i) {
                const bool passed = hit >= 0 && t1 >= 0 && run > past;
                if (x[i] > 0.0 && !passed) hit = v + i;
                run += x[i];
            }
            chosen = t2 >= 0 ? hit : -1;
        }
        __syncthreads();
        token = chosen;
        __syncthreads();
    }
    if (tid == 0) a.next[b] = token;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
// A row may start in the middle of a 16-byte vector of up to 8 tokens.
int64_t row_chunks(int vocab) { return ((int64_t)vocab + 7 + kChunk - 1) / kChunk; }
int64_t row_groups(int vocab) { return (row_chunks(vocab) + kWaves - 1) / kWaves; }

template <typename T>
hipError_t verify_type(const VerifyArgs& a, hipStream_t st) {
    const int chunks = (int)row_chunks(a.vocab), groups = (int)row_groups(a.vocab), sets = a.draft ? 2 : 1;
    const bool greedy = a.c == 0.0;
    // Each reads what those before it left: none runs behind one that was not launched.
    hipError_t e = hipSuccess;
    auto go = [&](auto kernel, dim3 grid, int threads, auto... more) {
        if (e != hipSuccess) return;
        hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, st, a, chunks, more...);
        e = hipGetLastError();
    };
    if (a.total_rows > 0) {
        const VerifyGrid g = verify_grid(verify_workgroups(a.total_rows, a.vocab));
        go(greedy ? stats_kernel<T, true> : stats_kernel<T, false>, dim3(g.x, g.y, sets), kThreads, groups);
    }
    go(walk_kernel<T>, dim3(a.n_seqs), kWalkThreads);
    if (!greedy) go(sums_kernel<T>, dim3(chunks, a.n_seqs, sets), kThreads);
    if (a.draft) go(rest_kernel<T>, dim3(chunks, a.n_seqs), kThreads);
    go(pick_kernel<T>, dim3(a.n_seqs), kThreads);
    return e;
}
// Workspace in order: parts, kept, removed, verdicts, sums, rest and inverses.
struct Sizes {
    size_t parts, rows, verdicts, sums, rest;
    Sizes(int n_seqs, int total_rows, int vocab, bool draft) {
        const size_t chunks = row_chunks(vocab), sets = draft ? 2 : 1;
        parts = round256(sets * total_rows * chunks * sizeof(Part));
        rows = round256((size_t)n_seqs * kVerifyRowWords * 4);
        verdicts = round256((size_t)n_seqs * sizeof(Verdict));
        sums = round256(sets * n_seqs * chunks * 8);
        rest = draft ? round256((size_t)n_seqs * chunks * 8) + round256((size_t)n_seqs * 16) : 0;
    }
};

}  // namespace

int64_t verify_workgroups(int total_rows, int vocab) { return total_rows * row_groups(vocab); }

size_t verify_workspace_bytes(int n_seqs, int total_rows, int vocab, bool draft) {
    const Sizes z(n_seqs, total_rows, vocab, draft);
    return z.parts + 2 * z.rows + z.verdicts + z.sums + z.rest;
}

hipError_t launch_verify(VerifyArgs a, int dtype, void* ws, hipStream_t st) {
    const Sizes z(a.n_seqs, a.total_rows, a.vocab, a.draft != nullptr);
    char* at = (char*)ws;
    a.parts = at;
    a.kept = (uint32_t*)(at += z.parts);
    a.removed = (uint32_t*)(at += z.rows);
    a.verdicts = at += z.rows;
    a.sums = (double*)(at += z.verdicts);
    a.rest = (double*)(at += z.sums);
    a.inverse = (double*)(at + round256((size_t)a.n_seqs * row_chunks(a.vocab) * 8));
    a.cf = (float)a.c;
    if (dtype == DLM_BF16) return verify_type<__bf16>(a, st);
    if (dtype == DLM_F16) return verify_type<_Float16>(a, st);
    return verify_type<float>(a, st);
}
