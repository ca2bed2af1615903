// Verification of drafted tokens against the target's logits (dlm_verify).
//
// Row r of the logits says p(v) = 2^(c (z_v - max z)) / sum, c = log2(e) / temperature.
// A drafted token x below the node at hand is accepted when u q(x) < p(x); when it is
// not, what is left of p is max(p - q, 0) (a certain draft: p without x), and the next
// token is the first whose running sum of that passes u' times the whole.
//
// Sums and their comparisons are float64: a token is drawn where a running sum over the
// vocabulary passes a border, and float32 sums over 157184 tokens move the borders by more
// than many tokens weigh.  The powers are float64 too: reduced to a half around the nearest
// integer, a polynomial (the series of 2^f to the 11th power, off by 6e-15 of the value).
//
//   stats    every row of target and draft in chunks of kChunk tokens: maximum and sum
//   walk     a workgroup per sequence: rows' totals, drafted tokens' p and q, the path
//   rest     with a draft: sums of max(p - q, 0) by chunk, for sequences that rejected
//   pick     a workgroup per sequence: the next token from chunk sums and one chunk; the
//            kept rows packed
//
// Bound by the bytes of the logits, each read once by `stats`.
#include <float.h>

#include <algorithm>

#include "common.h"
#include "verify.h"

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 8192;                      // tokens of a chunk: 32 per thread
constexpr int kPer = kChunk / kThreads;

// Maximum and sum of 2^(c (z - max)) of a chunk of a row, and the first place of the
// maximum (-1: nothing in it).
struct Part {
    double s;
    float m;
    int32_t at;
};
// What `walk` found for a sequence.
struct Verdict {
    double sp, sq;                                // sums of the node's rows
    float mp, mq;
    int32_t count, node, rejected, best;          // kept rows; node; its rejected child (-1: none); greedy's token
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

// ------------------------------------------------------------------ stats

// Chunk blockIdx.x % chunks of row blockIdx.x / chunks; blockIdx.y: target or draft.
// A row's vectors start at the 16-byte border at or before its first token, `off` tokens
// ahead of it, whatever the stride; the vectors that reach past the row's ends are read
// token by token.
template <typename T, bool GREEDY>
__global__ __launch_bounds__(kThreads) void stats_kernel(const VerifyArgs a, int chunks) {
    constexpr int E = Elems<T>::N, NV = kPer / E;
    __shared__ float wave_m[4];
    __shared__ int wave_at[4];
    __shared__ double wave_s[4];
    const bool draft = blockIdx.y;
    const int64_t r = blockIdx.x / (unsigned)chunks;
    const int ch = blockIdx.x % (unsigned)chunks;
    const T* row = (const T*)(draft ? a.draft : a.target) + r * (draft ? a.draft_stride : a.target_stride);
    const int off = (int)(((uintptr_t)row & 15) / sizeof(T));
    const int v0 = ch * kChunk - off;
    float z[NV][E];
    float m = -INFINITY;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int v = v0 + (k * kThreads + (int)threadIdx.x) * E;
        if (v >= 0 && v + E <= a.vocab) {
            typedef T VT __attribute__((ext_vector_type(E)));
            const VT x = __builtin_nontemporal_load((const VT*)(row + v));
#pragma unroll
            for (int e = 0; e < E; ++e) z[k][e] = (float)x[e];
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) z[k][e] = v + e >= 0 && v + e < a.vocab ? (float)row[v + e] : -INFINITY;
        }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            z[k][e] = clean(z[k][e]);
            m = fmaxf(m, z[k][e]);
        }
    const int wave = threadIdx.x >> 6;
    m = wave_max(m);
    if ((threadIdx.x & 63) == 0) wave_m[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(wave_m[0], wave_m[1]), fmaxf(wave_m[2], wave_m[3]));
    if constexpr (GREEDY) {
        int at = 0x7fffffff;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (z[k][e] == m && m > -INFINITY) at = min(at, v0 + (k * kThreads + (int)threadIdx.x) * E + e);
        for (int o = 32; o; o >>= 1) at = min(at, __shfl_xor(at, o, 64));
        if ((threadIdx.x & 63) == 0) wave_at[wave] = at;
        __syncthreads();
        if (threadIdx.x == 0) {
            at = min(min(wave_at[0], wave_at[1]), min(wave_at[2], wave_at[3]));
            ((Part*)a.parts)[r * chunks + ch] = Part{0.0, m, m > -INFINITY ? at : -1};
        }
        return;
    }
    double s = 0.0;
    if (m > -INFINITY) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) s += weight(z[k][e], m, a.c);
    }
    s = wave_sum64(s);
    if ((threadIdx.x & 63) == 0) wave_s[wave] = s;
    __syncthreads();
    if (threadIdx.x == 0)
        ((Part*)a.parts)[((int64_t)draft * a.total_rows + r) * chunks + ch] =
            Part{(wave_s[0] + wave_s[1]) + (wave_s[2] + wave_s[3]), m, -1};
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

template <typename T>
__global__ __launch_bounds__(kThreads) void walk_kernel(const VerifyArgs a, int chunks) {
    __shared__ double sum[2][kVerifyMaxRows], p[kVerifyMaxRows], q[kVerifyMaxRows];
    __shared__ float top[2][kVerifyMaxRows];
    __shared__ int best[kVerifyMaxRows], parent[kVerifyMaxRows], token[kVerifyMaxRows];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const Window w = window(a, b);
    const bool greedy = a.c == 0.0;
    Verdict* out = (Verdict*)a.verdicts + b;
    if (w.n == 0) {
        if (tid == 0) *out = Verdict{0.0, 0.0, 0.f, 0.f, 0, 0, -1, -1};
        return;
    }
    // Totals of the rows: a wave each.
    const int sets = a.draft ? 2 : 1;
    for (int x = tid >> 6; x < sets * w.n; x += kThreads / 64) {
        const int d = x >= w.n, i = d ? x - w.n : x;
        const Part* part = (const Part*)a.parts + ((int64_t)d * a.total_rows + w.start + i) * chunks;
        float m = -INFINITY;
        for (int ch = lane; ch < chunks; ch += 64) m = fmaxf(m, part[ch].m);
        m = wave_max(m);
        double s = 0.0;
        int at = 0x7fffffff;
        for (int ch = lane; ch < chunks; ch += 64) {
            const Part y = part[ch];
            if (y.m > -INFINITY) s += y.s * weight(y.m, m, a.c);
            if (y.at >= 0 && y.m == m) at = min(at, y.at);
        }
        s = wave_sum64(s);
        for (int o = 32; o; o >>= 1) at = min(at, __shfl_xor(at, o, 64));
        if (lane == 0) {
            sum[d][i] = s;
            top[d][i] = m;
            if (!d) best[i] = at == 0x7fffffff ? -1 : at;
        }
    }
    for (int i = tid; i < w.n; i += kThreads) {
        const int up = a.parent ? a.parent[w.start + i] : i - 1;
        parent[i] = i > 0 && up >= 0 && up < i ? up : -1;
        token[i] = a.tokens[w.start + i];
    }
    __syncthreads();
    for (int i = tid; i < w.n; i += kThreads) {
        const int up = parent[i], x = token[i];
        double pi = 0.0, qi = a.draft ? 0.0 : 1.0;
        if (up >= 0 && (unsigned)x < (unsigned)a.vocab) {
            const int64_t r = (int64_t)w.start + up;
            if (greedy) {
                pi = x == best[up] ? 1.0 : 0.0;
            } else {
                if (sum[0][up] > 0.0) pi = weight(logit((const T*)a.target + r * a.target_stride, x), top[0][up], a.c) / sum[0][up];
                if (a.draft) qi = sum[1][up] > 0.0 ? weight(logit((const T*)a.draft + r * a.draft_stride, x), top[1][up], a.c) / sum[1][up] : 0.0;
                // A sibling before it with the same token: nothing is left of it.
                if (a.parent)
                    for (int j = up + 1; j < i; ++j)
                        if (parent[j] == up && token[j] == x) pi = 0.0;
            }
        }
        p[i] = pi;
        q[i] = qi;
    }
    __syncthreads();
    if (tid) return;
    int* path = a.path + w.start;
    int at = 0, count = 1, rejected = -1;
    double mass = 1.0;                            // what is left of the node's p
    path[0] = 0;
    for (int i = 1; i < w.n; ++i) {
        if (parent[i] != at) continue;
        if (unit(a.u[w.start + i]) * mass * q[i] < p[i]) {
            at = i;
            path[count++] = i;
            rejected = -1;
            mass = 1.0;
        } else {
            rejected = i;
            if (a.draft) break;                   // a chain: no other child
            mass = fmax(mass - p[i], 0.0);
        }
    }
    *out = Verdict{sum[0][at], a.draft ? sum[1][at] : 0.0, top[0][at], a.draft ? top[1][at] : 0.f, count, at, rejected, best[at]};
}

// ------------------------------------------------------------------ rest

// A token's weight in what the next one is drawn from: p, or max(p - q, 0).
template <typename T>
struct Rest {
    const T *prow, *qrow;                         // qrow NULL: p alone
    float mp, mq;
    double sp, sq, c;
    __device__ __forceinline__ double operator()(int64_t v) const {
        const double x = weight(logit(prow, v), mp, c);
        if (!qrow) return x;
        return fmax(x / sp - (sq > 0.0 ? weight(logit(qrow, v), mq, c) / sq : 0.0), 0.0);
    }
};
template <typename T>
__device__ __forceinline__ Rest<T> rest_of(const VerifyArgs& a, const Verdict& d, int start, bool with_draft) {
    const int64_t r = (int64_t)start + d.node;
    return Rest<T>{(const T*)a.target + r * a.target_stride,
                   with_draft ? (const T*)a.draft + r * a.draft_stride : nullptr, d.mp, d.mq, d.sp, d.sq, a.c};
}

// Sum over the workgroup, the same in every thread.
__device__ __forceinline__ double block_sum(double v, double* lds) {
    v = wave_sum64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void rest_kernel(const VerifyArgs a, int chunks) {
    __shared__ double lds[4];
    const int b = blockIdx.y, ch = blockIdx.x;
    const Window w = window(a, b);
    const Verdict d = ((const Verdict*)a.verdicts)[b];
    if (w.n == 0 || d.rejected < 0 || !(d.sp > 0.0)) return;
    const Rest<T> rest = rest_of<T>(a, d, w.start, true);
    double s = 0.0;
#pragma unroll 4
    for (int k = 0; k < kPer; ++k) {
        const int v = ch * kChunk + k * kThreads + (int)threadIdx.x;
        if (v < a.vocab) s += rest(v);
    }
    s = block_sum(s, lds);
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
    __syncthreads();
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    double before = 0.0;
    for (int i = 0; i < wave; ++i) before += lds[i];
    *total = ((lds[0] + lds[1]) + lds[2]) + lds[3];
    return before + (x - v);
}

// A workgroup finds the first of n items whose running sum of weights passes `target`;
// thread t has items t * per .. and their weights come from `f`.  Rounding may leave none:
// then the last of positive weight.  -1: no positive weight.  *base: the sum before it.
template <typename F>
__device__ __forceinline__ int first_past(int n, double target, double start, F f, double* lds, int* found, double* base) {
    const int per = (n + kThreads - 1) / kThreads;
    const int i0 = min((int)threadIdx.x * per, n), i1 = min(i0 + per, n);
    double own = 0.0;
    int last = -1;
    for (int i = i0; i < i1; ++i) {
        const double x = f(i);
        own += x;
        if (x > 0.0) last = i;
    }
    double total;
    const double before = start + block_scan(own, lds, &total);
    __syncthreads();
    if (threadIdx.x == 0) {
        found[0] = 0x7fffffff;
        found[1] = -1;
    }
    __syncthreads();
    double run = before;
    int hit = 0x7fffffff;
    if (before + own > target)                    // monotone: the first such thread holds it
        for (int i = i0; i < i1; ++i) {
            const double x = f(i);
            if (run + x > target && x > 0.0) {
                hit = i;
                break;
            }
            run += x;
        }
    if (hit != 0x7fffffff) atomicMin(&found[0], hit);
    if (last >= 0) atomicMax(&found[1], last);
    __syncthreads();
    const int first = found[0], back = found[1];
    const int at = first != 0x7fffffff ? first : back;
    __syncthreads();
    if (at >= i0 && at < i1) {
        run = before;
        for (int i = i0; i < at; ++i) run += f(i);
        lds[0] = run;
    }
    __syncthreads();
    *base = lds[0];
    return at;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void pick_kernel(const VerifyArgs a, int chunks, int rest_chunks) {
    __shared__ double lds[4];
    __shared__ int found[2], counts[2];
    __shared__ uint32_t gone[kChunk / 32];        // tokens of the chunk that were rejected
    const int b = blockIdx.x, tid = threadIdx.x;
    const Verdict* verdicts = (const Verdict*)a.verdicts;
    const Verdict d = verdicts[b];
    const Window w = window(a, b);

    // The kept rows behind those of the sequences before.
    int mine = 0, all = 0;
    for (int s = tid; s < a.n_seqs; s += kThreads) {
        const int n = verdicts[s].count;
        all += n;
        if (s < b) mine += n;
    }
    if (tid < 2) counts[tid] = 0;
    __syncthreads();
    atomicAdd(&counts[0], mine);
    atomicAdd(&counts[1], all);
    __syncthreads();
    const int base = counts[0], total_keep = min(counts[1], a.total_rows);
    for (int i = tid; i < d.count; i += kThreads)
        if (base + i < a.total_rows) a.keep[base + i] = a.path[w.start + i];
    for (int64_t i = total_keep + (int64_t)b * kThreads + tid; i < a.total_rows; i += (int64_t)a.n_seqs * kThreads) a.keep[i] = -1;
    if (tid == 0) {
        a.keep_start[b] = min(base, a.total_rows);
        if (b == a.n_seqs - 1) a.keep_start[a.n_seqs] = total_keep;
    }

    if (d.count == 0 || a.c == 0.0 || !(d.sp > 0.0)) {        // nothing to draw from, or nothing to draw
        if (tid == 0) a.next[b] = d.count && a.c == 0.0 ? d.best : -1;
        return;
    }
    const double u = unit(a.u_next[b]);
    const int64_t row = (int64_t)w.start + d.node;
    const bool is_tree = !a.draft;
    bool with_draft = a.draft && d.rejected >= 0;
    // Rejected children of a certain draft.
    auto removed = [&](int i) {
        return is_tree && d.rejected >= 0 && i > d.node && i <= d.rejected &&
               (a.parent ? a.parent[w.start + i] == d.node : i == d.node + 1);
    };
    const Part* part = (const Part*)a.parts + row * chunks;
    const double* sums = a.rest + (int64_t)b * rest_chunks;
    if (with_draft) {                             // p = q but for rounding: then from p
        double s = 0.0;
        for (int ch = tid; ch < rest_chunks; ch += kThreads) s += sums[ch];
        if (!(block_sum(s, lds) > 0.0)) with_draft = false;
    }
    const Rest<T> rest = rest_of<T>(a, d, w.start, with_draft);
    const int off = with_draft ? 0 : (int)(((uintptr_t)rest.prow & 15) / sizeof(T));
    const int n_chunks = with_draft ? rest_chunks : chunks;
    auto chunk_weight = [&](int ch) {
        if (with_draft) return sums[ch];
        const Part y = part[ch];
        double s = y.m > -INFINITY ? y.s * weight(y.m, d.mp, a.c) : 0.0;
        if (is_tree && d.rejected >= 0) {
            for (int i = d.node + 1; i <= d.rejected; ++i) {
                if (!removed(i)) continue;
                const int x = a.tokens[w.start + i];
                if ((unsigned)x >= (unsigned)a.vocab || (x + off) / kChunk != ch) continue;
                bool again = false;
                for (int j = d.node + 1; j < i; ++j) again |= removed(j) && a.tokens[w.start + j] == x;
                if (!again) s -= rest(x);
            }
        }
        return fmax(s, 0.0);
    };
    double sum = 0.0, before;
    for (int ch = tid; ch < n_chunks; ch += kThreads) sum += chunk_weight(ch);
    const double target = u * block_sum(sum, lds);
    int ch = first_past(n_chunks, target, 0.0, chunk_weight, lds, found, &before);
    int token = -1;
    // Rounding may leave a chunk of positive weight without such a token: the next ones.
    for (int tries = 0; ch >= 0 && ch < n_chunks && token < 0; ++tries, ch = ch + 1 == n_chunks ? 0 : ch + 1) {
        if (tries == n_chunks) break;
        const int v0 = ch * kChunk - off;
        for (int i = tid; i < kChunk / 32; i += kThreads) gone[i] = 0;
        __syncthreads();
        if (is_tree && d.rejected >= 0)
            for (int i = d.node + 1 + tid; i <= d.rejected; i += kThreads) {
                const int x = a.tokens[w.start + i];
                if (removed(i) && x >= v0 && x < v0 + kChunk && (unsigned)x < (unsigned)a.vocab)
                    atomicOr(&gone[(x - v0) >> 5], 1u << ((x - v0) & 31));
            }
        __syncthreads();
        double none;
        const int i = first_past(kChunk, tries ? 0.0 : target, tries ? 0.0 : before, [&](int y) {
            const int v = v0 + y;
            if (v < 0 || v >= a.vocab || ((gone[y >> 5] >> (y & 31)) & 1)) return 0.0;
            return rest(v);
        }, lds, found, &none);
        if (i >= 0) token = v0 + i;
        __syncthreads();
    }
    if (tid == 0) a.next[b] = token;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
// A row may start in the middle of a 16-byte vector of up to 8 tokens.
int64_t stat_chunks(int vocab) { return ((int64_t)vocab + 7 + kChunk - 1) / kChunk; }
int64_t rest_chunks(int vocab) { return ((int64_t)vocab + kChunk - 1) / kChunk; }

template <typename T>
hipError_t verify_type(const VerifyArgs& a, hipStream_t st) {
    const int chunks = (int)stat_chunks(a.vocab), rest = (int)rest_chunks(a.vocab);
    const dim3 grid((unsigned)((int64_t)a.total_rows * chunks), a.draft ? 2 : 1);
    if (a.total_rows > 0) {
        if (a.c == 0.0) hipLaunchKernelGGL((stats_kernel<T, true>), grid, dim3(kThreads), 0, st, a, chunks);
        else hipLaunchKernelGGL((stats_kernel<T, false>), grid, dim3(kThreads), 0, st, a, chunks);
    }
    hipLaunchKernelGGL((walk_kernel<T>), dim3(a.n_seqs), dim3(kThreads), 0, st, a, chunks);
    if (a.draft) hipLaunchKernelGGL((rest_kernel<T>), dim3(rest, a.n_seqs), dim3(kThreads), 0, st, a, rest);
    hipLaunchKernelGGL((pick_kernel<T>), dim3(a.n_seqs), dim3(kThreads), 0, st, a, chunks, rest);
    return hipGetLastError();
}

}  // namespace

int64_t verify_workgroups(int total_rows, int vocab) { return total_rows * stat_chunks(vocab); }

size_t verify_workspace_bytes(int n_seqs, int total_rows, int vocab, bool draft) {
    return round256((size_t)(draft ? 2 : 1) * total_rows * stat_chunks(vocab) * sizeof(Part)) +
           round256((size_t)total_rows * 4) + round256((size_t)n_seqs * sizeof(Verdict)) +
           round256(draft ? (size_t)n_seqs * rest_chunks(vocab) * 8 : 0);
}

hipError_t launch_verify(VerifyArgs a, int dtype, void* ws, hipStream_t st) {
    char* at = (char*)ws;
    a.parts = at;
    at += round256((size_t)(a.draft ? 2 : 1) * a.total_rows * stat_chunks(a.vocab) * sizeof(Part));
    a.path = (int32_t*)at;
    at += round256((size_t)a.total_rows * 4);
    a.verdicts = at;
    at += round256((size_t)a.n_seqs * sizeof(Verdict));
    a.rest = (double*)at;
    if (dtype == DLM_BF16) return verify_type<__bf16>(a, st);
    if (dtype == DLM_F16) return verify_type<_Float16>(a, st);
    return verify_type<float>(a, st);
}
