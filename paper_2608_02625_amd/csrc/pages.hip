// The life of a cache's pages: room for a pass (reserve), its end (commit),
// shared copies (fork), freeing (truncate), and closing up the pool (compact).
//
// References are the only record of which pages are free: ids are handed out by
// scanning them in order, so every outcome is a function of the tables alone,
// and nothing has to be kept between calls.  Counting and handing out is the
// work of one workgroup (latency: a few dependent loads; 8 sequences forked into
// 24 more and a block reserved in each: 4 + 7 us); moving tokens is bound by bytes
// and spread over layers, sequences and key heads.
#include <algorithm>

#include "common.h"
#include "cache.h"

namespace {

constexpr int kPlanThreads = 1024;

// Rows [start, end) of sequence b's window, cut to the packed rows.
__device__ __forceinline__ int window_rows(const int32_t* row_start, int b, int total_rows) {
    const int s = row_start[b], e = min(row_start[b + 1], total_rows);
    return s >= 0 && e > s ? e - s : 0;
}
__device__ __forceinline__ int pages_for(int64_t tokens, int page_log2) {
    return (int)((tokens + (1 << page_log2) - 1) >> page_log2);
}
__device__ __forceinline__ bool names_page(int p, const CacheArgs& c) { return p >= 0 && p < c.n_pages; }

// Exclusive prefix sum over a workgroup of kPlanThreads threads; *total gets the
// sum.  `tmp` holds one int per wave.
__device__ __forceinline__ int block_scan(int v, int* tmp, int* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    __syncthreads();                                  // tmp is free
    if (lane == 63) tmp[wave] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        before += w < wave ? tmp[w] : 0;
        all += tmp[w];
    }
    *total = all;
    return before + x - v;
}

// Ids of pages that are free (want_free) or used, within [lo, hi), in order, to
// list[]: at most `most` of them.  Returns how many there are, all of them
// counted only if fewer than `most`.
__device__ int list_pages(const int32_t* ref, int lo, int hi, bool want_free, int most, int32_t* list, int* tmp) {
    int found = 0;
    for (int base = lo; base < hi && found < most; base += 4 * kPlanThreads) {
        int id[4], n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = base + 4 * (int)threadIdx.x + i;
            const bool hit = p < hi && (ref[p] == 0) == want_free;
            if (hit) id[n++] = p;
        }
        int all;
        int at = found + block_scan(n, tmp, &all);
        for (int i = 0; i < n; ++i, ++at)
            if (at < most) list[at] = id[i];
        found += all;
    }
    return found;
}

// ------------------------------------------------------------------ reserve

struct ReservePlan {          // workspace of reserve
    int32_t* list;            // free pages, then pages given up   [n_pages] each
    int32_t* given_up;
    int2* copy;               // per sequence: page to copy from and to (-1: none)
};

// A sequence is looked after by 16 lanes, which walk the entries of its window.
constexpr int kSeqLanes = 16;

__global__ __launch_bounds__(kPlanThreads) void reserve_plan_kernel(CacheArgs c, const int32_t* __restrict__ row_start,
                                                                    int total_rows, int32_t* ok, ReservePlan ws) {
    __shared__ int tmp[kPlanThreads / 64];
    __shared__ int need[kCacheMaxSeqs], start[kCacheMaxSeqs];
    __shared__ int n_given;
    const int sub = threadIdx.x % kSeqLanes, grp = threadIdx.x / kSeqLanes;
    const int shift = threadIdx.x & 63 & ~(kSeqLanes - 1);     // the lanes' bits in a ballot of the wave
    auto wants = [&](int old) { return !names_page(old, c) || c.ref[old] > 1; };
    auto span = [&](int b, int& first, int& last) {            // table entries of the window, false: it does not fit
        const int n = window_rows(row_start, b, total_rows), len = c.len[b];
        first = last = 0;
        if (n == 0) return true;
        if (len < 0 || pages_for((int64_t)len + n, c.page_log2) > c.max_pages) return false;
        first = len >> c.page_log2;
        last = pages_for((int64_t)len + n, c.page_log2);
        return true;
    };
    if (threadIdx.x == 0) n_given = 0;
    for (int b0 = 0; b0 < c.n_seqs; b0 += kPlanThreads / kSeqLanes) {
        const int b = b0 + grp;
        int first = 0, last = 0, n = 0;
        const bool fit = b < c.n_seqs && span(b, first, last);
        for (int e = first + sub; e < last; e += kSeqLanes) n += wants(c.table[(int64_t)b * c.max_pages + e]);
#pragma unroll
        for (int o = kSeqLanes / 2; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
        if (sub == 0 && b < c.n_seqs) need[b] = fit ? n : -1;
    }
    __syncthreads();
    int total;
    const int mine = threadIdx.x < c.n_seqs ? max(need[threadIdx.x], 0) : 0;
    const int before = block_scan(mine, tmp, &total);
    const int n_free = list_pages(c.ref, 0, c.n_pages, true, min(total, c.n_pages), ws.list, tmp);
    if (threadIdx.x < c.n_seqs) {
        const bool served = need[threadIdx.x] == 0 || (need[threadIdx.x] > 0 && before + mine <= n_free);
        start[threadIdx.x] = served ? before : -1;
        if (ok) ok[threadIdx.x] = served;
    }
    __syncthreads();                                  // the list and start[] are written
    for (int b0 = 0; b0 < c.n_seqs; b0 += kPlanThreads / kSeqLanes) {
        const int b = b0 + grp;
        int first = 0, last = 0;
        const bool go = b < c.n_seqs && span(b, first, last) && start[b] >= 0 && need[b] > 0;
        if (b < c.n_seqs && sub == 0) ws.copy[b] = int2{-1, -1};
        if (!go) first = last = 0;
        int at = go ? start[b] : 0;
        // every lane of a wave makes the same number of turns (ballots)
        int turns = (last - first + kSeqLanes - 1) / kSeqLanes;
#pragma unroll
        for (int o = 32; o >= kSeqLanes; o >>= 1) turns = max(turns, __shfl_xor(turns, o, 64));
        for (int t = 0; t < turns; ++t) {
            const int e = first + t * kSeqLanes + sub;
            int old = -1;
            bool want = false;
            if (e < last) {
                old = c.table[(int64_t)b * c.max_pages + e];
                want = wants(old);
            }
            const uint32_t votes = (uint32_t)(__ballot(want) >> shift) & ((1u << kSeqLanes) - 1);
            const int id = want ? ws.list[at + __popc(votes & ((1u << sub) - 1))] : -1;
            if (names_page(id, c)) {
                c.table[(int64_t)b * c.max_pages + e] = id;
                c.ref[id] = 1;                        // free before: no table names it, no lane asks for it
                if (names_page(old, c)) {
                    // The old page's reference goes only after every lane has decided.
                    ws.given_up[atomicAdd(&n_given, 1)] = old;
                    if (e == first && (c.len[b] & (c.page_len - 1))) ws.copy[b] = int2{old, id};
                }
            }
            at += __popc(votes);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n_given; i += kPlanThreads) atomicSub(&c.ref[ws.given_up[i]], 1);
}

// Tokens of the last, partly filled page of each sequence that got a page of its
// own: one workgroup per (sequence, layer, K or V).  32 sequences, 20 layers, 102 MB
// read and written: 17 us, 6 TB/s (the pages fit the caches).
__global__ __launch_bounds__(256) void reserve_copy_kernel(CacheArgs c, const int2* __restrict__ copy) {
    const int b = blockIdx.y;
    const int2 move = copy[b];
    if (move.x < 0) return;
    const int bytes = (c.len[b] & (c.page_len - 1)) * c.head_dim * 2;
    const int64_t head = (int64_t)c.page_len * c.head_dim * 2, page = head * c.n_kv;
    char* pool = (blockIdx.x & 1 ? c.v : c.k) + (int64_t)(blockIdx.x >> 1) * c.n_pages * page;
    const char* src = pool + move.x * page;
    char* dst = pool + move.y * page;
    constexpr int kHeads = 4;                         // at a time, their loads in flight together
    for (int o = threadIdx.x * 16; o < bytes; o += blockDim.x * 16)
        for (int h = 0; h < c.n_kv; h += kHeads) {
            u32x4 x[kHeads];
#pragma unroll
            for (int i = 0; i < kHeads; ++i)
                if (h + i < c.n_kv) x[i] = *reinterpret_cast<const u32x4*>(src + (h + i) * head + o);
#pragma unroll
            for (int i = 0; i < kHeads; ++i)
                if (h + i < c.n_kv) *reinterpret_cast<u32x4*>(dst + (h + i) * head + o) = x[i];
        }
}

// ------------------------------------------------------------------ commit

// A sequence's list of kept rows, checked by the whole workgroup.
struct Kept {
    int n, len, m, first;     // window rows, tokens before, kept rows, index of the first kept one
    int entry;                // of the window's first token, in thread 0, if ok
    bool ok;                  // the list and the pages allow it
};
__device__ Kept check_commit(const CacheArgs& c, int b, const int32_t* row_start, int total_rows, const int32_t* keep,
                             const int32_t* keep_start, int total_keep) {
    Kept k;
    k.n = window_rows(row_start, b, total_rows);
    k.len = c.len[b];
    k.first = 0;
    k.m = k.n;
    k.entry = -1;
    bool bad = k.len < 0 || pages_for((int64_t)k.len + k.n, c.page_log2) > c.max_pages;
    if (keep_start) {
        k.first = keep_start[b];
        k.m = keep_start[b + 1] - k.first;
        bad |= k.first < 0 || k.m < 0 || k.m > k.n || k.first > total_keep - k.m;
    }
    if (bad) k.m = 0;
    int moved = 0, wrong = bad;
    if (keep && !bad)
        for (int i = threadIdx.x; i < k.m; i += blockDim.x) {
            const int a = keep[k.first + i];
            wrong |= a < 0 || a >= k.n || (i > 0 && keep[k.first + i - 1] >= a);
            moved |= a != i;
        }
    moved = __syncthreads_or(moved);
    if (!bad) {
        const int lo = k.len >> c.page_log2, hi = pages_for((int64_t)k.len + k.n, c.page_log2);
        const int w = pages_for((int64_t)k.len + k.m, c.page_log2);        // written if rows move
        for (int e = lo + threadIdx.x; e < hi; e += blockDim.x) {
            const int p = c.table[(int64_t)b * c.max_pages + e];
            if (e == lo) k.entry = p;
            if (!names_page(p, c))
                wrong = 1;
            else if (moved && e < w)
                wrong |= c.ref[p] > 1;
        }
    }
    k.ok = !__syncthreads_or(wrong);
    return k;
}

// References change as soon as the first sequence frees pages, so none is checked after
// that, and a sequence that passed its checks says so to the kernels behind in its own
// table: the entry of its window's first token, which names a page p of the pool, holds
// -2 - p until its pages are freed.  A table that comes with such an entry names no page
// there, so its sequence is left out, and the check makes the entry -1, which is none too.
__device__ __forceinline__ bool is_verdict(int entry, const CacheArgs& c) { return entry < -1 && -2 - entry < c.n_pages; }
__device__ __forceinline__ int page_of(int entry, const CacheArgs& c) { return is_verdict(entry, c) ? -2 - entry : entry; }
// The verdict's place in the table, null if the window is empty or lies outside of the row.
__device__ __forceinline__ int32_t* verdict_entry(const CacheArgs& c, int b, int n, int len) {
    if (n == 0 || len < 0 || pages_for((int64_t)len + n, c.page_log2) > c.max_pages) return nullptr;
    return c.table + (int64_t)b * c.max_pages + (len >> c.page_log2);
}

// Entries of a table row from `from` on: their pages lose a reference.  Entry `verdict`
// (-1: none) stands for `page`.
__device__ __forceinline__ void release_from(const CacheArgs& c, int b, int from, int verdict = -1, int page = -1) {
    for (int e = from + (int)threadIdx.x; e < c.max_pages; e += blockDim.x) {
        const int64_t at = (int64_t)b * c.max_pages + e;
        const int entry = c.table[at], p = e == verdict ? page : entry;
        if (names_page(p, c)) atomicSub(&c.ref[p], 1);
        if (entry != -1) c.table[at] = -1;
    }
}

// Checks, and without a list (no row moves, no reference counts) the whole of it.
__global__ __launch_bounds__(256) void commit_check_kernel(CacheArgs c, const int32_t* __restrict__ row_start,
                                                           int total_rows, const int32_t* __restrict__ keep,
                                                           const int32_t* __restrict__ keep_start, int total_keep,
                                                           int32_t* ok) {
    const int b = blockIdx.x;
    if (window_rows(row_start, b, total_rows) == 0) {
        if (ok && threadIdx.x == 0) ok[b] = 1;
        return;
    }
    const Kept k = check_commit(c, b, row_start, total_rows, keep, keep_start, total_keep);
    if (k.ok && !keep) release_from(c, b, pages_for((int64_t)k.len + k.m, c.page_log2));
    if (threadIdx.x == 0) {
        if (k.ok && !keep) c.len[b] = k.len + k.m;
        int32_t* verdict = verdict_entry(c, b, k.n, k.len);
        if (keep && k.ok) *verdict = -2 - k.entry;
        else if (keep && verdict && is_verdict(*verdict, c)) *verdict = -1;
        if (ok) ok[b] = k.ok;
    }
}

// Kept rows to the front of the window: one workgroup per (layer, K or V, key head)
// and sequence.  A chunk of rows is read whole before it is written; later rows lie
// behind every place already written (the list rises, so its i-th row is never in
// front of place i).  Latency: five loads that need each other (8 sequences that keep
// one of four blocks of 64, 20 layers of 4 heads of 128, 37 MB: 10 us, with the checks
// and the freeing 18).
constexpr int kMoveLoads = 4;

__global__ __launch_bounds__(256) void commit_move_kernel(CacheArgs c, const int32_t* __restrict__ row_start,
                                                          int total_rows, const int32_t* __restrict__ keep,
                                                          const int32_t* __restrict__ keep_start, int total_keep) {
    const int b = blockIdx.y;
    const int chunks = c.head_dim / 8, rows_at_once = 256 * kMoveLoads / chunks;
    const int h = blockIdx.x % c.n_kv, lk = blockIdx.x / c.n_kv;
    const int64_t head = (int64_t)c.page_len * c.head_dim * 2, page = head * c.n_kv;
    char* pool = (lk & 1 ? c.v : c.k) + (int64_t)(lk >> 1) * c.n_pages * page + h * head;
    const int first = keep_start[b], m = keep_start[b + 1] - first, len = c.len[b];
    const int32_t* verdict = verdict_entry(c, b, window_rows(row_start, b, total_rows), len);
    if (!verdict || !is_verdict(*verdict, c) || first < 0 || m <= 0 || first > total_keep - m) return;
    // Place of a token (chunk threadIdx % chunks of it), in some page whatever the table holds.
    auto place = [&](int row) {
        const int64_t t = (int64_t)len + max(row, 0);
        const int e = (int)min(t >> c.page_log2, (int64_t)c.max_pages - 1);
        const int p = page_of(c.table[(int64_t)b * c.max_pages + e], c);
        return pool + (names_page(p, c) ? p : 0) * page + (t & (c.page_len - 1)) * c.head_dim * 2 +
               (threadIdx.x % chunks) * 16;
    };
    for (int r0 = 0; r0 < m; r0 += rows_at_once) {
        u32x4 x[kMoveLoads];
        char* to[kMoveLoads];
        bool moves[kMoveLoads];
#pragma unroll
        for (int i = 0; i < kMoveLoads; ++i) {
            const int r = r0 + (i * 256 + (int)threadIdx.x) / chunks;
            const int from = r < m ? keep[first + r] : r;
            moves[i] = from != r;
            to[i] = place(r);
            if (moves[i]) x[i] = *reinterpret_cast<const u32x4*>(place(from));
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMoveLoads; ++i)
            if (moves[i]) *reinterpret_cast<u32x4*>(to[i]) = x[i];
        __syncthreads();
    }
}

__global__ __launch_bounds__(256) void commit_release_kernel(CacheArgs c, const int32_t* __restrict__ row_start,
                                                             int total_rows, const int32_t* __restrict__ keep_start) {
    const int b = blockIdx.x;
    const int before = c.len[b], len = before + keep_start[b + 1] - keep_start[b];
    int32_t* verdict = verdict_entry(c, b, window_rows(row_start, b, total_rows), before);
    if (!verdict || !is_verdict(*verdict, c)) return;
    const int page = page_of(*verdict, c), at = before >> c.page_log2, held = pages_for(len, c.page_log2);
    __syncthreads();                                  // every thread has read the length and the entry
    release_from(c, b, held, at, page);
    if (threadIdx.x == 0) {
        if (at < held) *verdict = page;
        c.len[b] = len;
    }
}

// ------------------------------------------------------------------ fork, truncate, reset

__global__ __launch_bounds__(256) void fork_kernel(CacheArgs c, int n_pairs, const int32_t* __restrict__ src,
                                                   const int32_t* __restrict__ dst, int32_t* ok) {
    const int i = blockIdx.x;
    const int s = src[i], d = dst[i];
    int wrong = s < 0 || s >= c.n_seqs || d < 0 || d >= c.n_seqs;
    for (int j = threadIdx.x; j < n_pairs; j += blockDim.x) wrong |= src[j] == d || (j != i && dst[j] == d);
    wrong = __syncthreads_or(wrong);
    if (ok && threadIdx.x == 0) ok[i] = !wrong;
    if (wrong) return;
    // No pair writes a sequence that another one reads, and references only add up.
    const int len = c.len[s];
    const int held = len < 0 ? 0 : min(pages_for(len, c.page_log2), c.max_pages);
    for (int e = threadIdx.x; e < c.max_pages; e += blockDim.x) {
        const int64_t at = (int64_t)d * c.max_pages + e;
        const int old = c.table[at];
        const int p = e < held ? c.table[(int64_t)s * c.max_pages + e] : -1;
        if (names_page(old, c)) atomicSub(&c.ref[old], 1);
        if (names_page(p, c)) atomicAdd(&c.ref[p], 1);
        if (old != p) c.table[at] = p;
    }
    if (threadIdx.x == 0) c.len[d] = len;
}

__global__ __launch_bounds__(256) void truncate_kernel(CacheArgs c, const int32_t* __restrict__ new_len) {
    const int b = blockIdx.x;
    const int want = new_len ? new_len[b] : 0;
    if (want < 0) return;
    const int len = min(want, max(c.len[b], 0));
    __syncthreads();                                  // every thread has read the length
    release_from(c, b, min(pages_for(len, c.page_log2), c.max_pages));
    if (threadIdx.x == 0) c.len[b] = len;
}

__global__ __launch_bounds__(256) void reset_kernel(CacheArgs c) {
    const int64_t n = (int64_t)c.n_seqs * c.max_pages, step = (int64_t)gridDim.x * blockDim.x;
    const int64_t i0 = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    for (int64_t i = i0; i < n; i += step) c.table[i] = -1;
    for (int64_t i = i0; i < c.n_pages; i += step) c.ref[i] = 0;
    for (int64_t i = i0; i < c.n_seqs; i += step) c.len[i] = 0;
}

// ------------------------------------------------------------------ compact

struct CompactPlan {
    int32_t* src;             // [n_pages]
    int32_t* dst;             // [n_pages]
    int32_t* to;              // [n_pages] new id of each page that moves, else -1
    int32_t* n_moves;
};

__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(CacheArgs c, CompactPlan ws, int32_t* n_used_out) {
    __shared__ int tmp[kPlanThreads / 64];
    int used = 0;
    for (int p = threadIdx.x; p < c.n_pages; p += kPlanThreads) {
        used += c.ref[p] != 0;
        ws.to[p] = -1;
    }
    int n_used;
    block_scan(used, tmp, &n_used);
    // as many used pages past n_used as free ones below it
    const int n = list_pages(c.ref, n_used, c.n_pages, false, c.n_pages, ws.src, tmp);
    list_pages(c.ref, 0, n_used, true, c.n_pages, ws.dst, tmp);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPlanThreads) ws.to[ws.src[i]] = ws.dst[i];
    if (threadIdx.x == 0) {
        *ws.n_moves = n;
        if (n_used_out) *n_used_out = n_used;
    }
}

// Pages to their new places.  The work list (page, layer, K or V, piece of 16 KB) is
// walked by a fixed grid, since only the device knows its length; the last workgroups
// bring tables and references in line meanwhile, which the copies do not read.  More
// than the caches hold in general, so past their replacement (273 MB read and written:
// 52 us, 5.3 TB/s; the plan 4.7 us).
constexpr int kPiece = 16384;                         // 4 accesses of 16 bytes per thread

__global__ __launch_bounds__(256) void compact_move_kernel(CacheArgs c, CompactPlan ws, int copy_blocks) {
    const int n = *ws.n_moves;
    if ((int)blockIdx.x < copy_blocks) {
        const int page = c.n_kv * c.page_len * c.head_dim * 2;            // at most 4 MB, a multiple of 2 KB
        const int pieces = (page + kPiece - 1) / kPiece, per_page = 2 * c.n_layers * pieces;
        const int64_t units = (int64_t)n * per_page;
        for (int64_t u = blockIdx.x; u < units; u += copy_blocks) {
            const int i = (int)(u / per_page), rest = (int)(u % per_page);
            const int lk = rest / pieces, o0 = rest % pieces * kPiece + (int)threadIdx.x * 16;
            char* pool = (lk & 1 ? c.v : c.k) + (int64_t)(lk >> 1) * c.n_pages * page;
            const char* src = pool + (int64_t)ws.src[i] * page;
            char* dst = pool + (int64_t)ws.dst[i] * page;
            u32x4 x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (o0 + q * 4096 < page) x[q] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + o0 + q * 4096));
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (o0 + q * 4096 < page) __builtin_nontemporal_store(x[q], reinterpret_cast<u32x4*>(dst + o0 + q * 4096));
        }
        return;
    }
    const int64_t t0 = (int64_t)(blockIdx.x - copy_blocks) * blockDim.x + threadIdx.x;
    const int64_t step = (int64_t)(gridDim.x - copy_blocks) * blockDim.x;
    for (int64_t i = t0; i < (int64_t)c.n_seqs * c.max_pages; i += step) {
        const int p = c.table[i];
        if (names_page(p, c) && ws.to[p] >= 0) c.table[i] = ws.to[p];
    }
    for (int64_t i = t0; i < n; i += step) {
        c.ref[ws.dst[i]] = c.ref[ws.src[i]];
        c.ref[ws.src[i]] = 0;
    }
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t pages_workspace_bytes(int n_seqs, int n_pages) {
    return 3 * round256((size_t)n_pages * 4) + round256((size_t)n_seqs * 8) + 256;
}

hipError_t launch_cache_reset(const CacheArgs& c, hipStream_t st) {
    const int64_t n = std::max<int64_t>((int64_t)c.n_seqs * c.max_pages, c.n_pages);
    hipLaunchKernelGGL(reset_kernel, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 1024)), dim3(256), 0, st, c);
    return hipGetLastError();
}

hipError_t launch_reserve(const CacheArgs& c, const int32_t* row_start, int total_rows, int32_t* ok, void* ws,
                          hipStream_t st) {
    char* p = (char*)ws;
    const size_t ids = round256((size_t)c.n_pages * 4);
    const ReservePlan plan{(int32_t*)p, (int32_t*)(p + ids), (int2*)(p + 2 * ids)};
    hipLaunchKernelGGL(reserve_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, c, row_start, total_rows, ok, plan);
    hipLaunchKernelGGL(reserve_copy_kernel, dim3(2 * c.n_layers, c.n_seqs), dim3(256), 0, st, c, plan.copy);
    return hipGetLastError();
}

hipError_t launch_commit(const CacheArgs& c, const int32_t* row_start, int total_rows, const int32_t* keep,
                         const int32_t* keep_start, int total_keep, int32_t* ok, hipStream_t st) {
    hipLaunchKernelGGL(commit_check_kernel, dim3(c.n_seqs), dim3(256), 0, st, c, row_start, total_rows, keep,
                       keep_start, total_keep, ok);
    if (keep) {
        hipLaunchKernelGGL(commit_move_kernel, dim3(2 * c.n_layers * c.n_kv, c.n_seqs), dim3(256), 0, st, c,
                           row_start, total_rows, keep, keep_start, total_keep);
        hipLaunchKernelGGL(commit_release_kernel, dim3(c.n_seqs), dim3(256), 0, st, c, row_start, total_rows, keep_start);
    }
    return hipGetLastError();
}

hipError_t launch_fork(const CacheArgs& c, int n_pairs, const int32_t* src, const int32_t* dst, int32_t* ok,
                       hipStream_t st) {
    if (n_pairs == 0) return hipSuccess;
    hipLaunchKernelGGL(fork_kernel, dim3(n_pairs), dim3(256), 0, st, c, n_pairs, src, dst, ok);
    return hipGetLastError();
}

hipError_t launch_truncate(const CacheArgs& c, const int32_t* new_len, hipStream_t st) {
    hipLaunchKernelGGL(truncate_kernel, dim3(c.n_seqs), dim3(256), 0, st, c, new_len);
    return hipGetLastError();
}

hipError_t launch_compact(const CacheArgs& c, int32_t* n_used, void* ws, hipStream_t st) {
    char* p = (char*)ws;
    const size_t ids = round256((size_t)c.n_pages * 4);
    const CompactPlan plan{(int32_t*)p, (int32_t*)(p + ids), (int32_t*)(p + 2 * ids), (int32_t*)(p + 3 * ids)};
    hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, c, plan, n_used);
    const int copy_blocks = 2048, table_blocks = 64;
    hipLaunchKernelGGL(compact_move_kernel, dim3(copy_blocks + table_blocks), dim3(256), 0, st, c, plan, copy_blocks);
    return hipGetLastError();
}
