// Attention of packed windows over a paged cache (dlm_cache_attend).
//
// Rows.  The query heads that share a key head read the same keys, so they are
// packed with the window's rows: row r of (sequence, key head) is window row r /
// G, query head r % G of the group of G.  A workgroup takes up to 128 packed
// rows, 32 per wave, and one run of keys.
//
// Keys.  Tiles of 32 keys go from their pages to LDS by buffer copies that bypass
// registers (staged, XOR-swizzled 16-byte chunks); a page is a scalar, so a
// copy's descriptor is the page itself, cut to the tokens it holds: places behind
// the last token and entries without a page read as zeros, and nothing outside a
// page is ever touched.  64-bit page addresses put no limit on the pool's size.
//
// Products.  Scores are computed transposed, S^T = K Q^T, so a lane owns one row
// (with lane ^ 32): maxima and sums stay in the lane, and the probabilities are
// the B operand of O^T = V^T P^T as they stand.  V stays row-major in its page;
// its transposed fragments come from transposing LDS reads (ds_read_b64_tr_b16:
// 16 lanes hand in 4 rows of 16 values and get a column of 4 each), 4 keys per
// read in the order that the scores' accumulator has them.  Probabilities are
// rounded to the cache's type for the product (the matrix instruction takes
// nothing wider at this rate; half a step, 2^-8 or 2^-11 of each, to either side: see
// kShift for float16's range), sums add the unrounded ones.  Up to 32 packed rows a
// second product adds what the rounding left over: the kernel waits for bytes there
// (64 sequences 81.2 -> 81.7 us, 641 keys of one 7.7 -> 8.2), and the error in bf16 goes
// from 0.0022 to 0.0017 of the result's size, the result's own rounding.  Above that it
// would cost 7 % (13 rows of 4 heads per key head, 97.8 -> 105.0), 6 % (trees, 24.0 ->
// 25.5) and 25 % (prompts, 86.8 -> 108.7).  The running maximum moves only when a tile
// raises it by more than 2^8 (float16: 2^4) in the exp2 domain.
//
// Masks.  Only tiles that meet the window, the last token or a missing page are
// masked, by a 32-bit word per row.  A product with 0 does not hide an infinity
// or a NaN in a value that a row must not see, so masked tiles look for such
// values; where there are any they are taken out of the product and put back, as
// infinities or NaN, into the rows that see them.
//
// Shared prefixes.  Sequences of a group that begin with the same pages have their rows
// packed together against those pages (kPrefix), each sequence's rows against what follows
// (kSuffix), and join_rows_kernel joins what the two left.  share_kernel finds the pages
// from the tables, once for all layers of a pass.  A token of 64 sequences behind 16384
// shared ones, 16 heads of 128 on 4, 16 to 1024 tokens of their own (101 MB, without
// sharing 2.3 GB): 31.5 + 5.8 us a layer, without sharing 139.
//
// Work.  What bounds the kernel depends on the rows: bytes for a few, products
// for many.  Either way the chip is filled by units of at most C steps of keys,
// C such that all sequences' steps make about as many as the chip holds: a long sequence is
// split, short ones are not, whatever the mix.  Only the device knows the
// lengths, so each wave works the list out from them (one scan over the
// sequences).  Split rows leave maximum, sum and unnormalised output in the
// workspace, and a second kernel joins them in order: results do not depend on
// timing.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "cache.h"

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

// Probabilities are held times 2^kShift, relative to the running maximum, which a row's
// scores may pass by up to kHeadroom in the exp2 domain.  float16 keeps half a step only
// down to 2^-14 (2^-25 of absolute error below): with its largest values at 2^15 that is 25
// bits below the maximum, a score 17 lower, and what is lost below that is 2^-36 of the
// maximum's weight per key (2^-16 for a million keys).  Without the factor keys 17 below one
// other count 41 % too much, keys 18 below not at all.  A smaller headroom moves the maximum
// more often: 8 windows of 1024 rows, 16 heads of 128 on 4, f16: 90.7 us, with 7 and 8 (half
// a step kept to 14 below) 88.3, with 13 and 2 93.3; few rows cost the same with any.
template <bool F16>
constexpr int kShift = F16 ? 11 : 0;
template <bool F16>
constexpr int kHeadroom = F16 ? 15 - kShift<F16> : 8;

template <bool F16>
__device__ __forceinline__ f32x16 mfma(const s16x8& a, const s16x8& b, const f32x16& c) {
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
#else
    return c;
#endif
}
// Two floats to a pair of 16-bit values, rounded to nearest even.
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    if constexpr (F16) {
        const uint16_t a = __builtin_bit_cast(uint16_t, (_Float16)lo), b = __builtin_bit_cast(uint16_t, (_Float16)hi);
        return (uint32_t)a | ((uint32_t)b << 16);
    } else {
        return pack_bf16x2(lo, hi);
    }
}
// Whether a 16-bit value is an infinity or a NaN.
template <bool F16>
__device__ __forceinline__ bool is_wild(uint32_t bits16) {
    constexpr uint32_t e = F16 ? 0x7c00u : 0x7f80u;
    return (bits16 & e) == e;
}

template <bool F16>
__device__ __forceinline__ float widen(uint32_t bits16) {
    if constexpr (F16) return (float)__builtin_bit_cast(_Float16, (uint16_t)bits16);
    else return __uint_as_float(bits16 << 16);
}

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
// The pointer is restrict so that the read carries alias information of its own:
// without any, the compiler lets it wait for every copy into LDS in flight, of other
// tiles too (the copies that it needs are awaited by count).
__device__ __forceinline__ s16x4 transposed_read(lds_s16x4* __restrict__ p) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p);
#else
    return s16x4{};
#endif
}
__device__ __forceinline__ s16x4 lds_transpose(lds_ptr_t p) { return transposed_read((lds_s16x4*)p); }

// lds_dma16_buf, past the caches' replacement (ONCE: nobody else reads the bytes).
template <bool ONCE>
__device__ __forceinline__ void copy16(buf_rsrc_t r, uint32_t voffset, lds_ptr_t lds) {
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, lds, 16, (int)voffset, 0, 0, ONCE ? 2 : 0);
#endif
}

template <int CPR>
__device__ __forceinline__ int k_key(int row) {          // of K rows: 32 rows at one chunk hit distinct banks
    if constexpr (CPR == 16) return row & 15;
    else return (row & 7) ^ ((row >> 3) & 1);
}
template <int CPR>
__device__ __forceinline__ int v_key(int row) {          // of V rows: 4 rows at one run of 4 chunks do
    if constexpr (CPR == 16) return (row & 3) << 2;
    else return ((row >> 1) & 1) << 2;
}

// max / sum of v and its value in lane ^ 32
__device__ __forceinline__ float both_max(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
#else
    return v;
#endif
}
__device__ __forceinline__ float both_sum(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
#else
    return v;
#endif
}

// ------------------------------------------------------------------ the list of units

constexpr int kTile = 32;                     // keys of a tile

struct AttnArgs {
    CacheArgs c;
    int64_t layer_base;                       // bytes in front of the layer in each pool
    const int32_t* row_start;
    int total_rows, max_rows, max_keys, group, n_heads;
    const uint16_t* q;
    int64_t q_stride;
    const uint32_t* mask;
    int mask_words;
    float scale_log2, lim;                    // lim: 2^kHeadroom in the exp2 domain, in units of the scores
    uint16_t* o;
    int64_t o_stride;
    float* lse;
    int rows_per_wg;                          // packed rows of a workgroup
    int step;                                 // keys of a step
    int rows_log2, step_log2;                 // both are powers of two
    int min_steps;                            // least steps of a unit
    int units;                                // units aimed at: the workgroups that the chip holds at once
    int max_slots;                            // places for parts; enough for any sound row starts
    float* part_o;                            // [max_slots][rows_per_wg][head_dim]
    float2* part_ml;                          // [max_slots][rows_per_wg]
    // Shared prefixes (kPrefix, kSuffix): what share_kernel wrote, and what is left of rows
    // that are not split, [total_rows][n_heads].
    const int4* groups;                       // [n_seqs]: leader, prefix, first entry of rows, rows
    const int4* members;                      // [n_seqs]: the group's prefix, group, place of its first row in the group
    const int32_t* rows;                      // [total_rows]: the groups' rows
    float* row_o;                             // this launch's (kPrefix; kSuffix behind a prefix)
    float2* row_ml;
    int4* info;                               // [n_seqs]: first slot, parts, row tiles of an item
};

// What a launch attends to: a sequence's keys; the prefix that the sequences of a group
// share, for the rows of all of them; a sequence's keys behind its group's prefix, joined
// with what the prefix left.
enum Mode { kPlain, kPrefix, kSuffix };

struct Seq {
    int n, start, len, keys;                  // rows, first packed row, tokens before, keys in all
    int first;                                // first key, a multiple of a tile
    int table;                                // its table row
};
template <int MODE>
__device__ __forceinline__ Seq sequence(const AttnArgs& a, int b) {
    Seq s{0, 0, 0, 0, 0, b};
    if constexpr (MODE == kPrefix) {
        if (b < a.c.n_seqs) {
            const int4 g = a.groups[b];
            s.table = min(max(g.x, 0), a.c.n_seqs - 1);
            s.start = max(g.z, 0);
            s.n = min(max(g.w, 0), a.max_rows);
            s.len = s.keys = min(max(g.y, 0), a.max_keys) & ~(kTile - 1);     // as kSuffix's first
        }
        return s;
    }
    if (b < a.c.n_seqs) {
        s.start = a.row_start[b];
        const int end = min(a.row_start[b + 1], a.total_rows);
        // compared first: the difference of two unsound starts may pass 32 bits
        s.n = s.start >= 0 && end > s.start ? min(end - s.start, a.max_rows) : 0;
        s.len = max(a.c.len[b], 0);
        s.keys = (int)min((int64_t)s.len + s.n, (int64_t)a.max_keys);
        if constexpr (MODE == kSuffix) s.first = min(max(a.members[b].x, 0), s.keys) & ~(kTile - 1);
    }
    return s;
}
// Packed row of row i of a sequence or a group.
template <int MODE>
__device__ __forceinline__ int64_t packed_row(const AttnArgs& a, const Seq& s, uint32_t i) {
    if constexpr (MODE == kPrefix) {
        const int64_t at = min((int64_t)s.start + i, (int64_t)a.total_rows - 1);
        return min(max(a.rows[at], 0), a.total_rows - 1);
    }
    return (int64_t)s.start + i;
}

// What a wave works out about one unit, or one split item, of the list.
struct Unit {
    Seq s;
    int b, row_tile, kvh;
    int t0, t1;                               // tiles of 32 keys
    int slot, parts;                          // workspace slot of this part; parts of its item
    int tiles;                                // row tiles of its sequence or group
};

// Inclusive prefix sum over the wave by lane moves (a shuffle through LDS each would
// cost a call of few keys more than its products): within rows of 16, then the totals
// of rows 0 and 2 into the next, then of lane 31 into the upper half.
__device__ __forceinline__ int wave_scan(int v) {
#if defined(__HIP_DEVICE_COMPILE__)
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);     // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);     // row_bcast:15
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);     // row_bcast:31
#endif
    return v;
}
// Value of lane l, the same for the whole wave.
__device__ __forceinline__ int from_lane(int v, int l) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_readlane(v, l);
#else
    return v;
#endif
}

// Row tiles and steps of a sequence or a group.
__device__ __forceinline__ void seq_shape(const AttnArgs& a, const Seq& s, int& tiles, int& steps) {
    tiles = (s.n * a.group + a.rows_per_wg - 1) >> a.rows_log2;
    steps = max((s.keys - s.first + a.step - 1) >> a.step_log2, 1);
}

// The index-th unit (or, with `items`, the index-th item of several parts) in the
// order sequence, key head, part, row tile; false if there are fewer.  A lane
// looks after a sequence, 64 at a time.  given: most steps of a unit (0: worked out here).
template <bool ITEMS, int MODE>
__device__ __forceinline__ bool find_unit(const AttnArgs& a, int index, Unit& u, int given = 0) {
    const int lane = threadIdx.x & 63;
    auto shape = [&](const Seq& s, int& tiles, int& steps) { seq_shape(a, s, tiles, steps); };
    const Seq first = sequence<MODE>(a, lane);
    // Steps of all items: float32, since row starts that overlap may make more of them
    // than an int holds, and what follows needs no more than its bound (max_slots).
    float sum = 0.f;
    int items = 0;
    for (int b0 = 0; given == 0 && b0 < a.c.n_seqs; b0 += 64) {
        int tiles, steps;
        shape(b0 ? sequence<MODE>(a, b0 + lane) : first, tiles, steps);
        sum += wave_sum_dpp((float)tiles * (float)steps * (float)a.c.n_kv);
        items += from_lane(wave_scan(tiles * a.c.n_kv), 63);
    }
    // Cut into runs of sum / n steps an item's last one is half empty on average, so
    // this aims at `units` of them together.
    const int n = max(a.units - items / 2, a.units / 2);
    const int most = given ? given : max(a.min_steps, (int)fminf(ceilf(sum / (float)n), 0x1p30f));
    int before = 0, slots_before = 0;
    for (int b0 = 0; b0 < a.c.n_seqs; b0 += 64) {
        int tiles, steps;
        const Seq s = b0 ? sequence<MODE>(a, b0 + lane) : first;
        shape(s, tiles, steps);
        const int parts = (int)((uint32_t)(steps + most - 1) / (uint32_t)most);
        const int all = tiles * a.c.n_kv * parts, split = parts > 1 ? all : 0;
        const int count = ITEMS ? (parts > 1 ? tiles * a.c.n_kv : 0) : all;
        const int end = before + wave_scan(count), slot_end = slots_before + wave_scan(split);
        const uint64_t hit = __ballot(index < end && index >= end - count);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            u.b = uniform(b0 + l);
            u.s.n = from_lane(s.n, l);
            u.s.start = from_lane(s.start, l);
            u.s.len = from_lane(s.len, l);
            u.s.keys = from_lane(s.keys, l);
            u.s.first = MODE == kSuffix ? from_lane(s.first, l) : 0;
            u.s.table = MODE == kPrefix ? from_lane(s.table, l) : u.b;
            u.parts = from_lane(parts, l);
            const int n_tiles = from_lane(tiles, l);
            const int all_steps = from_lane(steps, l);
            uint32_t i = (uint32_t)(index - from_lane(end - count, l));
            const int slot0 = from_lane(slot_end - split, l);
            u.tiles = n_tiles;
            u.row_tile = uniform((int)(i % (uint32_t)n_tiles));
            i /= (uint32_t)n_tiles;
            int part = 0;
            if (!ITEMS) {
                part = uniform((int)(i % (uint32_t)u.parts));
                i /= (uint32_t)u.parts;
            }
            u.kvh = uniform((int)i);
            // slots of an item's parts lie next to each other
            u.slot = slot0 + (u.kvh * n_tiles + u.row_tile) * u.parts + part;
            const int each = (int)((uint32_t)(all_steps + u.parts - 1) / (uint32_t)u.parts) << (a.step_log2 - 5);
            u.t0 = uniform((MODE == kSuffix ? u.s.first / kTile : 0) + part * each);
            u.t1 = uniform(min(u.t0 + each, (u.s.keys + kTile - 1) / kTile));
            return u.parts == 1 || u.slot + u.parts - part <= a.max_slots;
        }
        before = from_lane(end, 63);
        slots_before = from_lane(slot_end, 63);
    }
    return false;
}

// Prefixes and own keys in one launch: units of about as many keys each, so many that all of
// them together make what the chip holds at once (a tile of keys costs a workgroup about as
// much against 128 rows, by its products, as against a few, by its bytes).
struct Balance {
    int most_pre, most_own, pre_units;
};
__device__ __forceinline__ Balance balance(const AttnArgs& pre, const AttnArgs& own) {
    const int lane = threadIdx.x & 63;
    float keys = 0.f;
    int items = 0;
    for (int b0 = 0; b0 < own.c.n_seqs; b0 += 64) {
        const Seq p = sequence<kPrefix>(pre, b0 + lane), s = sequence<kSuffix>(own, b0 + lane);
        int tp, ts, steps;
        seq_shape(pre, p, tp, steps);
        seq_shape(own, s, ts, steps);
        keys += wave_sum_dpp(((float)tp * (float)p.keys + (float)ts * (float)(s.keys - s.first)) * (float)own.c.n_kv);
        items += from_lane(wave_scan((tp + ts) * own.c.n_kv), 63);
    }
    const int n = max(own.units - items / 2, own.units / 2);
    const float each = keys / (float)n;
    Balance r{max(pre.min_steps, (int)fminf(ceilf(each / (float)pre.step), 0x1p30f)),
              max(own.min_steps, (int)fminf(ceilf(each / (float)own.step), 0x1p30f)), 0};
    for (int b0 = 0; b0 < own.c.n_seqs; b0 += 64) {
        int tiles, steps;
        seq_shape(pre, sequence<kPrefix>(pre, b0 + lane), tiles, steps);
        const int parts = (int)((uint32_t)(steps + r.most_pre - 1) / (uint32_t)r.most_pre);
        r.pre_units += from_lane(wave_scan(tiles * pre.c.n_kv * parts), 63);
    }
    return r;
}

// Where join_rows_kernel finds the parts of a sequence or a group, from its first unit.
template <int MODE>
__device__ __forceinline__ void note_item(const AttnArgs& a, const Unit& u) {
    if constexpr (MODE != kPlain)
        if (threadIdx.x == 0 && u.row_tile == 0 && u.kvh == 0 && u.t0 == u.s.first / kTile) a.info[u.b] = int4{u.slot, u.parts, u.tiles, 0};
}
// A row's maximum, sum and output taken together with another part's.
struct Two {
    float m, f0, f1;
};
__device__ __forceinline__ Two together(const AttnArgs& a, float m0, float m1) {
    const float m = fmaxf(m0, m1);
    return {m, m0 == m ? 1.f : __builtin_amdgcn_exp2f((m0 - m) * a.scale_log2),
            m1 == m ? 1.f : __builtin_amdgcn_exp2f((m1 - m) * a.scale_log2)};
}

// ------------------------------------------------------------------ tiles

template <int HD>
struct Dims {
    static constexpr int CPR = HD / 8;                    // 16-byte chunks of a row
    static constexpr int ROW = HD * 2;
    static constexpr int HALF = kTile * ROW;              // bytes of a K or V tile
    static constexpr int NB = HD / 32, NKS = HD / 16;     // 32-feature blocks; 16-feature steps
    static constexpr int ROWS_PER_COPY = 64 / CPR;        // rows of a 1 KB copy
};

// Where the keys of one (sequence, key head) lie.  Everything here is scalar but the
// table entries, of which lane i keeps number base + i: a tile's come from there by a
// lane index, without a load in front of its copies.
template <int HD>
struct Keys {
    const char *k, *v;
    const int32_t* table;
    uint32_t page_bytes;
    int keys, n_pages, max_pages, page_log2, page_mask, base, held;
    int gaps = 0;                                         // some entry so far that has tokens has no page

    __device__ __forceinline__ Keys(const AttnArgs& a, const Unit& u) {
        const uint32_t head = (uint32_t)a.c.page_len * Dims<HD>::ROW;
        k = a.c.k + a.layer_base + (int64_t)u.kvh * head;
        v = a.c.v + a.layer_base + (int64_t)u.kvh * head;
        page_bytes = head * a.c.n_kv;                     // at most 4 MB
        table = a.c.table + (int64_t)u.s.table * a.c.max_pages;
        keys = u.s.keys;
        n_pages = a.c.n_pages;
        max_pages = a.c.max_pages;
        page_log2 = a.c.page_log2;
        page_mask = a.c.page_len - 1;
        fetch((u.t0 * kTile) >> page_log2);
    }
    // Entries past the row's end are read as its last one, whose keys then lie behind
    // the last token.
    __device__ __forceinline__ void fetch(int first) {
        base = first;
        held = table[min(first + (int)(threadIdx.x & 63), max_pages - 1)];
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" : "+v"(held));                    // waited for here, not wherever it is used
#endif
        const int e = first + (int)(threadIdx.x & 63);
        const uint64_t none = __ballot((int64_t)e << page_log2 < keys && !is_page(held));
        gaps = uniform(gaps | (int)((uint32_t)none | (uint32_t)(none >> 32)));
    }
    // Entries of the two groups of 16 keys of a tile, or of one of them.
    __device__ __forceinline__ void need(int kt) {
        const int e0 = (kt * kTile) >> page_log2;
        if (__builtin_expect((uint32_t)(e0 - base) > 62u, 0)) fetch(e0);
    }
    __device__ __forceinline__ int entry(int kt, int s) {
        need(kt);
        return from_lane(held, ((kt * kTile + s * 16) >> page_log2) - base);
    }
    __device__ __forceinline__ int2 entries(int kt) {
        need(kt);
        return int2{from_lane(held, ((kt * kTile) >> page_log2) - base),
                    from_lane(held, ((kt * kTile + 16) >> page_log2) - base)};
    }
    __device__ __forceinline__ bool is_page(int page) const { return (uint32_t)page < (uint32_t)n_pages; }
    // Bit s: group s of the tile has no page.
    __device__ __forceinline__ uint32_t missing(const int2& e) const {
        return (is_page(e.x) ? 0u : 1u) | (is_page(e.y) ? 0u : 2u);
    }
    // Byte offset in the pools, and bytes that hold tokens, of the 16 keys of group s.
    __device__ __forceinline__ int64_t offset(int page, int kt, int s) const {
        return (int64_t)((uint64_t)(uint32_t)(is_page(page) ? page : 0) * page_bytes) +
               ((kt * kTile + s * 16) & page_mask) * Dims<HD>::ROW;
    }
    __device__ __forceinline__ int bytes(int page, int kt, int s) const {
        const int g = kt * 2 + s, full = keys >> 4;
        const int n = g < full ? 16 : g == full ? keys & 15 : 0;
        return is_page(page) ? n * Dims<HD>::ROW : 0;
    }
};

// Word w of a row's mask (0 outside of it).  Scalar w: a branch.
__device__ __forceinline__ uint32_t mask_word(const AttnArgs& a, const uint32_t* mask_row, int w) {
    return w >= 0 && w < a.mask_words ? mask_row[w] : 0;
}
// Which keys of the tile from k0 on a row sees; lo, hi: words (k0 - len) / 32, rounded
// down, and the next one of its mask.
__device__ __forceinline__ uint32_t seen_keys(const AttnArgs& a, const Seq& s, uint32_t lo, uint32_t hi, int k0,
                                              uint32_t gone) {
    uint32_t see = 0xffffffffu;
    if (a.mask) {
        const int rel = k0 - s.len, sh = rel & 31;        // first key's place in the window
        see = sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
        if (rel < 0) see |= rel <= -32 ? 0xffffffffu : (1u << -rel) - 1;      // tokens before the window
    }
    const int left = s.keys - k0;
    if (left < 32) see &= left <= 0 ? 0 : (1u << left) - 1;
    if (gone & 1) see &= 0xffff0000u;
    if (gone & 2) see &= 0x0000ffffu;
    return see;
}

// 32 rows: lane (j, g) holds row j, keys 8 (e / 4) + 4 g + e % 4 of a tile's scores
// and features 32 n + 8 (e / 4) + 4 g + e % 4 of the output.
template <bool F16, int HD>
struct RowTile {
    using D = Dims<HD>;
    f32x16 o[D::NB];
    float m, l, bias;                                     // m in units of the scores; bias: -m scale_log2

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < D::NB; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[n][e] = 0.f;
        m = -INFINITY;
        l = bias = 0.f;
    }
    __device__ __forceinline__ static void hide(f32x16& st, uint32_t see, int g) {
        see >>= 4 * g;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (!((see >> (8 * (e >> 2) + (e & 3))) & 1)) st[e] = -INFINITY;
    }
    // Scores to probabilities (times 2^kShift), the B operand of O^T = V^T P^T: rounded,
    // and, of two TERMS, what the rounding left over.
    // `lim`: how far, in units of the scores, a maximum may lie above m.
    template <int TERMS>
    __device__ __forceinline__ void softmax(const f32x16& st, float scale_log2, float lim, s16x8 (&pf)[TERMS][2]) {
        float mt = st[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mt = fmaxf(mt, st[e]);
        mt = both_max(mt);
        // Each row by its own scores alone, so that its bits do not depend on others'.
        const bool move = mt - m > lim;                   // not if both are -inf
        if (__any(move)) {
            const float m_new = move ? mt : m;
            const float alpha = move ? __builtin_amdgcn_exp2f((m - m_new) * scale_log2) : 1.f;
            l *= alpha;
#pragma unroll
            for (int n = 0; n < D::NB; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[n][e] *= alpha;
            m = m_new;
            bias = m == -INFINITY ? 0.f : fmaf(-m, scale_log2, (float)kShift<F16>);
        }
        float sum = 0.f;
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
            u32x4 w, rest;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(st[8 * s2 + 2 * i], scale_log2, bias));
                const float p1 = __builtin_amdgcn_exp2f(fmaf(st[8 * s2 + 2 * i + 1], scale_log2, bias));
                sum += p0 + p1;
                w[i] = pack2<F16>(p0, p1);
                if constexpr (TERMS == 2)
                    rest[i] = pack2<F16>(p0 - widen<F16>(w[i] & 0xffffu), p1 - widen<F16>(w[i] >> 16));
            }
            pf[0][s2] = __builtin_bit_cast(s16x8, w);
            if constexpr (TERMS == 2) pf[1][s2] = __builtin_bit_cast(s16x8, rest);
        }
        l += sum;
    }
};

// LDS byte addresses of V fragments of a tile.  A stage starts at a multiple of a row
// and a chunk's number is the only thing in the address bits that it takes up, so the
// n-th four chunks are one base with a constant xor-ed in.  Transposing reads: lane i
// of 16 hands in 4 values of row i / 4; rows 8 apart have the same key.
template <int HD>
__device__ __forceinline__ int v_base(int lane) {
    const int row = 4 * (lane >> 5) + ((lane & 15) >> 2);
    return row * Dims<HD>::ROW + (lane & 1) * 8 +
           (((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ v_key<Dims<HD>::CPR>(row)) << 4);
}

// V^T fragments of two 32-feature blocks (n2, n2 + 1) of a tile; va: LDS byte address of
// its V rows plus v_base.
template <int HD>
__device__ __forceinline__ void read_values(s16x8 (&vf)[2][2], lds_ptr_t lds, int va, int n2) {
    using D = Dims<HD>;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
            const int at = (va ^ ((n2 + n) << 6)) + 16 * s2 * D::ROW;
            const s16x4 lo = lds_transpose((lds_ptr_t)((lds_char*)lds + at));
            const s16x4 hi = lds_transpose((lds_ptr_t)((lds_char*)lds + at + 8 * D::ROW));
            vf[n][s2] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
}

// O^T += V^T P^T of RT row tiles; v: LDS byte address of the V tile, vf: its first
// fragments (asked for before the softmax, which hides their latency).  `masked`: some
// row does not see all of it, so that infinities and NaN are looked for and, if there
// are any (the result), left out.  One path with scalar branches: two copies of the
// products would hold the accumulators twice.
template <bool F16, int HD, int RT, int TERMS>
__device__ __forceinline__ bool add_values(RowTile<F16, HD> (&rt)[RT], const s16x8 (&pf)[RT][TERMS][2], s16x8 (&vf)[2][2],
                                           lds_ptr_t lds, int v, int lane, int base, bool masked) {
    using D = Dims<HD>;
    const int g = lane >> 5, j = lane & 31;
    uint32_t wild = 0;                                    // keys with an infinity or NaN
    if (__builtin_expect(masked, 0)) {
        uint32_t hi = 0, lo = 0;                          // largest magnitudes among a key's values
#pragma unroll
        for (int x = 0; x < D::CPR / 2; ++x) {
            // a row's chunks in an order of its own: rows lie a multiple of all banks apart
            const u32x4 w = *(__attribute__((address_space(3))) const u32x4*)((lds_char*)lds + v + j * D::ROW +
                                                                             (g * (D::CPR / 2) + (x ^ (j & (D::CPR / 2 - 1)))) * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                hi = max(hi, w[i] & 0x7fffffffu);
                lo = max(lo, (w[i] << 16) & 0x7fffffffu);
            }
            if (x % 2) sched_fence();                     // few registers at a time
        }
        const uint64_t votes = __ballot(is_wild<F16>(max(hi, lo) >> 16));
        wild = uniform((int)((uint32_t)votes | (uint32_t)(votes >> 32)));
    }
#pragma unroll
    for (int n2 = 0; n2 < D::NB; n2 += 2) {
        if (n2) {
            read_values<HD>(vf, lds, v + base, n2);
            sched_fence();
        }
        if (__builtin_expect(wild, 0)) {                  // finite values only
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const short y = vf[x >> 1][x & 1][i];
                    vf[x >> 1][x & 1][i] = is_wild<F16>((uint16_t)y) ? (short)0 : y;
                }
        }
#pragma unroll
        for (int x = 0; x < 2 * TERMS; ++x)               // 16 keys, then the terms
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    rt[r].o[n2 + n] = mfma<F16>(vf[n][x / TERMS], pf[r][x % TERMS][x / TERMS], rt[r].o[n2 + n]);
    }
    return wild != 0;
}

// Rare: the infinities and NaN that add_values left out, whatever their probability,
// into the rows that see their keys; straight from the pages, once, after the last
// tile.  Tiles first, first + step, ... below end; `clear`: keys that every row sees.
template <bool F16, int HD, int RT>
__device__ __forceinline__ void add_wild(RowTile<F16, HD> (&rt)[RT], const AttnArgs& a, const Unit& u, Keys<HD>& keys,
                                         const uint32_t* const (&mrow)[RT], int first, int end, int step, int clear, int g) {
    using D = Dims<HD>;
#pragma unroll 1
    for (int kt = first; kt < end; kt += step) {
        const int2 e = keys.entries(kt);
        const uint32_t gone = keys.missing(e);
        if (kt * kTile + kTile <= clear && !gone) continue;
        uint32_t see[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int w = (kt * kTile - u.s.len) >> 5;
            see[r] = seen_keys(a, u.s, a.mask ? mask_word(a, mrow[r], w) : 0, a.mask ? mask_word(a, mrow[r], w + 1) : 0,
                               kt * kTile, gone);
        }
#pragma unroll 1
        for (int i = 0; i < kTile; ++i) {
            if ((gone >> (i >> 4)) & 1 || kt * kTile + i >= keys.keys) continue;
            const char* row = keys.v + keys.offset(i < 16 ? e.x : e.y, kt, i >> 4) + (i & 15) * D::ROW + 8 * g;
#pragma unroll
            for (int n = 0; n < D::NB; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const u32x2 w = *reinterpret_cast<const u32x2*>(row + (n * 32 + 8 * q) * 2);
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const uint32_t bits = (x & 1 ? w[x >> 1] >> 16 : w[x >> 1]) & 0xffffu;
#pragma unroll
                        for (int r = 0; r < RT; ++r)
                            if (((see[r] >> i) & 1) && is_wild<F16>(bits)) rt[r].o[n][4 * q + x] += widen<F16>(bits);
                    }
                    sched_fence();
                }
        }
    }
}

// Four features of a finished row.
template <bool F16>
__device__ __forceinline__ void store_out(const AttnArgs& a, int64_t t, int head, int feature, int hd, const f32x4& v,
                                          float inv) {
    const u32x2 w = {pack2<F16>(v[0] * inv, v[1] * inv), pack2<F16>(v[2] * inv, v[3] * inv)};
    *reinterpret_cast<u32x2*>(a.o + t * a.o_stride + head * hd + feature) = w;
}
template <bool F16>
__device__ __forceinline__ float log_sum(const AttnArgs& a, float m, float l) {
    return l == 0.f ? -INFINITY : fmaf(m, a.scale_log2, __builtin_amdgcn_logf(l) - (float)kShift<F16>) * 0.69314718f;
}

// ------------------------------------------------------------------ many rows

// More than 64 packed rows: 4 waves of 32 rows share tiles of K and V in LDS, three
// stages of them, copied by all.  WK = 1: 168 VGPRs at head_dim 128, so three
// workgroups (12 waves) share a CU, 50 KB of LDS each.  WK = 2, for calls with too few
// rows to fill the chip: two such groups of waves take tiles in turn and add up in the
// end, half the steps and half the parts to join for the same split.
// A tile is 16 matrix and about 90 other vector instructions per wave; on long windows
// the matrix cores are busy 59 % of the cycles and the clock falls to 1.7 - 1.9 GHz, so
// what bounds it is the card's power as much as the cycles (two tiles per step, 15 %
// fewer instructions: no faster).  16 heads of 128 on 4, windows that see themselves:
// 8 x 1024 rows 80 us (860 TFLOP/s; 8 us of it start and end), 4 x 4096 rows 534 to 570
// us by the box (965 to 1030).
constexpr int kManyRows = 128, kManyStages = 3;

// A K tile of these kernels: 64 bytes of space behind each 1 KB copy turn its rows by
// a quarter of the banks against the next copy's, so that only two address bits are
// left to xor (a row's place within a copy): fragments four chunks apart differ by a
// constant, which is the read's offset.
constexpr int kCopyStep = 1024 + 64;
template <int HD>
__device__ __forceinline__ int k_turn(int row) {          // of a chunk's number
    return HD == 128 ? row & 3 : (row >> 1) & 3;
}

// LDS of a workgroup.
template <int HD, int WK>
constexpr int kManyLds = WK * kManyStages * (kTile / Dims<HD>::ROWS_PER_COPY * kCopyStep + Dims<HD>::HALF);

// Workgroup `wg` of a launch.  smem: the kernel's only LDS variable: with a second one the
// compiler tells the two apart, takes a fragment read to depend on every copy in flight into
// this one, and waits for them all.
template <bool F16, int HD, bool ONCE, int WK, int MODE, int TERMS = 1>
__device__ __forceinline__ void attend_many(const AttnArgs& a, int wg, char* smem, int given = 0) {
    using D = Dims<HD>;
    constexpr int K_TILE = kTile / D::ROWS_PER_COPY * kCopyStep;
    constexpr int NS = kManyStages, STAGE = K_TILE + D::HALF;
    constexpr int COPIES = D::HALF / 1024 / 4;            // 1 KB copies per wave of a K or V tile

    const int tid = threadIdx.x, lane = tid & 63, wave = uniform((tid >> 6) & 3), wk = uniform(tid >> 8);
    const int g = lane >> 5, j = lane & 31;
    Unit u;
    if (!find_unit<false, MODE>(a, wg, u, given)) return;
    note_item<MODE>(a, u);
    const int rows = min(u.s.n * a.group - u.row_tile * kManyRows, kManyRows);           // of this workgroup
    const bool busy = wave * 32 < rows;                   // this wave has rows
    const int r = min(wave * 32 + j, rows - 1) + u.row_tile * kManyRows;
    const int head = u.kvh * a.group + (int)((uint32_t)r % (uint32_t)a.group);
    const int64_t t = packed_row<MODE>(a, u.s, (uint32_t)r / (uint32_t)a.group);
    Keys<HD> keys(a, u);

    // Copies: lane L of copy p reads the chunk that belongs at byte 16 L of its 1 KB
    // block; a wave's blocks of a tile lie within one group of 16 keys.
    uint32_t k_off[COPIES], v_off[COPIES];
#pragma unroll
    for (int p = 0; p < COPIES; ++p) {
        const int row = (wave * COPIES + p) * D::ROWS_PER_COPY + lane / D::CPR, pc = lane % D::CPR;
        k_off[p] = (uint32_t)((row & 15) * D::ROW + ((pc ^ k_turn<HD>(row)) << 4));
        v_off[p] = (uint32_t)((row & 15) * D::ROW + ((pc ^ v_key<D::CPR>(row)) << 4));
    }
    const lds_ptr_t lds = (lds_ptr_t)smem;
    const int sub = wave * COPIES * D::ROWS_PER_COPY / 16;
    auto issue = [&](int kt, int at_lds) {                // at_lds: the stage
        const int page = keys.entry(kt, sub), bytes = keys.bytes(page, kt, sub);
        const int64_t at = keys.offset(page, kt, sub);
        const buf_rsrc_t kr = make_rsrc(keys.k + at, bytes), vr = make_rsrc(keys.v + at, bytes);
        lds_char* kd = (lds_char*)lds + at_lds + wave * COPIES * kCopyStep;
        lds_char* vd = (lds_char*)lds + at_lds + K_TILE + wave * COPIES * 1024;
#pragma unroll
        for (int p = 0; p < COPIES; ++p) copy16<ONCE>(kr, k_off[p], (lds_ptr_t)(kd + p * kCopyStep));
#pragma unroll
        for (int p = 0; p < COPIES; ++p) copy16<ONCE>(vr, v_off[p], (lds_ptr_t)(vd + p * 1024));
    };

    s16x8 qf[D::NKS];
    {
        const uint16_t* qp = a.q + t * a.q_stride + head * HD + g * 8;
#pragma unroll
        for (int ks = 0; ks < D::NKS; ++ks) qf[ks] = *reinterpret_cast<const s16x8*>(qp + ks * 16);
    }
    RowTile<F16, HD> rt[1];
    rt[0].clear();
    // K fragments: chunk 2 ks + g of row j, by the parity of ks.
    const int krow = j / D::ROWS_PER_COPY * kCopyStep + j % D::ROWS_PER_COPY * D::ROW;
    const int kfrag[2] = {krow + ((g ^ k_turn<HD>(j)) << 4), krow + (((2 + g) ^ k_turn<HD>(j)) << 4)};
    const int vfrag = v_base<HD>(lane);
    const uint32_t* mrow = a.mask ? a.mask + t * a.mask_words : nullptr;
    const int clear = a.mask ? min(u.s.len, u.s.keys) : u.s.keys;         // keys that every row sees

    // Tiles u.t0 + wk + WK i, i < n, the same n for all waves (they meet at every one):
    // copies past the last tile repeat it, and a step on it is one that no row sees.
    const int n = (u.t1 - u.t0 + WK - 1) / WK;
    auto tile_at = [&](int i) { return min(u.t0 + wk + i * WK, u.t1 - 1); };
    bool wild = false;
    if (n > 0) {
        int use = wk * NS * STAGE, then = use + STAGE, put = then + STAGE;    // the stages, in turn
        static_assert(NS == 3, "two tiles in flight beside the one at work");
        // Words of the row's mask for a tile, where it meets the window.
        uint32_t lo = 0, hi = 0;
        auto words = [&](int kt) {
            if (__builtin_expect(kt * kTile + kTile > clear, 0)) {
                const int w = (kt * kTile - u.s.len) >> 5;
                lo = mask_word(a, mrow, w);
                hi = mask_word(a, mrow, w + 1);
            }
        };
        words(tile_at(0));
        issue(tile_at(0), use);
        issue(tile_at(1), then);
        // The queries' and the words' loads end here and not inside the loop, where
        // their wait would take the copies in flight with it.
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" : "+v"(lo), "+v"(hi));
#pragma unroll
        for (int ks = 0; ks < D::NKS; ++ks) asm volatile("" ::"v"(qf[ks]));
#endif
        for (int i = 0; i < n; ++i) {
            wait_vmcnt<(NS - 2) * 2 * COPIES>();          // this wave's copies of the tile have landed
            lds_barrier();                                // everyone's have; the stage before is free
            issue(tile_at(i + NS - 1), put);
            const int sb = use;
            use = then;
            then = put;
            put = sb;
            if (!busy) continue;
            const int kt = u.t0 + wk + i * WK, k0 = kt * kTile;
            int gone = kt < u.t1 ? 0 : 3;                 // groups that no row sees
            if (__builtin_expect(keys.gaps, 0)) gone |= (int)keys.missing(keys.entries(min(kt, u.t1 - 1)));
            const int masked = ((clear - k0 - kTile) >> 31) | gone;

            f32x16 st;
#pragma unroll
            for (int e = 0; e < 16; ++e) st[e] = 0.f;
            lds_char* ka[2] = {(lds_char*)lds + sb + kfrag[0], (lds_char*)lds + sb + kfrag[1]};
#pragma unroll
            for (int k4 = 0; k4 < D::NKS; k4 += 4) {
                s16x8 kf[4];
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    kf[x] = *(__attribute__((address_space(3))) const s16x8*)(ka[x & 1] + ((k4 + x) >> 1) * 64);
                sched_fence();
#pragma unroll
                for (int x = 0; x < 4; ++x) st = mfma<F16>(kf[x], qf[k4 + x], st);
            }
            s16x8 vf[2][2];
            read_values<HD>(vf, lds, sb + K_TILE + vfrag, 0);
            sched_fence();
            if (__builtin_expect(masked, 0)) rt[0].hide(st, seen_keys(a, u.s, lo, hi, k0, (uint32_t)gone), g);
            if (a.mask) words(tile_at(i + 1));
            s16x8 pf[1][TERMS][2];
            rt[0].softmax(st, a.scale_log2, a.lim, pf[0]);
            wild |= add_values<F16, HD, 1, TERMS>(rt, pf, vf, lds, sb + K_TILE, lane, vfrag, masked);
        }
    }

    wait_all_memory();                                    // no copy may still land in LDS
    if (__builtin_expect(wild, 0)) add_wild<F16, HD, 1>(rt, a, u, keys, {mrow}, u.t0 + wk, u.t1, WK, clear, g);
    f32x16* o = rt[0].o;
    float l = both_sum(rt[0].l), m = rt[0].m;
    const int row = wave * 32 + j;
    if constexpr (WK == 2) {
        // The second group's outputs through LDS, lane by lane: both hold the same rows
        // and features in the same registers.
        static_assert(4 * (D::NB * 16 + 2) * 64 * 4 <= WK * NS * STAGE, "the outputs fit the stages");
        float* slot = reinterpret_cast<float*>(smem) + wave * ((D::NB * 16 + 2) * 64) + lane;
        __syncthreads();
        if (wk == 1) {
#pragma unroll
            for (int nb = 0; nb < D::NB; ++nb)
#pragma unroll
                for (int e = 0; e < 16; ++e) slot[(nb * 16 + e) * 64] = o[nb][e];
            slot[D::NB * 16 * 64] = m;
            slot[(D::NB * 16 + 1) * 64] = l;
        }
        __syncthreads();
        if (wk == 1) return;
        const float m1 = slot[D::NB * 16 * 64], l1 = slot[(D::NB * 16 + 1) * 64];
        const float mn = fmaxf(m, m1);
        const float f0 = m == mn ? 1.f : __builtin_amdgcn_exp2f((m - mn) * a.scale_log2);
        const float f1 = m1 == mn ? 1.f : __builtin_amdgcn_exp2f((m1 - mn) * a.scale_log2);
#pragma unroll
        for (int nb = 0; nb < D::NB; ++nb)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[nb][e] = o[nb][e] * f0 + slot[(nb * 16 + e) * 64] * f1;
        l = l * f0 + l1 * f1;
        m = mn;
    }
    if (!busy) return;
    const bool split = u.parts > 1;
    if (split || MODE == kPrefix || (MODE == kSuffix && u.s.first > 0)) {                       // what is left of a row until its parts are joined
        if (row < rows) {
            const int64_t at = split ? (int64_t)u.slot * kManyRows + row : t * a.n_heads + head;
            float* p = (split ? a.part_o : a.row_o) + at * HD + 4 * g;
#pragma unroll
            for (int nb = 0; nb < D::NB; ++nb)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<f32x4*>(p + nb * 32 + 8 * e) =
                        f32x4{o[nb][4 * e], o[nb][4 * e + 1], o[nb][4 * e + 2], o[nb][4 * e + 3]};
            if (g == 0) (split ? a.part_ml : a.row_ml)[at] = float2{m, l};
        }
        return;
    }
    // Rows that saw nothing: the sum is 0 and so is every product.
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* orow = a.o + t * a.o_stride + head * HD;
#pragma unroll
    for (int nb = 0; nb < D::NB; ++nb) {
        uint32_t p[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i][0] = pack2<F16>(o[nb][4 * i] * inv, o[nb][4 * i + 1] * inv);
            p[i][1] = pack2<F16>(o[nb][4 * i + 2] * inv, o[nb][4 * i + 3] * inv);
        }
        swap_halves16(p);
        if (row < rows) {
            uint16_t* dst = orow + nb * 32 + 16 * g;
            *reinterpret_cast<u32x4*>(dst) = u32x4{p[0][0], p[0][1], p[2][0], p[2][1]};
            *reinterpret_cast<u32x4*>(dst + 8) = u32x4{p[1][0], p[1][1], p[3][0], p[3][1]};
        }
    }
    if (a.lse && g == 0 && row < rows) a.lse[t * a.n_heads + head] = log_sum<F16>(a, m, l);
}

// Neighbouring units share their keys (row tiles): workgroups go to the 8 XCDs in turn, so
// each XCD takes runs of 8 units.
__device__ __forceinline__ int xcd_order(int wg) { return (wg & ~63) + (wg & 7) * 8 + ((wg >> 3) & 7); }

template <bool F16, int HD, bool ONCE, int WK, int MODE>
__global__ __launch_bounds__(256 * WK) __attribute__((amdgpu_waves_per_eu(WK == 1 ? 3 : 2))) void
attend_many_kernel(const AttnArgs a) {
    __shared__ __attribute__((aligned(16))) char smem[kManyLds<HD, WK>];
    attend_many<F16, HD, ONCE, WK, MODE>(a, xcd_order(blockIdx.x), smem);
}

// ------------------------------------------------------------------ few rows

// Up to 64 packed rows (RT row tiles per wave): bound by the bytes of K and V, each
// read once, so what counts is how many are in flight.  Every wave takes tiles of its
// own (every WAVES-th of the unit), without barriers, through S stages of its own:
// keys of the next tile are asked for as soon as the products with this one's have
// read them, and values likewise.  Up to 32 rows: one stage, so that a workgroup's 64
// KB (66 with the join's sums) leave room for a second one, which works while the first
// starts or ends; 64 rows hold twice the accumulators (420 VGPRs, one wave per SIMD):
// two stages.  All of the 128 KB per CU are in flight but for the tiles at work.
// 64 sequences of 256 to 16384 tokens, a row each, 16 heads of 128 on 4 (472 MB): 82 us,
// 5.8 TB/s; 13 rows of 32 heads on 8 behind 131072 tokens (537 MB): 92 us, 5.8 TB/s; 641
// keys of 64: 8.2 us, of which 5.3 are there for a single key (a launch, four loads that
// need each other, the end).
constexpr int kFewWaves = 4;
template <int HD, int RT, int S>
struct FewLds {
    static constexpr int RING = 2 * S * Dims<HD>::HALF;   // a wave's stages: S tiles of K, then of V
    static constexpr int OUT = 32 * RT * HD * 4;          // a wave's outputs in the end, then maxima and sums
    static constexpr int OWN = RING > OUT + 32 * RT * 8 ? RING : OUT + 32 * RT * 8;
    static constexpr int ALL = kFewWaves * OWN;
};

template <bool F16, int HD, int RT, int S, int MODE>
__device__ __forceinline__ void attend_few(const AttnArgs& a, int wg, char* smem, int given = 0) {
    using D = Dims<HD>;
    constexpr int WAVES = kFewWaves, TERMS = RT == 1 ? 2 : 1;
    constexpr int COPIES = D::HALF / 1024;                // 1 KB copies of a V tile
    constexpr int C4 = HD / 4;
    constexpr int OUT = FewLds<HD, RT, S>::OUT, OWN = FewLds<HD, RT, S>::OWN;

    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int g = lane >> 5, j = lane & 31;
    Unit u;
    if (!find_unit<false, MODE>(a, wg, u, given)) return;
    note_item<MODE>(a, u);
    const int rows = u.s.n * a.group;                     // one row tile: all rows of (sequence, key head)
    Keys<HD> keys(a, u);
    const lds_ptr_t lds = (lds_ptr_t)smem;
    const int ring = wave * OWN;

    s16x8 qf[RT][D::NKS];
    const uint32_t* mrow[RT];
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const int r = min(x * 32 + j, rows - 1);
        const int64_t t = packed_row<MODE>(a, u.s, (uint32_t)r / (uint32_t)a.group);
        const uint16_t* qp = a.q + t * a.q_stride + (u.kvh * a.group + (int)((uint32_t)r % (uint32_t)a.group)) * HD + g * 8;
#pragma unroll
        for (int ks = 0; ks < D::NKS; ++ks) qf[x][ks] = *reinterpret_cast<const s16x8*>(qp + ks * 16);
        mrow[x] = a.mask ? a.mask + t * a.mask_words : nullptr;
    }
    uint32_t k_off[COPIES], v_off[COPIES];                // within a group of 16 keys, as above
#pragma unroll
    for (int p = 0; p < COPIES; ++p) {
        const int row = p * D::ROWS_PER_COPY + lane / D::CPR, pc = lane % D::CPR;
        k_off[p] = (uint32_t)((row & 15) * D::ROW + ((pc ^ k_key<D::CPR>(row)) << 4));
        v_off[p] = (uint32_t)((row & 15) * D::ROW + ((pc ^ v_key<D::CPR>(row)) << 4));
    }
    auto issue = [&](const char* pool, const uint32_t (&off)[COPIES], int kt, int dst, const int2& e) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int page = s ? e.y : e.x;
            const buf_rsrc_t r = make_rsrc(pool + keys.offset(page, kt, s), keys.bytes(page, kt, s));
#pragma unroll
            for (int p = s * (COPIES / 2); p < (s + 1) * (COPIES / 2); ++p)
                copy16<true>(r, off[p], (lds_ptr_t)((lds_char*)lds + dst + p * 1024));
        }
    };
    RowTile<F16, HD> rt[RT];
#pragma unroll
    for (int x = 0; x < RT; ++x) rt[x].clear();
    const int kfrag = j * D::ROW + ((g ^ k_key<D::CPR>(j)) << 4);
    const int vfrag = v_base<HD>(lane);
    const int clear = a.mask ? min(u.s.len, u.s.keys) : u.s.keys;

    // Tiles u.t0 + wave + WAVES i, i < n.  Copies past the last one repeat it.
    const int n = (u.t1 - u.t0 - wave + WAVES - 1) / WAVES;           // may be <= 0
    auto tile_at = [&](int i) { return u.t0 + wave + min(i, n - 1) * WAVES; };
    // This wave's LDS reads are behind: their stage may be copied into.
    auto reads_done = [&]() {
        wait_lgkmcnt<0>();
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" ::: "memory");
#endif
    };
    auto landed = [&]() {                                 // all but what was asked for after the oldest tile
        wait_vmcnt<COPIES * (2 * S - 1)>();
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" ::: "memory");
#endif
    };
    bool wild = false;
    if (n > 0) {
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int2 e = keys.entries(tile_at(i));
            issue(keys.k, k_off, tile_at(i), ring + i * D::HALF, e);
            issue(keys.v, v_off, tile_at(i), ring + (S + i) * D::HALF, e);
        }
        int2 now = keys.entries(tile_at(0)), next = keys.entries(tile_at(S));
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
        for (int x = 0; x < RT; ++x)                      // as above: the queries' loads end here
#pragma unroll
            for (int ks = 0; ks < D::NKS; ++ks) asm volatile("" ::"v"(qf[x][ks]));
#endif
        // Mask words of a tile, read a tile ahead as above.
        uint32_t lo[RT], hi[RT];
        auto words = [&](int kt, uint32_t (&l)[RT], uint32_t (&h)[RT]) {
            const int w = (kt * kTile - u.s.len) >> 5;
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                l[x] = mask_word(a, mrow[x], w);
                h[x] = mask_word(a, mrow[x], w + 1);
            }
        };
        words(tile_at(0), lo, hi);
        int stage = 0;
        for (int i = 0; i < n; ++i) {
            const int k0 = tile_at(i) * kTile;
            const int ks_at = ring + stage * D::HALF, vs_at = ks_at + S * D::HALF;
            landed();
            f32x16 st[RT];
#pragma unroll
            for (int x = 0; x < RT; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e) st[x][e] = 0.f;
            const int ka = ks_at + kfrag;
#pragma unroll
            for (int k4 = 0; k4 < D::NKS; k4 += 4) {
                s16x8 kf[4];
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    kf[y] = *(__attribute__((address_space(3))) const s16x8*)((lds_char*)lds + (ka ^ ((k4 + y) << 5)));
                sched_fence();
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int x = 0; x < RT; ++x) st[x] = mfma<F16>(kf[y], qf[x][k4 + y], st[x]);
            }
            uint32_t lo_next[RT], hi_next[RT];
            words(tile_at(i + 1), lo_next, hi_next);
            reads_done();
            issue(keys.k, k_off, tile_at(i + S), ks_at, next);
            const uint32_t gone = keys.missing(now);
            const bool masked = k0 + kTile > clear || gone;
            s16x8 pf[RT][TERMS][2];
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                if (__builtin_expect(masked, 0)) rt[x].hide(st[x], seen_keys(a, u.s, lo[x], hi[x], k0, gone), g);
                rt[x].softmax(st[x], a.scale_log2, a.lim, pf[x]);
            }
            landed();
            s16x8 vf[2][2];
            read_values<HD>(vf, lds, vs_at + vfrag, 0);
            sched_fence();
            wild |= add_values<F16, HD, RT, TERMS>(rt, pf, vf, lds, vs_at, lane, vfrag, masked);
            reads_done();
            issue(keys.v, v_off, tile_at(i + S), vs_at, next);
            now = S == 1 ? next : keys.entries(tile_at(i + 1));
            next = keys.entries(tile_at(i + 1 + S));
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                lo[x] = lo_next[x];
                hi[x] = hi_next[x];
            }
            stage = stage + 1 == S ? 0 : stage + 1;
        }
    }
    wait_all_memory();                                    // no copy may still land in LDS
    if (__builtin_expect(wild, 0)) add_wild<F16, HD, RT>(rt, a, u, keys, mrow, u.t0 + wave, u.t1, WAVES, clear, g);

    // The waves' shares of the rows, joined through LDS: each wave's outputs in its
    // own stages, 16-byte chunks turned by the row against bank conflicts.
    auto ml = [&](int w, int row) -> float2& { return reinterpret_cast<float2*>(smem + w * OWN + OUT)[row]; };
    float* own = reinterpret_cast<float*>(smem + ring);
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const float l = both_sum(rt[x].l);
#pragma unroll
        for (int nb = 0; nb < D::NB; ++nb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x16& o = rt[x].o[nb];
                *reinterpret_cast<f32x4*>(own + (x * 32 + j) * HD + (((nb * 8 + 2 * i + g) ^ (j & (C4 - 1))) << 2)) =
                    f32x4{o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]};
            }
        if (g == 0) ml(wave, x * 32 + j) = float2{rt[x].m, l};
    }
    __syncthreads();
    for (int x = tid; x < rows * C4; x += 256) {
        const int row = x / C4, c4 = x % C4;
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, ml(w, row).x);
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float2 part = ml(w, row);
            const float f = part.x == m ? 1.f : __builtin_amdgcn_exp2f((part.x - m) * a.scale_log2);
            const f32x4 v = *reinterpret_cast<const f32x4*>(smem + w * OWN + (row * HD + ((c4 ^ (row & 31 & (C4 - 1))) << 2)) * 4);
            l += part.y * f;
            o += v * f;
        }
        const int64_t t = packed_row<MODE>(a, u.s, (uint32_t)row / (uint32_t)a.group);
        const int h = u.kvh * a.group + (int)((uint32_t)row % (uint32_t)a.group);
        if (u.parts > 1) {
            *reinterpret_cast<f32x4*>(a.part_o + ((int64_t)u.slot * a.rows_per_wg + row) * HD + c4 * 4) = o;
            if (c4 == 0) a.part_ml[(int64_t)u.slot * a.rows_per_wg + row] = float2{m, l};
        } else if (MODE == kPrefix || (MODE == kSuffix && u.s.first > 0)) {
            *reinterpret_cast<f32x4*>(a.row_o + (t * a.n_heads + h) * HD + c4 * 4) = o;
            if (c4 == 0) a.row_ml[t * a.n_heads + h] = float2{m, l};
        } else {
            store_out<F16>(a, t, h, c4 * 4, HD, o, l == 0.f ? 0.f : 1.f / l);
            if (a.lse && c4 == 0) a.lse[t * a.n_heads + h] = log_sum<F16>(a, m, l);
        }
    }
}

template <bool F16, int HD, int RT, int S, int MODE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(HD == 64 && RT == 1 ? 4 : RT == 1 ? 2 : 1))) void
attend_few_kernel(const AttnArgs a) {
    __shared__ __attribute__((aligned(16))) char smem[FewLds<HD, RT, S>::ALL];
    attend_few<F16, HD, RT, S, MODE>(a, blockIdx.x, smem);
}

// Prefixes and up to 32 packed rows' own keys in one launch, so that neither waits for the
// other's start and end: units of the prefixes first.  Both take two terms of a probability, as
// the same windows do without a shared prefix.
template <bool F16, int HD, bool MANY>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(HD == 64 ? 3 : 2))) void
attend_both_kernel(const AttnArgs pre, const AttnArgs own) {
    constexpr int FEW = FewLds<HD, 1, 1>::ALL, ALL = MANY && kManyLds<HD, 1> > FEW ? kManyLds<HD, 1> : FEW;
    __shared__ __attribute__((aligned(16))) char smem[ALL];
    const Balance l = balance(pre, own);
    const int wg = blockIdx.x;
    if (wg < l.pre_units) {
        if constexpr (MANY) attend_many<F16, HD, false, 1, kPrefix, 2>(pre, wg < (l.pre_units & ~63) ? xcd_order(wg) : wg, smem, l.most_pre);
        else attend_few<F16, HD, 1, 1, kPrefix>(pre, wg, smem, l.most_pre);
    } else {
        attend_few<F16, HD, 1, 1, kSuffix>(own, wg - l.pre_units, smem, l.most_own);
    }
}

// The parts of an item's rows, joined in order: blockIdx.x the item, blockIdx.y a
// group of rows (every gridDim.y-th).  A thread takes 4 features of a row, and of
// the parts a run of a quarter, so that their loads are in flight together.  Bound by
// latency: 5 us with nothing to join, 6.9 for 256 parts of 64 KB.
constexpr int kJoinRuns = 4;

template <bool F16, int HD>
__global__ __launch_bounds__(256) void join_kernel(const AttnArgs a) {
    constexpr int C4 = HD / 4, ROWS = 256 / (C4 * kJoinRuns);
    __shared__ f32x4 run_o[kJoinRuns][ROWS][C4];
    __shared__ float2 run_ml[kJoinRuns][ROWS];
    Unit u;
    if (!find_unit<true, kPlain>(a, blockIdx.x, u)) return;
    const int rows = min(u.s.n * a.group - u.row_tile * a.rows_per_wg, a.rows_per_wg);
    const int c4 = threadIdx.x % C4, local = threadIdx.x / C4 % ROWS, run = threadIdx.x / (C4 * ROWS);
    const int each = (u.parts + kJoinRuns - 1) / kJoinRuns;
    const int p0 = min(run * each, u.parts), p1 = min(p0 + each, u.parts);
    for (int r0 = blockIdx.y * ROWS; r0 < rows; r0 += gridDim.y * ROWS) {
        const int row = min(r0 + local, rows - 1);
        const float2* ml = a.part_ml + (int64_t)u.slot * a.rows_per_wg + row;
        const float* po = a.part_o + ((int64_t)u.slot * a.rows_per_wg + row) * HD + c4 * 4;
        float m = -INFINITY, l = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        auto add = [&](const float2& part, const f32x4& v) {
            const float mn = fmaxf(m, part.x);
            const float f0 = m == mn ? 1.f : __builtin_amdgcn_exp2f((m - mn) * a.scale_log2);
            const float f1 = part.x == mn ? 1.f : __builtin_amdgcn_exp2f((part.x - mn) * a.scale_log2);
            l = l * f0 + part.y * f1;
            o = o * f0 + v * f1;
            m = mn;
        };
        int p = p0;
        for (; p + 8 <= p1; p += 8) {
            float2 part[8];
            f32x4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                part[i] = ml[(int64_t)(p + i) * a.rows_per_wg];
                v[i] = *reinterpret_cast<const f32x4*>(po + (int64_t)(p + i) * a.rows_per_wg * HD);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) add(part[i], v[i]);
        }
        for (; p < p1; ++p) add(ml[(int64_t)p * a.rows_per_wg], *reinterpret_cast<const f32x4*>(po + (int64_t)p * a.rows_per_wg * HD));
        run_o[run][local][c4] = o;
        if (c4 == 0) run_ml[run][local] = float2{m, l};
        __syncthreads();
        if (run == 0 && r0 + local < rows) {
#pragma unroll
            for (int i = 1; i < kJoinRuns; ++i) add(run_ml[i][local], run_o[i][local][c4]);
            const int pr = row + u.row_tile * a.rows_per_wg;
            const int64_t t = (int64_t)u.s.start + (uint32_t)pr / (uint32_t)a.group;
            const int h = u.kvh * a.group + (int)((uint32_t)pr % (uint32_t)a.group);
            store_out<F16>(a, t, h, c4 * 4, HD, o, l == 0.f ? 0.f : 1.f / l);
            if (a.lse && c4 == 0) a.lse[t * a.n_heads + h] = log_sum<F16>(a, m, l);
        }
        __syncthreads();
    }
}

// Rows behind a shared prefix, and rows of sequences that are split: what the prefix left
// (its parts, or one) and what the sequence's own keys left, joined in that order.
// blockIdx.x: the row; blockIdx.y: some of its heads.
template <bool F16, int HD>
__global__ __launch_bounds__(256) void join_rows_kernel(const AttnArgs a, const AttnArgs pre) {
    constexpr int C4 = HD / 4, ROWS = 256 / (C4 * kJoinRuns);
    __shared__ f32x4 run_o[kJoinRuns][ROWS][C4];
    __shared__ float2 run_ml[kJoinRuns][ROWS];
    const int lane = threadIdx.x & 63, t = blockIdx.x;
    int b = -1, start = 0;
    for (int b0 = 0; b0 < a.c.n_seqs && b < 0; b0 += 64) {
        const Seq s = sequence<kSuffix>(a, b0 + lane);
        const uint64_t hit = __ballot(s.n > 0 && t >= s.start && t - s.start < s.n);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            b = uniform(b0 + l);
            start = from_lane(s.start, l);
        }
    }
    if (b < 0) return;                                    // a row that no window covers
    const int4 own = a.info[b], member = a.members[b];
    const bool shared = member.x > 0;
    if (!shared && own.y <= 1) return;                    // written already
    const int4 front = shared ? pre.info[min(max(member.y, 0), a.c.n_seqs - 1)] : int4{0, 0, 0, 0};
    const int c4 = threadIdx.x % C4, local = threadIdx.x / C4 % ROWS, run = threadIdx.x / (C4 * ROWS);
    const int h = min((int)blockIdx.y * ROWS + local, a.n_heads - 1), kvh = h / a.group, j = h % a.group;
    // Where the parts lie: slot, row in it, or the row's own place.
    auto parts_of = [&](const AttnArgs& x, const int4& item, int row, int& n, int64_t& at) {
        const int pr = row * a.group + j, tile = pr >> x.rows_log2;
        n = min(max(item.y, 0), x.max_slots);
        const int64_t slot = item.x + ((int64_t)kvh * item.z + tile) * n;
        if (n > 1 && (slot < 0 || slot + n > x.max_slots)) n = 0;         // unsound row starts
        at = n > 1 ? slot * x.rows_per_wg + (pr & (x.rows_per_wg - 1)) : (int64_t)t * a.n_heads + h;
    };
    int n0 = 0, n1;
    int64_t at0 = 0, at1;
    if (shared) parts_of(pre, front, member.z + t - start, n0, at0);
    parts_of(a, own, t - start, n1, at1);
    const float* o0 = (n0 > 1 ? pre.part_o : pre.row_o) + at0 * HD + c4 * 4;
    const float* o1 = (n1 > 1 ? a.part_o : a.row_o) + at1 * HD + c4 * 4;
    const float2* ml0 = (n0 > 1 ? pre.part_ml : pre.row_ml) + at0;
    const float2* ml1 = (n1 > 1 ? a.part_ml : a.row_ml) + at1;
    const int n = n0 + n1, each = (n + kJoinRuns - 1) / kJoinRuns;
    const int p0 = min(run * each, n), p1 = min(p0 + each, n);
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](const float2& part, const f32x4& v) {
        const Two w = together(a, m, part.x);
        l = l * w.f0 + part.y * w.f1;
        o = o * w.f0 + v * w.f1;
        m = w.m;
    };
    constexpr int U = 8;
    for (int p = p0; p < p1; p += U) {
        float2 part[U];
        f32x4 v[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int x = min(p + i, p1 - 1);
            const int64_t k = x < n0 ? (int64_t)x * pre.rows_per_wg : (int64_t)(x - n0) * a.rows_per_wg;
            part[i] = (x < n0 ? ml0 : ml1)[k];
            v[i] = *reinterpret_cast<const f32x4*>((x < n0 ? o0 : o1) + k * HD);
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (p + i < p1) add(part[i], v[i]);
    }
    run_o[run][local][c4] = o;
    if (c4 == 0) run_ml[run][local] = float2{m, l};
    __syncthreads();
    if (run || (int)blockIdx.y * ROWS + local >= a.n_heads) return;
#pragma unroll
    for (int i = 1; i < kJoinRuns; ++i) add(run_ml[i][local], run_o[i][local][c4]);
    store_out<F16>(a, t, h, c4 * 4, HD, o, l == 0.f ? 0.f : 1.f / l);
    if (a.lse && c4 == 0) a.lse[(int64_t)t * a.n_heads + h] = log_sum<F16>(a, m, l);
}

// How a call is laid out: packed rows of a workgroup, keys of a step, units, least
// steps of a unit.  A second kernel that joins parts costs about 5 us, so short
// sequences are not split.  Whole against split, us per call of a replayed graph, 16
// heads on 4.  Few rows, up to 1024 keys whole: one row of 128, one sequence, 640 keys
// 8.5 / 8.9, 1024 11.0 / 9.1, 1280 12.7 / 9.5; of 32 sequences 768 12.0 / 15.1, 1024
// 14.8 / 18.3, 2048 25.7 / 28.0 (a single sequence would change over at 768, 32 of them
// not below 3000).  33 to 64 rows, the same line: 8 windows of 16 rows of 64, 512 keys
// 10.9 / 11.8, 768 13.4 / 12.0, 1280 18.5 / 12.5.  Many rows, up to 512 whole: 8 windows
// of 64 rows of 128, 320 keys 11.4 / 21.4, 1024 21.1 / 27.9, 1536 28.3 / 26.9; one of 64
// rows of 64, 512 10.6 / 11.4, 640 12.1 / 11.5, 1024 16.6 / 11.7.
// Many rows: with no more row tiles than CUs two wave groups each (8 trees of up to 64
// rows over 512 to 4096 keys: 16.7 + 6.9 us with the join, one group 20.7 + 9.0); with
// more of them one group, three workgroups per CU (8 x 1024 rows: 80 us, two groups
// 107).
struct Shape {
    int rows_per_wg, step, units, min_steps;
};
Shape shape_for(int max_rows, int group, int64_t many_items, int max_keys) {
    const int64_t rows = (int64_t)max_rows * group;
    if (rows <= 32) return {32, 4 * kTile, 512, max_keys <= 1024 ? 8 : 2};
    if (rows <= 64) return {64, 4 * kTile, 256, max_keys <= 1024 ? 8 : 2};
    if (many_items <= 256) return {kManyRows, 2 * kTile, 256, max_keys <= 512 ? 8 : 4};
    return {kManyRows, kTile, 512, 8};
}
// Split items have at least two parts of which all but one are full, so they make
// at most twice the units aimed at (and a few for the sum's rounding).
int slots_for(const Shape& s) { return 2 * s.units + 8; }
int64_t item_bound(int n_seqs, int n_kv, int total_rows, int max_rows, int group, int rows_per_wg) {
    const int64_t per_seq = ((int64_t)max_rows * group + rows_per_wg - 1) / rows_per_wg;
    return n_kv * std::min<int64_t>(n_seqs * per_seq, (int64_t)total_rows * group / rows_per_wg + n_seqs);
}
size_t round256(size_t n) { return (n + 255) / 256 * 256; }

int64_t round64(int64_t n) { return (n + 63) / 64 * 64; }
template <bool F16, int HD, int MODE>
hipError_t launch(const AttnArgs& a, int64_t items, bool may_split, hipStream_t st) {
    const int64_t wgs = round64(items + (may_split ? a.units : 0));
    if (wgs > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)wgs), block(256);
    if (a.rows_per_wg == 32)
        hipLaunchKernelGGL((attend_few_kernel<F16, HD, 1, 1, MODE>), grid, block, 0, st, a);
    else if (a.rows_per_wg == 64)
        hipLaunchKernelGGL((attend_few_kernel<F16, HD, 2, 2, MODE>), grid, block, 0, st, a);
    else {
        const bool once = (int64_t)a.max_rows * a.group <= kManyRows;     // one row tile: each key is read once
        const bool two = a.step == 2 * kTile;
        if (two && once)
            hipLaunchKernelGGL((attend_many_kernel<F16, HD, true, 2, MODE>), grid, dim3(512), 0, st, a);
        else if (two)
            hipLaunchKernelGGL((attend_many_kernel<F16, HD, false, 2, MODE>), grid, dim3(512), 0, st, a);
        else if (once)
            hipLaunchKernelGGL((attend_many_kernel<F16, HD, true, 1, MODE>), grid, block, 0, st, a);
        else
            hipLaunchKernelGGL((attend_many_kernel<F16, HD, false, 1, MODE>), grid, block, 0, st, a);
    }
    if (MODE == kPlain && may_split) {
        // Where there are many items few of them are split: a workgroup then walks rows.
        const int rows = (int)std::min<int64_t>(a.rows_per_wg, (int64_t)a.max_rows * a.group);
        const int per = 256 / (HD / 4 * kJoinRuns);
        const int64_t x = std::min<int64_t>(items, a.units);
        const int64_t y = std::min<int64_t>((rows + per - 1) / per, std::max<int64_t>(1, 2048 / x));
        hipLaunchKernelGGL((join_kernel<F16, HD>), dim3((unsigned)x, (unsigned)y), dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

// Whether some item of a call may have several parts.
bool may_split(const Shape& s, int max_keys) { return ((int64_t)max_keys + s.step - 1) / s.step > s.min_steps; }
size_t parts_bytes(const Shape& s, int head_dim) {
    const size_t rows = (size_t)slots_for(s) * s.rows_per_wg;
    return round256(rows * head_dim * 4) + round256(rows * 8);
}
// A launch's shape, and its parts at ws.
void take_shape(AttnArgs& a, const Shape& s, void* ws) {
    a.rows_per_wg = s.rows_per_wg;
    a.step = s.step;
    a.rows_log2 = __builtin_ctz((unsigned)s.rows_per_wg);
    a.step_log2 = __builtin_ctz((unsigned)s.step);
    a.units = s.units;
    a.min_steps = s.min_steps;
    a.max_slots = slots_for(s);
    a.part_o = (float*)ws;
    a.part_ml = (float2*)((char*)ws + round256((size_t)a.max_slots * s.rows_per_wg * a.c.head_dim * 4));
}
// n_items: sequences or groups at most.
int64_t items_of(const AttnArgs& a, int n_items) {
    return item_bound(n_items, a.c.n_kv, a.total_rows, a.max_rows, a.group, a.rows_per_wg);
}
// The list's counts are 32-bit, whatever the row starts.
bool countable(const AttnArgs& a) {
    return (int64_t)a.c.n_seqs * a.c.n_kv * (((int64_t)a.max_rows * a.group + a.rows_per_wg - 1) / a.rows_per_wg) <= (1 << 29);
}
template <int MODE>
hipError_t attend(const AttnArgs& a, int dtype, int n_items, bool split, hipStream_t st) {
    const CacheArgs& c = a.c;
    const int64_t items = items_of(a, n_items);
    if (!countable(a)) return hipErrorInvalidValue;
    if (dtype == DLM_F16)
        return c.head_dim == 128 ? launch<true, 128, MODE>(a, items, split, st) : launch<true, 64, MODE>(a, items, split, st);
    return c.head_dim == 128 ? launch<false, 128, MODE>(a, items, split, st) : launch<false, 64, MODE>(a, items, split, st);
}
// One launch for all sequences, and the join of their parts.
hipError_t attend_plain(AttnArgs& a, int dtype, void* ws, hipStream_t st) {
    const CacheArgs& c = a.c;
    const Shape s = shape_for(a.max_rows, a.group, item_bound(c.n_seqs, c.n_kv, a.total_rows, a.max_rows, a.group, kManyRows),
                              a.max_keys);
    take_shape(a, s, ws);
    return attend<kPlain>(a, dtype, c.n_seqs, may_split(s, a.max_keys), st);
}

AttnArgs attend_args(const CacheArgs& c, int dtype, int layer, const int32_t* row_start, int total_rows, int max_rows,
                     int max_keys, int n_heads, const void* q, int64_t q_stride, const uint32_t* mask, int mask_words,
                     float scale, void* o, int64_t o_stride, float* lse) {
    AttnArgs a{};
    a.c = c;
    a.layer_base = (int64_t)layer * c.n_pages * c.n_kv * c.page_len * c.head_dim * 2;
    a.row_start = row_start;
    a.total_rows = total_rows;
    a.max_rows = max_rows;
    a.max_keys = max_keys;
    a.group = n_heads / c.n_kv;
    a.n_heads = n_heads;
    a.q = (const uint16_t*)q;
    a.q_stride = q_stride;
    a.mask = mask;
    a.mask_words = mask ? mask_words : 0;                 // no words without a mask
    a.scale_log2 = scale * 1.4426950408889634f;
    a.lim = std::min((dtype == DLM_F16 ? kHeadroom<true> : kHeadroom<false>) / a.scale_log2, 3e38f);
    a.o = (uint16_t*)o;
    a.o_stride = o_stride;
    a.lse = lse;
    return a;
}

// ------------------------------------------------------------------ shared prefixes

// Layout of what cache_share leaves, in int32 words.
struct ShareWords {
    int64_t groups, members, rows, all;
};
__host__ __device__ inline ShareWords share_words(int n_seqs, int total_rows) {
    const int64_t groups = 0, members = 4 * (int64_t)n_seqs, rows = 2 * members;
    return {groups, members, rows, rows + total_rows};
}

__device__ __forceinline__ int block_add(int v, int* lds) {       // over 1024 threads
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    int t = 0;
    for (int i = 0; i < 16; ++i) t += lds[i];
    return t;
}
__device__ __forceinline__ int block_min(int v, int* lds) {
    for (int o = 32; o; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    int t = lds[0];
    for (int i = 1; i < 16; ++i) t = min(t, lds[i]);
    return t;
}

// Group blockIdx.x, a thread per sequence: its members with rows, the tokens whose pages
// all their tables begin with, and their rows one after the other.  A group is left alone
// (prefix 0) if it has a single member, nothing in common, or more rows than the caller said.
__global__ __launch_bounds__(1024) void share_kernel(CacheArgs c, const int32_t* __restrict__ row_start, int total_rows,
                                                     int max_rows, const int32_t* __restrict__ group, int max_group_rows,
                                                     int32_t* __restrict__ out) {
    __shared__ int lds[16], members[kCacheMaxSeqs], wave_rows[16], wave_members[16];
    const ShareWords w = share_words(c.n_seqs, total_rows);
    const int g = blockIdx.x, s = threadIdx.x, lane = s & 63, wave = s >> 6;
    int id = -1, n = 0, start = 0, len = 0;
    if (s < c.n_seqs) {
        id = group[s];
        start = row_start[s];
        const int end = min(row_start[s + 1], total_rows);
        n = start >= 0 && end > start ? min(end - start, max_rows) : 0;
        len = max(c.len[s], 0);
        if ((unsigned)id >= (unsigned)c.n_seqs || n == 0) {
            if (s == g) *reinterpret_cast<int4*>(out + w.members + 4 * s) = int4{0, 0, 0, 0};
            id = -1;
        }
    }
    const bool in = id == g;
    const uint64_t any = __ballot(in);
    // All rows in 32 bits: total_rows <= 2^24 and at most 1024 sequences, so 2^34 by unsound
    // row starts; counted in units that cannot pass, and compared as such.
    const int all = block_add((n + 15) >> 4, lds);                // at most 2^30
    const int exact = all > (1 << 26) ? total_rows + 1 : block_add(n, lds);
    const int mine = block_add(in ? 1 : 0, lds);
    if (mine == 0) {                                              // nobody's group
        if (s == 0) *reinterpret_cast<int4*>(out + w.groups + 4 * g) = int4{0, 0, 0, 0};
        return;
    }
    const int leader = block_min(in ? s : 0x7fffffff, lds);
    // Rows and members before this thread's.
    const int rows_in = in ? n : 0;
    int scan = rows_in;
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(scan, o, 64);
        if (lane >= o) scan += y;
    }
    if (lane == 63) {
        wave_rows[wave] = scan;
        wave_members[wave] = __popcll(any);
    }
    __syncthreads();
    int off = scan - rows_in, place = __popcll(any & ((1ull << lane) - 1)), rows = 0;
    for (int i = 0; i < 16; ++i) {
        if (i < wave) {
            off += wave_rows[i];
            place += wave_members[i];
        }
        rows += wave_rows[i];
    }
    if (in) members[place] = s;
    const int list = exact > total_rows ? 0 : block_add(id >= 0 && id < g ? n : 0, lds);
    // Tokens that every member counts, in whole pages.
    int pages = block_min(in ? min(len >> c.page_log2, c.max_pages) : 0x7fffffff, lds);
    if (mine < 2 || rows > max_group_rows || exact > total_rows) pages = 0;
    int same = pages;
    const int32_t* front = c.table + (int64_t)leader * c.max_pages;
    for (int m = wave; m < mine && pages; m += 16) {
        const int32_t* row = c.table + (int64_t)members[m] * c.max_pages;
#pragma unroll 4
        for (int e = lane; e < pages; e += 64) {
            const int page = row[e];
            if (page != front[e] || (uint32_t)page >= (uint32_t)c.n_pages) same = min(same, e);
        }
    }
    same = block_min(same, lds);
    const int prefix = (same << c.page_log2) & ~(kTile - 1);
    if (in) *reinterpret_cast<int4*>(out + w.members + 4 * s) = int4{prefix, g, off, 0};
    if (s == 0)
        *reinterpret_cast<int4*>(out + w.groups + 4 * g) = prefix ? int4{leader, prefix, list, rows} : int4{0, 0, 0, 0};
    if (prefix)
        for (int i = 0; in && i < n; ++i) out[w.rows + list + off + i] = start + i;
}

// Units aimed at where prefixes and own keys share a launch: two per CU, the workgroups that the
// chip holds with heads of 128 (64 sequences behind 16384 shared tokens: 384 to 640 cost the
// same); with heads of 64 it holds four per CU.
constexpr int kBothUnits = 512;
// A group has at least two sequences.
int most_groups(int n_seqs) { return std::max(n_seqs / 2, 1); }
Shape prefix_shape(int n_seqs, int n_kv, int total_rows, int max_rows, int max_group_rows, int group, int max_keys) {
    if ((int64_t)max_rows * group <= 32) {                // beside the sequences' own keys
        if ((int64_t)max_group_rows * group <= 32) return {32, 4 * kTile, kBothUnits, 2};
        return {kManyRows, kTile, kBothUnits, 8};
    }
    return shape_for(max_group_rows, group, item_bound(most_groups(n_seqs), n_kv, total_rows, max_group_rows, group, kManyRows),
                     max_keys);
}
Shape own_shape(int n_seqs, int n_kv, int total_rows, int max_rows, int group, int max_keys) {
    return shape_for(max_rows, group, item_bound(n_seqs, n_kv, total_rows, max_rows, group, kManyRows), max_keys);
}
// Whether it pays.  What it saves are bytes: without it every sequence reads its keys, most
// of them from the caches.  What it costs are a join that is always there, and each row's
// values out and in again.  So: the keys of as many sequences as there are windows of
// max_rows, against 48 MB and 1000 bytes for each value of the result.  Plain / shared, us,
// bf16, a group of n sequences with 40 tokens of their own.  16 heads of 128 on 4, a row
// each: n 4, 2048 shared tokens 10.2 / 11.8, 4096 13.4 / 12.6, 6144 16.0 / 13.0 (not shared: the
// line is too high for so few), 8192 15.1 / 14.0, 16384 22.3 / 18.1; n 16, 2048 13.5 / 15.2, 4096
// 18.5 / 15.6; n 64, 1024 16.6 / 18.0, 2048 22.8 / 18.9, 4096 35.6 / 21.6; 4 rows each, n
// 16, 4096 19.2 / 21.2, 16384 43.1 / 34.0; 12 rows each, 4096 30.2 / 38.0, 16384 68.4 / 55.4.
// 16 heads of 64: n 16, 512 8.1 / 11.7, 1024 13.2 / 12.1, 2048 17.3 / 12.3.
bool shares(const AttnArgs& a, int max_group_rows) {
    if (!attend_may_share(a.max_rows, max_group_rows, a.group)) return false;
    // join_rows_kernel has a workgroup per row and some of its heads; an axis takes fewer than
    // 2^32 threads.
    if (a.total_rows >= (1 << 24)) return false;
    const double values = (double)a.total_rows * a.n_heads * a.c.head_dim;
    // Rows may be more than the windows have: no more of them than sequences.
    const double windows = std::min(((double)a.total_rows + a.max_rows - 1) / a.max_rows, (double)a.c.n_seqs);
    return windows * a.max_keys * (4. * a.c.n_kv * a.c.head_dim) >= 48e6 + 1000. * values;
}
size_t row_bytes(int total_rows, int n_heads, int head_dim) {
    const size_t n = (size_t)total_rows * n_heads;
    return round256(n * head_dim * 4) + round256(n * 8);
}

}  // namespace

size_t attend_workspace_bytes(int n_seqs, int n_kv, int head_dim, int total_rows, int max_rows, int group) {
    return parts_bytes(own_shape(n_seqs, n_kv, total_rows, max_rows, group, 0), head_dim);
}

hipError_t launch_attend(const CacheArgs& c, int dtype, int layer, const int32_t* row_start, int total_rows,
                         int max_rows, int max_keys, int n_heads, const void* q, int64_t q_stride,
                         const uint32_t* mask, int mask_words, float scale, void* o, int64_t o_stride, float* lse,
                         void* ws, hipStream_t st) {
    AttnArgs a = attend_args(c, dtype, layer, row_start, total_rows, max_rows, max_keys, n_heads, q, q_stride, mask, mask_words,
                             scale, o, o_stride, lse);
    return attend_plain(a, dtype, ws, st);
}

size_t share_bytes(int n_seqs, int total_rows) { return (size_t)share_words(n_seqs, total_rows).all * 4; }

hipError_t launch_share(const CacheArgs& c, const int32_t* row_start, int total_rows, int max_rows, const int32_t* group,
                        int max_group_rows, int32_t* share, hipStream_t st) {
    hipLaunchKernelGGL(share_kernel, dim3(c.n_seqs), dim3(1024), 0, st, c, row_start, total_rows, max_rows, group,
                       max_group_rows, share);
    return hipGetLastError();
}

bool attend_may_share(int max_rows, int max_group_rows, int group) {
    return max_group_rows > max_rows && (int64_t)max_rows * group <= kManyRows;
}

size_t attend_shared_workspace_bytes(int n_seqs, int n_kv, int head_dim, int total_rows, int max_rows, int max_group_rows,
                                     int group) {
    const size_t own = attend_workspace_bytes(n_seqs, n_kv, head_dim, total_rows, max_rows, group);
    if (!attend_may_share(max_rows, max_group_rows, group)) return own;
    return own + parts_bytes(prefix_shape(n_seqs, n_kv, total_rows, max_rows, max_group_rows, group, 0), head_dim) +
           2 * (row_bytes(total_rows, n_kv * group, head_dim) + round256((size_t)n_seqs * sizeof(int4)));
}

hipError_t launch_attend_shared(const CacheArgs& c, int dtype, int layer, const int32_t* row_start, int total_rows,
                                int max_rows, int max_group_rows, int max_keys, const int32_t* share, int n_heads,
                                const void* q, int64_t q_stride, const uint32_t* mask, int mask_words, float scale, void* o,
                                int64_t o_stride, float* lse, void* ws, hipStream_t st) {
    AttnArgs a = attend_args(c, dtype, layer, row_start, total_rows, max_rows, max_keys, n_heads, q, q_stride, mask, mask_words,
                             scale, o, o_stride, lse);
    if (!shares(a, max_group_rows)) return attend_plain(a, dtype, ws, st);
    const ShareWords w = share_words(c.n_seqs, total_rows);
    a.groups = (const int4*)(share + w.groups);
    a.members = (const int4*)(share + w.members);
    a.rows = share + w.rows;
    AttnArgs p = a;
    p.max_rows = max_group_rows;
    p.mask = nullptr;
    p.mask_words = 0;
    const bool both = (int64_t)max_rows * a.group <= 32;
    const Shape sp = prefix_shape(c.n_seqs, c.n_kv, total_rows, max_rows, max_group_rows, a.group, max_keys);
    Shape sa = own_shape(c.n_seqs, c.n_kv, total_rows, max_rows, a.group, max_keys);
    if (both) {                                           // few rows either way: 256 keys at least
        sa.units = kBothUnits;
        sa.min_steps = 2;
    }
    char* at = (char*)ws;
    auto carve = [&](AttnArgs& x, const Shape& s) {
        x.info = (int4*)at;
        at += round256((size_t)c.n_seqs * sizeof(int4));
        x.row_o = (float*)at;
        x.row_ml = (float2*)(at + round256((size_t)total_rows * n_heads * c.head_dim * 4));
        at += row_bytes(total_rows, n_heads, c.head_dim);
        take_shape(x, s, at);
        at += parts_bytes(s, c.head_dim);
    };
    carve(p, sp);
    carve(a, sa);
    hipError_t e;
    if (both) {
        if (!countable(p) || !countable(a)) return hipErrorInvalidValue;
        // An item makes less than one unit more than its share of `units` (balance): a few over
        // for the rounding of their sum.
        const int64_t wgs = items_of(p, most_groups(c.n_seqs)) + items_of(a, c.n_seqs) + kBothUnits + 8;
        if (wgs > 0x7fffffff) return hipErrorInvalidValue;
        const bool many = sp.rows_per_wg == kManyRows;
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(256), 0, st, p, a);
            return hipGetLastError();
        };
        auto pick = [&](auto f16) {
            constexpr bool F = decltype(f16)::value;
            if (c.head_dim == 128) return many ? go(attend_both_kernel<F, 128, true>) : go(attend_both_kernel<F, 128, false>);
            return many ? go(attend_both_kernel<F, 64, true>) : go(attend_both_kernel<F, 64, false>);
        };
        e = dtype == DLM_F16 ? pick(std::true_type{}) : pick(std::false_type{});
    } else {
        e = attend<kPrefix>(p, dtype, most_groups(c.n_seqs), may_split(sp, max_keys), st);
        if (e == hipSuccess) e = attend<kSuffix>(a, dtype, c.n_seqs, may_split(sa, max_keys), st);
    }
    if (e != hipSuccess) return e;
    const int per = 256 / (c.head_dim / 4 * kJoinRuns);
    const dim3 grid((unsigned)total_rows, (unsigned)((n_heads + per - 1) / per));
    auto kernel = dtype == DLM_F16 ? (c.head_dim == 128 ? join_rows_kernel<true, 128> : join_rows_kernel<true, 64>)
                                   : (c.head_dim == 128 ? join_rows_kernel<false, 128> : join_rows_kernel<false, 64>);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a, p);
    return hipGetLastError();
}
