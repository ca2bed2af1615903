// Attention of packed windows over a paged cache (dlm_cache_attend).
//
// Rows.  The query heads that share a key head read the same keys, so they are
// packed with the window's rows: row r of (sequence, key head) is window row r /
// G, query head r % G of the group of G.  A workgroup takes up to 128 packed
// rows, 32 per wave, and one run of keys.
//
// Keys.  Tiles of 32 keys go from their pages to LDS by buffer copies that bypass
// registers (NS stages, XOR-swizzled 16-byte chunks); a page is a scalar, so a
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
// nothing wider at this rate; relative 2^-9 or 2^-12 of each, of no sign), sums
// add the unrounded ones.  The running maximum moves only when a tile raises it
// by more than 2^8 in the exp2 domain.
//
// Masks.  Only tiles that meet the window, the last token or a missing page are
// masked, by a 32-bit word per row.  A product with 0 does not hide an infinity
// or a NaN in a value that a row must not see, so masked tiles look for such
// values; where there are any they are taken out of the product and put back, as
// infinities or NaN, into the rows that see them.
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

#include "common.h"
#include "cache.h"

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

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

__device__ __forceinline__ s16x4 lds_transpose(lds_ptr_t p) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
#else
    return s16x4{};
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
    float scale_log2;
    uint16_t* o;
    int64_t o_stride;
    float* lse;
    int rows_per_wg;                          // packed rows of a workgroup
    int step;                                 // keys of a step
    int min_steps;                            // least steps of a unit
    int units;                                // units aimed at
    float* part_o;                            // [slots][rows_per_wg][head_dim]
    float2* part_ml;                          // [slots][rows_per_wg]
};

struct Seq {
    int n, start, len, keys;                  // rows, first packed row, tokens before, keys in all
};
__device__ __forceinline__ Seq sequence(const AttnArgs& a, int b) {
    Seq s{0, 0, 0, 0};
    if (b < a.c.n_seqs) {
        s.start = a.row_start[b];
        const int end = min(a.row_start[b + 1], a.total_rows);
        s.n = s.start >= 0 ? min(max(end - s.start, 0), a.max_rows) : 0;
        s.len = max(a.c.len[b], 0);
        s.keys = (int)min((int64_t)s.len + s.n, (int64_t)a.max_keys);
    }
    return s;
}

// What a wave works out about one unit, or one split item, of the list.
struct Unit {
    Seq s;
    int b, row_tile, kvh;
    int t0, t1;                               // tiles of 32 keys
    int slot, parts;                          // workspace slot of this part; parts of its item
};

__device__ __forceinline__ int wave_scan(int v, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(v, o, 64);
        if (lane >= o) v += y;
    }
    return v;
}

// The index-th unit (or, with `items`, the index-th item of several parts) in the
// order sequence, key head, part, row tile; false if there are fewer.  A lane
// looks after a sequence, 64 at a time.
template <bool ITEMS>
__device__ __forceinline__ bool find_unit(const AttnArgs& a, int index, Unit& u) {
    const int lane = threadIdx.x & 63;
    const int per_tile = a.rows_per_wg;
    auto shape = [&](const Seq& s, int& tiles, int& steps) {
        tiles = (s.n * a.group + per_tile - 1) / per_tile;
        steps = max((s.keys + a.step - 1) / a.step, 1);
    };
    int sum = 0;                                          // steps of all items (fits: checked by the host)
    for (int b0 = 0; b0 < a.c.n_seqs; b0 += 64) {
        int tiles, steps;
        shape(sequence(a, b0 + lane), tiles, steps);
        int w = tiles * steps * a.c.n_kv;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) w += __shfl_xor(w, o, 64);
        sum += w;
    }
    const int most = max(a.min_steps, (sum + a.units - 1) / a.units);
    int before = 0, slots_before = 0;
    for (int b0 = 0; b0 < a.c.n_seqs; b0 += 64) {
        int tiles, steps;
        const Seq s = sequence(a, b0 + lane);
        shape(s, tiles, steps);
        const int parts = (steps + most - 1) / most;
        const int all = tiles * a.c.n_kv * parts, split = parts > 1 ? all : 0;
        const int count = ITEMS ? (parts > 1 ? tiles * a.c.n_kv : 0) : all;
        const int end = before + wave_scan(count, lane), slot_end = slots_before + wave_scan(split, lane);
        const uint64_t hit = __ballot(index < end && index >= end - count);
        if (hit) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            u.b = uniform(b0 + l);
            u.s.n = uniform(__shfl(s.n, l, 64));
            u.s.start = uniform(__shfl(s.start, l, 64));
            u.s.len = uniform(__shfl(s.len, l, 64));
            u.s.keys = uniform(__shfl(s.keys, l, 64));
            u.parts = uniform(__shfl(parts, l, 64));
            const int n_tiles = uniform(__shfl(tiles, l, 64));
            const int all_steps = uniform(__shfl(steps, l, 64));
            int i = index - uniform(__shfl(end - count, l, 64));
            const int slot0 = uniform(__shfl(slot_end - split, l, 64));
            u.row_tile = uniform(i % n_tiles);
            i /= n_tiles;
            int part = 0;
            if (!ITEMS) {
                part = uniform(i % u.parts);
                i /= u.parts;
            }
            u.kvh = uniform(i);
            // slots of an item's parts lie next to each other
            u.slot = slot0 + (u.kvh * n_tiles + u.row_tile) * u.parts + part;
            const int each = (all_steps + u.parts - 1) / u.parts * (a.step / kTile);
            u.t0 = uniform(part * each);
            u.t1 = uniform(min(u.t0 + each, (u.s.keys + kTile - 1) / kTile));
            return true;
        }
        before = __shfl(end, 63, 64);
        slots_before = __shfl(slot_end, 63, 64);
    }
    return false;
}

// ------------------------------------------------------------------ the kernel

// Between a tile's copies having landed for this wave and its use: the waves that
// share the tile meet, a wave of its own only has its earlier LDS reads behind it.
template <int WAVES>
__device__ __forceinline__ void tile_barrier() {
    if constexpr (WAVES > 1) {
        lds_barrier();
    } else {
        wait_lgkmcnt<0>();
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" ::: "memory");
#endif
    }
}

// Four features of a finished row.
template <bool F16>
__device__ __forceinline__ void store_out(const AttnArgs& a, int64_t t, int head, int feature, int hd, const f32x4& v,
                                          float inv) {
    const u32x2 w = {pack2<F16>(v[0] * inv, v[1] * inv), pack2<F16>(v[2] * inv, v[3] * inv)};
    *reinterpret_cast<u32x2*>(a.o + t * a.o_stride + head * hd + feature) = w;
}
__device__ __forceinline__ float log_sum(const AttnArgs& a, float m, float l) {
    return l == 0.f ? -INFINITY : (m * a.scale_log2 + __builtin_amdgcn_logf(l)) * 0.69314718f;
}

// WK groups of waves of a workgroup take its tiles in turn, each with NS stages
// of its own; the 4 / WK waves of a group share the tiles and take 32 rows each.
template <bool F16, int HD, int WK, int NS, int WPE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(WPE))) void attend_kernel(const AttnArgs a) {
    constexpr int WM = 4 / WK;
    constexpr int CPR = HD / 8;                           // 16-byte chunks of a row
    constexpr int ROW = HD * 2;
    constexpr int HALF = kTile * ROW;                     // bytes of a K or V tile
    constexpr int STAGE = 2 * HALF;
    constexpr int COPIES = HALF / 1024 / WM;              // 1 KB copies per wave of a K or V tile
    constexpr int NB = HD / 32, NKS = HD / 16;
    static_assert(COPIES >= 1 && NS >= 2, "stages");
    // The kernel's only LDS variable: with a second one the compiler tells the two
    // apart, takes a fragment read to depend on every copy in flight into this one,
    // and waits for them all.
    __shared__ __attribute__((aligned(16))) char smem[WK * NS * STAGE];

    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int g = lane >> 5, j = lane & 31;
    const int wm = wave % WM, wk = wave / WM;
    Unit u;
    // Neighbouring units share their keys (row tiles): workgroups go to the 8 XCDs
    // in turn, so each XCD takes runs of 8 units.
    const int wg = blockIdx.x;
    const int index = WK == 1 ? (wg & ~63) + (wg & 7) * 8 + ((wg >> 3) & 7) : wg;
    if (!find_unit<false>(a, index, u)) return;
    const int rows = min(u.s.n * a.group - u.row_tile * a.rows_per_wg, a.rows_per_wg);   // of this workgroup
    const bool busy = wm * 32 < rows;                     // this wave has rows
    const int r = min(wm * 32 + j, rows - 1) + u.row_tile * a.rows_per_wg;
    const int node = r / a.group, head = u.kvh * a.group + r % a.group;
    const int64_t t = (int64_t)u.s.start + node;          // packed row

    const lds_ptr_t lds = (lds_ptr_t)smem;
    const int ring = wk * NS * STAGE;
    // Copies: lane L of copy p reads the chunk that belongs at byte 16 L of its
    // 1 KB block; the block's rows lie within one group of 16 keys, which lie in one
    // page.
    constexpr int ROWS_PER_COPY = 64 / CPR;
    uint32_t k_off[COPIES], v_off[COPIES];
#pragma unroll
    for (int p = 0; p < COPIES; ++p) {
        const int row = (wm * COPIES + p) * ROWS_PER_COPY + lane / CPR, pc = lane % CPR;
        k_off[p] = (uint32_t)((row & 15) * ROW + ((pc ^ k_key<CPR>(row)) << 4));
        v_off[p] = (uint32_t)((row & 15) * ROW + ((pc ^ v_key<CPR>(row)) << 4));
    }
    const int64_t head_bytes = (int64_t)a.c.page_len * ROW;
    const char* kp = a.c.k + a.layer_base + u.kvh * head_bytes;
    const char* vp = a.c.v + a.layer_base + u.kvh * head_bytes;
    const int64_t page_bytes = head_bytes * a.c.n_kv;
    const int32_t* table = a.c.table + (int64_t)u.b * a.c.max_pages;
    // Pages of the two groups of 16 keys of a tile.  Entries past the row's end are
    // read as its last one, whose keys then lie behind the last token.
    struct Pages {
        int p[2];
    };
    auto pages_of = [&](int kt) {
        Pages x;
#pragma unroll
        for (int s = 0; s < 2; ++s)
            x.p[s] = uniform(ld_const(table + min((kt * kTile + s * 16) >> a.c.page_log2, a.c.max_pages - 1)));
        return x;
    };
    auto held = [&](int page) { return page >= 0 && page < a.c.n_pages; };
    constexpr int SUBS = COPIES * ROWS_PER_COPY > 16 ? 2 : 1;   // groups of 16 keys that a wave copies from
    uint32_t missing = 0;                                 // two bits per stage: groups without a page
    auto issue = [&](int kt, int stage, const Pages& pages) {
        const int kd = ring + stage * STAGE + wm * COPIES * 1024;
        missing &= ~(3u << (2 * stage));
        missing |= (uint32_t)uniform((held(pages.p[0]) ? 0 : 1) | (held(pages.p[1]) ? 0 : 2)) << (2 * stage);
#pragma unroll
        for (int s = 0; s < SUBS; ++s) {
            const int sub = SUBS == 2 ? s : wm * COPIES * ROWS_PER_COPY / 16;
            const int key = kt * kTile + sub * 16;
            const int page = uniform(sub ? pages.p[1] : pages.p[0]);
            const int bytes = uniform(held(page) ? min(max(u.s.keys - key, 0), 16) * ROW : 0);
            const int64_t at = uniform(held(page) ? page : 0) * page_bytes + (key & (a.c.page_len - 1)) * ROW;
            const buf_rsrc_t kr = make_rsrc(kp + at, bytes), vr = make_rsrc(vp + at, bytes);
#pragma unroll
            for (int p = 0; p < COPIES / SUBS; ++p) {
                const int c = s * (COPIES / SUBS) + p;
                lds_dma16_buf(kr, k_off[c], 0, (lds_ptr_t)((lds_char*)lds + kd + c * 1024));
            }
#pragma unroll
            for (int p = 0; p < COPIES / SUBS; ++p) {
                const int c = s * (COPIES / SUBS) + p;
                lds_dma16_buf(vr, v_off[c], 0, (lds_ptr_t)((lds_char*)lds + kd + HALF + c * 1024));
            }
        }
    };

    s16x8 qf[NKS];
    {
        const uint16_t* qp = a.q + t * a.q_stride + head * HD + g * 8;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) qf[ks] = *reinterpret_cast<const s16x8*>(qp + ks * 16);
    }
    f32x16 oacc[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[n][e] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;                 // m_run in units of the scores

    // Fragments.  A stage starts at a multiple of a row and a chunk's number is the
    // only thing in the address bits that it takes up, so the k-th chunk pair of K
    // (2 k + g, with the row's key) and the n-th four chunks of V are one base each
    // with a constant xor-ed in.
    const int kfrag = j * ROW + ((g ^ k_key<CPR>(j)) << 4);
    // Transposing reads: lane i of 16 hands in 4 values of row i / 4; rows 8 apart
    // have the same key.
    const int vrow = 4 * g + ((lane & 15) >> 2);
    const int vfrag = HALF + vrow * ROW + (lane & 1) * 8 +
                      (((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ v_key<CPR>(vrow)) << 4);
    const uint32_t* mrow = a.mask ? a.mask + t * a.mask_words : nullptr;

    // One tile's scores, softmax and products; masked: some row does not see all of
    // it.  One path with scalar branches around what masks need: two copies of the
    // products would hold the accumulators twice.
    auto tile = [&](bool masked, int k0, int sb, uint32_t gone) {

        const int ka = sb + kfrag, va = sb + vfrag;
        f32x16 st;
#pragma unroll
        for (int e = 0; e < 16; ++e) st[e] = 0.f;
#pragma unroll
        for (int k4 = 0; k4 < NKS; k4 += 4) {
            s16x8 kf[4];
#pragma unroll
            for (int x = 0; x < 4; ++x)
                kf[x] = *(__attribute__((address_space(3))) const s16x8*)((lds_char*)lds + (ka ^ ((k4 + x) << 5)));
            sched_fence();
#pragma unroll
            for (int x = 0; x < 4; ++x) st = mfma<F16>(kf[x], qf[k4 + x], st);
        }

        uint32_t see = 0xffffffffu;                       // keys that the row sees
        if (__builtin_expect(masked, 0)) {
            const int rel = k0 - u.s.len;                 // first key's place in the window
            if (mrow) {
                const int w = rel >> 5, sh = rel & 31;
                const uint32_t lo = w >= 0 && w < a.mask_words ? mrow[w] : 0;
                const uint32_t hi = w + 1 >= 0 && w + 1 < a.mask_words ? mrow[w + 1] : 0;
                see = sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
                if (rel < 0) see |= rel <= -32 ? 0xffffffffu : (1u << -rel) - 1;      // tokens before the window
            }
            const int left = u.s.keys - k0;
            if (left < 32) see &= left <= 0 ? 0 : (1u << left) - 1;
            if (gone & 1) see &= 0xffff0000u;
            if (gone & 2) see &= 0x0000ffffu;
            const uint32_t mine_see = see >> (4 * g);
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (!((mine_see >> (8 * (e >> 2) + (e & 3))) & 1)) st[e] = -INFINITY;
        }
        float mt = st[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mt = fmaxf(mt, st[e]);
        mt = both_max(mt);
        // Each row by its own scores alone, so that its bits do not depend on others'.
        const bool move = (mt - m_run) * a.scale_log2 > 8.f;
        if (__any(move)) {
            const float m_new = move ? mt : m_run;
            const float alpha = move ? __builtin_amdgcn_exp2f((m_run - m_new) * a.scale_log2) : 1.f;
            l_run *= alpha;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[n][e] *= alpha;
            m_run = m_new;
        }
        const float nb = m_run == -INFINITY ? 0.f : -m_run * a.scale_log2;
        float lt = 0.f;
        s16x8 pf[2];
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(st[8 * s2 + 2 * i], a.scale_log2, nb));
                const float p1 = __builtin_amdgcn_exp2f(fmaf(st[8 * s2 + 2 * i + 1], a.scale_log2, nb));
                lt += p0 + p1;
                w[i] = pack2<F16>(p0, p1);
            }
            pf[s2] = __builtin_bit_cast(s16x8, w);
        }
        l_run += lt;

        // V^T fragments of 16 keys: two transposing reads of 4 keys each.
        auto v_frag = [&](int n, int s2) {
            const int at = va ^ (n << 6);
            const s16x4 lo = lds_transpose((lds_ptr_t)((lds_char*)lds + at + (16 * s2) * ROW));
            const s16x4 hi = lds_transpose((lds_ptr_t)((lds_char*)lds + at + (16 * s2 + 8) * ROW));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        // Keys with an infinity or NaN in V, of a tile that some row does not see whole.
        uint32_t wild = 0;
        if (__builtin_expect(masked, 0)) {
            uint32_t hi = 0, lo = 0;                      // largest magnitudes among a key's values
#pragma unroll
            for (int x = 0; x < CPR / 2; ++x) {
                const u32x4 w = *(__attribute__((address_space(3))) const u32x4*)((lds_char*)lds + sb + HALF + j * ROW +
                                                                                 (g * (CPR / 2) + x) * 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    hi = max(hi, w[i] & 0x7fffffffu);
                    lo = max(lo, (w[i] << 16) & 0x7fffffffu);
                }
                if (x % 2) sched_fence();                 // few registers at a time
            }
            const uint64_t votes = __ballot(is_wild<F16>(max(hi, lo) >> 16));
            wild = uniform((int)((uint32_t)votes | (uint32_t)(votes >> 32)));
        }
#pragma unroll
        for (int n2 = 0; n2 < NB; n2 += 2) {
            s16x8 vf[2][2];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int s2 = 0; s2 < 2; ++s2) vf[n][s2] = v_frag(n2 + n, s2);
            sched_fence();
            if (__builtin_expect(wild, 0)) {              // finite values only; the others follow
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        short& v = reinterpret_cast<short(&)[8]>(vf[x >> 1][x & 1])[i];
                        v = is_wild<F16>((uint16_t)v) ? (short)0 : v;
                    }
            }
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
                for (int n = 0; n < 2; ++n) oacc[n2 + n] = mfma<F16>(vf[n][s2], pf[s2], oacc[n2 + n]);
        }
        if (__builtin_expect(wild, 0)) {
            // Rare: infinities and NaN, whatever their probability, into the rows that
            // see their keys.
            for (uint32_t left = wild; left; left &= left - 1) {
                const int key = __builtin_ctz(left);
                const bool sees = (see >> key) & 1;
                const int at = sb + HALF + key * ROW + 8 * g;
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const u32x2 w = *(__attribute__((address_space(3))) const u32x2*)((lds_char*)lds + at +
                                                                                         (((4 * n + i) ^ v_key<CPR>(key)) << 4));
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const uint32_t bits = (x & 1 ? w[x >> 1] >> 16 : w[x >> 1]) & 0xffffu;
                            if (sees && is_wild<F16>(bits)) oacc[n][4 * i + x] += widen<F16>(bits);
                        }
                        sched_fence();
                    }
            }
        }
    };

    // Tiles of this wave group: t0 + wk, t0 + wk + WK, ...  Copies past the last
    // one repeat it into a stage that is not read again.
    const int mine = (u.t1 - u.t0 - wk + WK - 1) / WK;    // may be <= 0
    const int last = u.t0 + wk + (mine - 1) * WK;
    Pages next{};
    if (mine > 0) {
#pragma unroll
        for (int s = 0; s < NS - 1; ++s) {
            const int kt = min(u.t0 + wk + s * WK, last);
            issue(kt, s, pages_of(kt));
        }
        next = pages_of(min(u.t0 + wk + (NS - 1) * WK, last));
    }
    // The queries' loads end here and not inside the loop, where their wait would
    // take the copies in flight with it.
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) asm volatile("" ::"v"(qf[ks]));
#endif
    const int clear = a.mask ? u.s.len : u.s.keys;        // keys that every row sees
    int stage = 0;
    for (int it = 0; it < mine; ++it) {
        const int kt = u.t0 + wk + it * WK;
        wait_vmcnt<(NS - 2) * 2 * COPIES>();              // this wave's copies of the tile have landed
        tile_barrier<WM>();                        // the group's have; the stage before is free
        issue(min(kt + (NS - 1) * WK, last), stage == 0 ? NS - 1 : stage - 1, next);
        next = pages_of(min(kt + NS * WK, last));
        const int sb = ring + stage * STAGE;
        const uint32_t gone = (missing >> (2 * stage)) & 3;
        stage = stage + 1 == NS ? 0 : stage + 1;
        if (!busy) continue;
        const int k0 = kt * kTile;
        tile(k0 + kTile > clear || gone, k0, sb, gone);
    }

    wait_all_memory();                                    // no copy may still land in LDS
    l_run = both_sum(l_run);

    if constexpr (WK == 1) {
        if (!busy) return;
        const int row = wm * 32 + j;
        if (u.parts > 1) {                                // what is left of a row until its parts are joined
            if (row < rows) {
                float* p = a.part_o + ((int64_t)u.slot * a.rows_per_wg + row) * HD + 4 * g;
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<f32x4*>(p + n * 32 + 8 * i) =
                            f32x4{oacc[n][4 * i], oacc[n][4 * i + 1], oacc[n][4 * i + 2], oacc[n][4 * i + 3]};
                if (g == 0) a.part_ml[(int64_t)u.slot * a.rows_per_wg + row] = float2{m_run, l_run};
            }
            return;
        }
        // Rows that saw nothing: the sum is 0 and so is every product.
        const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
        uint16_t* orow = a.o + t * a.o_stride + head * HD;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            uint32_t p[4][2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[i][0] = pack2<F16>(oacc[n][4 * i] * inv, oacc[n][4 * i + 1] * inv);
                p[i][1] = pack2<F16>(oacc[n][4 * i + 2] * inv, oacc[n][4 * i + 3] * inv);
            }
            swap_halves16(p);
            if (row < rows) {
                uint16_t* dst = orow + n * 32 + 16 * g;
                *reinterpret_cast<u32x4*>(dst) = u32x4{p[0][0], p[0][1], p[2][0], p[2][1]};
                *reinterpret_cast<u32x4*>(dst + 8) = u32x4{p[1][0], p[1][1], p[3][0], p[3][1]};
            }
        }
        if (a.lse && g == 0 && row < rows) a.lse[t * a.n_heads + head] = log_sum(a, m_run, l_run);
    } else {
        // The wave groups' shares of the 32 rows, joined through LDS: each wave's
        // outputs in its own stages, 16-byte chunks turned by the row against bank
        // conflicts.
        constexpr int C4 = HD / 4;
        constexpr int ML = 32 * HD * 4;                   // maxima and sums behind the outputs
        static_assert(ML + 32 * 8 <= NS * STAGE, "a wave's outputs fit its stages");
        float* own = reinterpret_cast<float*>(smem + ring);
        auto ml = [&](int w, int row) -> float2& { return reinterpret_cast<float2*>(smem + w * NS * STAGE + ML)[row]; };
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4*>(own + j * HD + (((n * 8 + 2 * i + g) ^ (j & (C4 - 1))) << 2)) =
                    f32x4{oacc[n][4 * i], oacc[n][4 * i + 1], oacc[n][4 * i + 2], oacc[n][4 * i + 3]};
        if (g == 0) ml(wk, j) = float2{m_run, l_run};
        __syncthreads();
        for (int x = tid; x < rows * C4; x += 256) {
            const int row = x / C4, c4 = x % C4;
            float m = -INFINITY, l = 0.f;
#pragma unroll
            for (int w = 0; w < WK; ++w) m = fmaxf(m, ml(w, row).x);
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const float2 part = ml(w, row);
                const float f = part.x == m ? 1.f : __builtin_amdgcn_exp2f((part.x - m) * a.scale_log2);
                const f32x4 v = *reinterpret_cast<const f32x4*>(smem + w * NS * STAGE + (row * HD + ((c4 ^ (row & (C4 - 1))) << 2)) * 4);
                l += part.y * f;
                o += v * f;
            }
            if (u.parts > 1) {
                *reinterpret_cast<f32x4*>(a.part_o + ((int64_t)u.slot * a.rows_per_wg + row) * HD + c4 * 4) = o;
                if (c4 == 0) a.part_ml[(int64_t)u.slot * a.rows_per_wg + row] = float2{m, l};
            } else {
                const int pr = row + u.row_tile * a.rows_per_wg;
                const int64_t to = (int64_t)u.s.start + pr / a.group;
                const int h = u.kvh * a.group + pr % a.group;
                store_out<F16>(a, to, h, c4 * 4, HD, o, l == 0.f ? 0.f : 1.f / l);
                if (a.lse && c4 == 0) a.lse[to * a.n_heads + h] = log_sum(a, m, l);
            }
        }
    }
}

// The parts of an item's rows, joined in order: blockIdx.x the item, blockIdx.y a
// group of rows; a thread takes 4 features of a row.
template <bool F16, int HD>
__global__ __launch_bounds__(256) void join_kernel(const AttnArgs a) {
    constexpr int C4 = HD / 4;
    Unit u;
    if (!find_unit<true>(a, blockIdx.x, u)) return;
    const int rows = min(u.s.n * a.group - u.row_tile * a.rows_per_wg, a.rows_per_wg);
    const int row = blockIdx.y * (256 / C4) + threadIdx.x / C4, c4 = threadIdx.x % C4;
    if (row >= rows) return;
    const float2* ml = a.part_ml + (int64_t)u.slot * a.rows_per_wg + row;
    const float* po = a.part_o + ((int64_t)u.slot * a.rows_per_wg + row) * HD + c4 * 4;
    float m = -INFINITY;
#pragma unroll 4
    for (int p = 0; p < u.parts; ++p) m = fmaxf(m, ml[(int64_t)p * a.rows_per_wg].x);
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int p = 0; p < u.parts; ++p) {
        const float2 part = ml[(int64_t)p * a.rows_per_wg];
        const f32x4 v = *reinterpret_cast<const f32x4*>(po + (int64_t)p * a.rows_per_wg * HD);
        const float f = part.x == m ? 1.f : __builtin_amdgcn_exp2f((part.x - m) * a.scale_log2);
        l += part.y * f;
        o += v * f;
    }
    const int pr = row + u.row_tile * a.rows_per_wg;
    const int64_t t = (int64_t)u.s.start + pr / a.group;
    const int h = u.kvh * a.group + pr % a.group;
    store_out<F16>(a, t, h, c4 * 4, HD, o, l == 0.f ? 0.f : 1.f / l);
    if (a.lse && c4 == 0) a.lse[t * a.n_heads + h] = log_sum(a, m, l);
}

// How a call is laid out: packed rows of a workgroup, keys of a step, units.
struct Shape {
    int rows_per_wg, step, units, min_steps;
};
Shape shape_for(int max_rows, int group) {
    // Up to 32 packed rows: one wave's worth, so the four waves of a workgroup take
    // different keys.  More: 32 rows per wave, keys shared.
    if ((int64_t)max_rows * group <= 32) return {32, 4 * kTile, 256, 2};
    return {128, kTile, 512, 4};
}
int64_t item_bound(int n_seqs, int n_kv, int total_rows, int max_rows, int group, int rows_per_wg) {
    const int64_t per_seq = ((int64_t)max_rows * group + rows_per_wg - 1) / rows_per_wg;
    return n_kv * std::min<int64_t>(n_seqs * per_seq, (int64_t)total_rows * group / rows_per_wg + n_seqs);
}
size_t round256(size_t n) { return (n + 255) / 256 * 256; }

template <bool F16, int HD>
hipError_t launch(const AttnArgs& a, int64_t items, bool may_split, hipStream_t st) {
    const int64_t wgs = (items + (may_split ? a.units : 0) + 63) / 64 * 64;
    if (wgs > 0x7fffffff) return hipErrorInvalidValue;
    if (a.rows_per_wg == 32)
        hipLaunchKernelGGL((attend_kernel<F16, HD, 4, HD == 128 ? 2 : 4, 1>), dim3((unsigned)wgs), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((attend_kernel<F16, HD, 1, 3, 3>), dim3((unsigned)wgs), dim3(256), 0, st, a);
    if (may_split) {
        const int rows = (int)std::min<int64_t>(a.rows_per_wg, (int64_t)a.max_rows * a.group), per = 256 / (HD / 4);
        hipLaunchKernelGGL((join_kernel<F16, HD>), dim3((unsigned)std::min<int64_t>(items, a.units), (rows + per - 1) / per),
                           dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

}  // namespace

// Split items have at least two parts of which all but one are full, so they make
// at most twice the units aimed at.
size_t attend_workspace_bytes(int n_seqs, int n_kv, int head_dim, int total_rows, int max_rows, int group) {
    (void)n_seqs, (void)n_kv, (void)total_rows;
    const Shape s = shape_for(max_rows, group);
    const size_t rows = (size_t)2 * s.units * s.rows_per_wg;
    return round256(rows * head_dim * 4) + round256(rows * 8);
}

hipError_t launch_attend(const CacheArgs& c, int dtype, int layer, const int32_t* row_start, int total_rows,
                         int max_rows, int max_keys, int n_heads, const void* q, int64_t q_stride,
                         const uint32_t* mask, int mask_words, float scale, void* o, int64_t o_stride, float* lse,
                         void* ws, hipStream_t st) {
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
    a.mask_words = mask_words;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.o = (uint16_t*)o;
    a.o_stride = o_stride;
    a.lse = lse;
    const Shape s = shape_for(max_rows, a.group);
    a.rows_per_wg = s.rows_per_wg;
    a.step = s.step;
    a.units = s.units;
    a.min_steps = s.min_steps;
    const size_t rows = (size_t)2 * s.units * s.rows_per_wg;
    a.part_o = (float*)ws;
    a.part_ml = (float2*)((char*)ws + round256(rows * c.head_dim * 4));
    const int64_t items = item_bound(c.n_seqs, c.n_kv, total_rows, max_rows, a.group, s.rows_per_wg);
    const int64_t steps = ((int64_t)max_keys + s.step - 1) / s.step;
    if (items * std::max<int64_t>(steps, 1) > 0x3fffffff) return hipErrorInvalidValue;    // the units' counts are 32-bit
    const bool may_split = steps > s.min_steps;
    if (dtype == DLM_F16)
        return c.head_dim == 128 ? launch<true, 128>(a, items, may_split, st) : launch<true, 64>(a, items, may_split, st);
    return c.head_dim == 128 ? launch<false, 128>(a, items, may_split, st) : launch<false, 64>(a, items, may_split, st);
}
