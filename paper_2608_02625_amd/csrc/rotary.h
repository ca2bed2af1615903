// What the kernels that rotate rows share (rope.hip, head_norm.hip): angles from
// integer phases, vector accesses, the widest access that a call's layout allows.
#pragma once

#include "common.h"
#include "cache.h"

namespace {

__device__ __forceinline__ void turn_sincos(uint64_t phase, float& s, float& c) {
    const uint64_t t = phase + (1ull << 61);
    const int quad = (int)(t >> 62);
    // signed distance from the quadrant's centre: 2^31 is an eighth of a turn
    const int32_t r = (int32_t)(((int64_t)(t & ((1ull << 62) - 1)) - (1ll << 61)) >> 30);
    float s0, c0;
    sincospif((float)r * 0x1p-33f, &s0, &c0);
    s = quad & 1 ? c0 : s0;
    c = quad & 1 ? s0 : c0;
    if (quad == 1 || quad == 2) c = -c;
    if (quad >= 2) s = -s;
}

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<__bf16>(__bf16 v) { return (float)v; }
template <>
__device__ __forceinline__ float to_f32<_Float16>(_Float16 v) { return (float)v; }
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }

template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
    T v[N];
};
// V neighbouring pairs.  A single one (V = 1) is what is left where rows lie anywhere, so it
// asks for no more than its elements' alignment (pairs_per_access has checked wider ones).
template <typename T, int V>
struct alignas(sizeof(T) * (V == 1 ? 1 : 2 * V)) Pairs {
    T v[2 * V];
};
static_assert(alignof(Pairs<__bf16, 1>) == 2 && alignof(Pairs<float, 1>) == 4, "a pair at an odd element");
static_assert(alignof(Pairs<__bf16, 2>) == 8 && alignof(Pairs<float, 2>) == 16, "whole accesses");
// One access; STREAM: past the caches' replacement.
template <bool STREAM, typename V>
__device__ __forceinline__ V load(const void* p) {
    if constexpr (STREAM && sizeof(V) == 16) return __builtin_bit_cast(V, __builtin_nontemporal_load((const u32x4*)p));
    else if constexpr (STREAM && sizeof(V) == 8) return __builtin_bit_cast(V, __builtin_nontemporal_load((const u32x2*)p));
    else return *(const V*)p;
}
template <bool STREAM, typename V>
__device__ __forceinline__ void store(void* p, const V& v) {
    if constexpr (STREAM && sizeof(V) == 16) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4*)p);
    else if constexpr (STREAM && sizeof(V) == 8) __builtin_nontemporal_store(__builtin_bit_cast(u32x2, v), (u32x2*)p);
    else *(V*)p = v;
}

template <int V>
__device__ __forceinline__ void angles(const uint64_t* phase, float scale, int64_t pos, int o, bool back, float (&c)[V],
                                       float (&s)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        turn_sincos(phase[o + i] * (uint64_t)pos, s[i], c[i]);
        s[i] *= back ? -scale : scale;
        c[i] *= scale;
    }
}

// Whether a sequence other than b counts token t, in this page (shared pages stand in the
// same entry of every table row: they come from forks).
__device__ bool counted_elsewhere(const CacheArgs& c, int b, int64_t t, int page) {
    const int64_t entry = t >> c.page_log2;
    for (int s = 0; s < c.n_seqs; ++s)
        if (s != b && c.len[s] > t && c.table[(int64_t)s * c.max_pages + entry] == page) return true;
    return false;
}

// Whether accesses of n values of `elem` bytes stay aligned at p and on a stride
// (in elements).
bool fits(const void* p, int elem, int n, int64_t stride) {
    return (uintptr_t)p % ((size_t)n * elem) == 0 && stride % n == 0;
}
// Whether a call's bytes are too many for the 256 MB memory-side cache to keep any for
// the next kernel: then they go past it.  A copy of 2 x 160 MB runs at 5.6 TB/s, past
// the caches at 6.2; one of 2 x 32 MB (which stays cached) at 6.8 and 5.7.
bool streams(int64_t bytes) { return bytes >= (int64_t)128 << 20; }
// Most pairs per access: V values (half layout) or 2 V (interleaved) make at most
// 16 bytes of the wider type; `aligned(n)` tells whether accesses of n values are.
template <typename F>
int pairs_per_access(const dlm_rope& r, int elem, F aligned) {
    for (int V = 16 / elem / (r.interleaved ? 2 : 1); V > 1; V /= 2) {
        const int n = r.interleaved ? 2 * V : V;
        if ((r.rot_dim / 2) % V == 0 && (r.head_dim - r.rot_dim) % V == 0 && r.head_dim % n == 0 && aligned(n)) return V;
    }
    return 1;
}
// A grid has fewer than 2^32 threads along an axis.
constexpr int64_t kWgsAcross = 1 << 20;

}  // namespace
