// Device helpers of the kernels around the paged cache: where a slot lies, rows of sixteen elements, the rotation.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_params.h"
#include "kernel_common.h"

namespace intattn {

__device__ __forceinline__ bool good_cache_scale(float s) { return s > 0.0f && s < __builtin_inff(); } // false for NaN

// lens[b], kept inside what the sequence can have
__device__ __forceinline__ int cache_len(const CacheParams &c, int b) { return min(max(c.lens[b], 0), c.capacity); }

// new tokens of sequence b of length n; a null pointer: as many as there can be
__device__ __forceinline__ int new_tokens(const int32_t *n_new, int b, int L, int n) { return min(max(n_new ? n_new[b] : L, 0), min(L, n)); }

// page and place in it of a slot below the capacity; the page is negative where it is not there
struct Slot {
    int page, at;
};
__device__ __forceinline__ Slot find_slot(const CacheParams &c, const int32_t *row, int slot)
{
    const int n = quotient(slot, c.by_page);
    const int page = row[n];
    return Slot{(uint32_t)page < (uint32_t)c.n_pages ? page : -1, slot - n * c.page_size};
}

// ------------------------------------------------------------------ rows in lanes of sixteen elements
// A lane takes 16 channels of a row: 16 u .. 16 u + 15, or, where the rotation pairs channel i with i + rot / 2, the eight pairs
// from i = 8 u on.  Pairs sit next to each other in x, so x[2 j], x[2 j + 1] are turned by the angle of pair 8 u + j in either
// layout.  Channels from rot on are in order in both.
struct Unit {
    int first, second; // channel of the first eight elements in memory and of the other eight
    bool halves;       // pairs straddle the two
};
__device__ __forceinline__ Unit unit_of(int u, int rot, bool halves)
{
    const bool split = halves && 16 * u < rot;
    return Unit{split ? 8 * u : 16 * u, split ? rot / 2 + 8 * u : 16 * u + 8, split};
}

template <int DTYPE> struct Raw16 {
    uint4 v[DTYPE == 0 ? 4 : 2];
};
template <int DTYPE> __device__ __forceinline__ Raw16<DTYPE> load_unit(const uint8_t *row, const Unit &u)
{
    constexpr int ES = DTYPE == 0 ? 4 : 2, N = DTYPE == 0 ? 2 : 1;
    Raw16<DTYPE> r;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        r.v[i] = *(const uint4 *)(row + (int64_t)u.first * ES + 16 * i);
        r.v[N + i] = *(const uint4 *)(row + (int64_t)u.second * ES + 16 * i);
    }
    return r;
}
// element i of the unit in memory order, in fp32 (exact)
template <int DTYPE> __device__ __forceinline__ float raw_element(const Raw16<DTYPE> &r, int i)
{
    constexpr int PER = DTYPE == 0 ? 4 : 8;
    const uint4 v = r.v[i / PER];
    const int j = i % PER;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (DTYPE == 0) return __uint_as_float(w[j]);
    else if constexpr (DTYPE == 1) return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[j / 2] >> (16 * (j & 1))));
    else return __uint_as_float((j & 1) ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
}

// ------------------------------------------------------------------ rotation
// Cosine and sine of pair i at token l of sequence b.  The angle is one product in 64 bits, and reducing and evaluating it there
// keeps far positions exact: at position 10^6 a 32-bit angle would be off by 0.03.
__device__ __forceinline__ double2 turn_of(const RotaryParams &r, int b, int l, int i)
{
    const int axis = (r.axis[i >> 2] >> (8 * (i & 3))) & 0xff;
    const double angle = (double)r.pos[axis * r.ps[0] + b * r.ps[1] + l * r.ps[2]] * r.freq[i];
    double s, c;
    sincos(angle, &s, &c);
    return make_double2(c, r.inverse ? -s : s);
}

// Both results in 64 bits, rounded once: a rotated row does not depend on how products are joined, and the integers that are made
// of it later are the definition's.
__device__ __forceinline__ void turn_pair(float &a, float &b, const double2 t)
{
    const double x = a, y = b;
    a = (float)(x * t.x - y * t.y);
    b = (float)(x * t.y + y * t.x);
}

// x in pair order from a unit in memory, turned if the unit is rotated; turns: those of the token's pairs
template <int DTYPE>
__device__ __forceinline__ void widen_unit(const Raw16<DTYPE> &raw, const Unit &un, bool rotated, const double2 *turns, int u, float (&x)[16])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float e0 = raw_element<DTYPE>(raw, 2 * j), e1 = raw_element<DTYPE>(raw, 2 * j + 1);
        const float h0 = raw_element<DTYPE>(raw, j), h1 = raw_element<DTYPE>(raw, 8 + j);
        x[2 * j] = un.halves ? h0 : e0;
        x[2 * j + 1] = un.halves ? h1 : e1;
    }
    if (rotated) {
#pragma unroll
        for (int j = 0; j < 8; ++j) turn_pair(x[2 * j], x[2 * j + 1], turns[8 * u + j]);
    }
}

} // namespace intattn
