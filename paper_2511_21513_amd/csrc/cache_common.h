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

// Tokens of a workgroup whose lanes take `items` pieces of each: up to `few` in three rounds of 256 lanes, or what fills one, with at
// most 1024 angles, and 512 workgroups left.
inline int tokens_of(int64_t tokens, int items, int few, int rot, int most)
{
    const int three = 768 / items < few ? 768 / items : few, one = 320 / items, angles = rot > 0 ? 2048 / rot : most;
    int64_t n = three > one ? three : one;
    n = n < angles ? n : angles;
    n = n < tokens / 512 ? n : tokens / 512;
    return (int)(n < 1 ? 1 : n < most ? n : most);
}

// ------------------------------------------------------------------ rows in lanes
// A lane takes 32 bytes of a row, two runs of HALF channels: HALF u and on of either half of the row, or, where the rotation pairs
// channel i with i + rot / 2, of either half of the rotated channels (so that a lane has both of each pair) and then of the others.
// The runs of neighbouring lanes follow each other: 32 bytes in one piece to a lane took a twentieth longer.
template <int DTYPE> constexpr int HALF = DTYPE == 0 ? 4 : 8;

struct Unit {
    int first, second;    // channels where the two runs start
    bool turn[2];         // whether they are rotated
};
// rot: rotated channels of this row (0: none)
template <int DTYPE, bool HALVES> __device__ __forceinline__ Unit unit_of(int u, int d, int rot)
{
    constexpr int N = HALF<DTYPE>;
    const int at = N * u;
    if constexpr (HALVES) {
        const bool in = 2 * at < rot;
        return Unit{in ? at : rot / 2 + at, in ? rot / 2 + at : d / 2 + at, {in, in}};
    } else {
        return Unit{at, d / 2 + at, {at < rot, d / 2 + at < rot}};
    }
}

struct Raw {
    v4i v[2];
};
template <int DTYPE> __device__ __forceinline__ Raw load_unit(const uint8_t *row, const Unit &u)
{
    constexpr int ES = DTYPE == 0 ? 4 : 2;
    return Raw{__builtin_nontemporal_load((const v4i *)(row + u.first * ES)), __builtin_nontemporal_load((const v4i *)(row + u.second * ES))};
}
// the elements in memory order, in fp32 (exact)
template <int DTYPE> __device__ __forceinline__ void widen(const Raw &r, float (&x)[2 * HALF<DTYPE>])
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t w[4] = {(uint32_t)r.v[h][0], (uint32_t)r.v[h][1], (uint32_t)r.v[h][2], (uint32_t)r.v[h][3]};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DTYPE == 0) {
                x[4 * h + i] = __uint_as_float(w[i]);
            } else if constexpr (DTYPE == 1) {
                x[8 * h + 2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i] & 0xffffu));
                x[8 * h + 2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i] >> 16));
            } else {
                x[8 * h + 2 * i] = __uint_as_float(w[i] << 16);
                x[8 * h + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
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

// A unit's pairs turned; turns: those of the token's pairs.  Both results in 64 bits, rounded once: a rotated row does not depend on how
// products are joined, and the integers that are made of it later are the definition's.
__device__ __forceinline__ void turn_pair(float &a, float &b, const double2 t)
{
    const double x = a, y = b;
    a = (float)(x * t.x - y * t.y);
    b = (float)(x * t.y + y * t.x);
}
template <int DTYPE, bool HALVES> __device__ __forceinline__ void turn_unit(float (&x)[2 * HALF<DTYPE>], const Unit &un, const double2 *turns)
{
    constexpr int N = HALF<DTYPE>;
    if constexpr (HALVES) {
        if (!un.turn[0]) return;
#pragma unroll
        for (int j = 0; j < N; ++j) turn_pair(x[j], x[N + j], turns[un.first + j]);
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (!un.turn[h]) continue;
#pragma unroll
            for (int j = 0; j < N / 2; ++j) turn_pair(x[N * h + 2 * j], x[N * h + 2 * j + 1], turns[(h ? un.second : un.first) / 2 + j]);
        }
    }
}

} // namespace intattn
