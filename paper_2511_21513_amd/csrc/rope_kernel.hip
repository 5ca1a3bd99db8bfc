// Rotary positions with up to four axes on one or two tensors, for gfx950:
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = pos[axis] * freq,
// for each pair of a row's first `rot` channels.  Every element is read and written once, so a large call is bound by HBM.  A
// workgroup takes a few tokens with all their heads, so that the angles of a token, which all heads share, are evaluated once
// (in 64 bits: cache_common.h) and lie in LDS.
#include "cache_common.h"

namespace intattn {

namespace {

constexpr int RNT = 256;

template <int DTYPE> __device__ __forceinline__ void store_unit(uint8_t *row, const Unit &un, const float (&x)[16])
{
    constexpr int ES = DTYPE == 0 ? 4 : 2;
    float m[16]; // in memory order
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        m[j] = un.halves ? x[2 * j] : x[j];
        m[8 + j] = un.halves ? x[2 * j + 1] : x[8 + j];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint8_t *at = row + (int64_t)(h ? un.second : un.first) * ES;
        if constexpr (DTYPE == 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                *(float4 *)(at + 16 * i) = make_float4(m[8 * h + 4 * i], m[8 * h + 4 * i + 1], m[8 * h + 4 * i + 2], m[8 * h + 4 * i + 3]);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint16_t lo, hi;
                if constexpr (DTYPE == 1) {
                    lo = __builtin_bit_cast(uint16_t, (_Float16)m[8 * h + 2 * i]);
                    hi = __builtin_bit_cast(uint16_t, (_Float16)m[8 * h + 2 * i + 1]);
                } else {
                    lo = __builtin_bit_cast(uint16_t, (__bf16)m[8 * h + 2 * i]);
                    hi = __builtin_bit_cast(uint16_t, (__bf16)m[8 * h + 2 * i + 1]);
                }
                w[i] = (uint32_t)lo | ((uint32_t)hi << 16);
            }
            *(uint4 *)at = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

template <int DTYPE> __global__ __launch_bounds__(RNT) void rope_kernel(const RopeParams p)
{
    extern __shared__ double2 turns[]; // [tokens][rot / 2]
    const int pairs = p.r.rot / 2;
    const int64_t all = (int64_t)p.B * p.L, t0 = (int64_t)blockIdx.x * p.tokens;
    const int n = (int)min((int64_t)p.tokens, all - t0);
    for (int i = threadIdx.x; i < n * pairs; i += RNT) {
        const int64_t t = t0 + i / pairs;
        turns[i] = turn_of(p.r, (int)(t / p.L), (int)(t % p.L), i % pairs);
    }
    __syncthreads();
    const int units = p.d / 16, items = n * p.H * units;
    for (int i = threadIdx.x; i < items; i += RNT) {
        const int u = i % units, row = i / units, h = row % p.H, t = row / p.H;
        const int b = (int)((t0 + t) / p.L), l = (int)((t0 + t) % p.L);
        const int w = h >= p.H0, head = h - (w ? p.H0 : 0);
        const Unit un = unit_of(u, p.r.rot, p.r.halves);
        const Raw16<DTYPE> raw = load_unit<DTYPE>(p.src[w] + b * p.ss[w][0] + head * p.ss[w][1] + l * p.ss[w][2], un);
        float x[16];
        widen_unit<DTYPE>(raw, un, 16 * u < p.r.rot, turns + t * pairs, u, x);
        store_unit<DTYPE>(p.dst[w] + b * p.ds[w][0] + head * p.ds[w][1] + l * p.ds[w][2], un, x);
    }
}

} // namespace

int launch_rope(const RopeParams &p_, int dtype, void *stream)
{
    RopeParams p = p_;
    const int64_t all = (int64_t)p.B * p.L;
    p.tokens = 1;
    const int64_t blocks = (all + p.tokens - 1) / p.tokens;
    const size_t lds = sizeof(double2) * (size_t)p.tokens * (size_t)(p.r.rot / 2);
    void (*kernel)(const RopeParams) = dtype == 0 ? rope_kernel<0> : dtype == 1 ? rope_kernel<1> : rope_kernel<2>;
    hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(RNT), lds, (hipStream_t)stream, p);
    return (int)hipGetLastError();
}

} // namespace intattn
