// Rotary positions with up to four axes on one or two tensors, for gfx950:
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = pos[axis] * freq,
// for each pair of a row's first `rot` channels.  Every element is read and written once, so a large call is bound by HBM.  A
// workgroup takes a few tokens with all their heads, so that the angles of a token, which all heads share, are evaluated once
// (in 64 bits: cache_common.h) and lie in LDS; the first rows are asked for before.
#include "cache_common.h"
#include "work_map.h"

namespace intattn {

namespace {

constexpr int RNT = 256, TOKENS = 64;

template <int DTYPE> __device__ __forceinline__ void store_unit(uint8_t *row, const Unit &un, const float (&x)[2 * HALF<DTYPE>])
{
    constexpr int ES = DTYPE == 0 ? 4 : 2, N = HALF<DTYPE>;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DTYPE == 0) {
                w[i] = __float_as_uint(x[N * h + i]);
            } else if constexpr (DTYPE == 1) {
                w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[N * h + 2 * i]) | ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[N * h + 2 * i + 1]) << 16);
            } else {
                w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[N * h + 2 * i]) | ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[N * h + 2 * i + 1]) << 16);
            }
        }
        // (past the caches: Q and K of 8192 tokens, bf16, 40 heads, 36.0 -> 31.1 us)
        __builtin_nontemporal_store(v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]}, (v4i *)(row + (h ? un.second : un.first) * ES));
    }
}

template <int DTYPE, bool HALVES> __global__ __launch_bounds__(RNT) void rope_kernel(const RopeParams p)
{
    constexpr int N = HALF<DTYPE>;
    extern __shared__ double2 turns[]; // [tokens][rot / 2]
    const int pairs = p.r.rot / 2, t0 = blockIdx.x * p.tokens, n = min(p.tokens, p.B * p.L - t0);
    const int items = n * p.per_token;
    struct Item {
        Unit un;
        int64_t src, dst; // offsets in tensor w
        int w, t;
    };
    auto item = [&](int i) {
        Item it;
        it.t = quotient(i, p.by_token);
        const int in = i - it.t * p.per_token, h = quotient(in, p.by_units);
        it.w = h >= p.H0;
        const int head = h - (it.w ? p.H0 : 0), b = quotient(t0 + it.t, p.by_L), l = t0 + it.t - b * p.L;
        it.un = unit_of<DTYPE, HALVES>(in - h * p.units, p.d, p.r.rot);
        const int64_t *s = p.ss[it.w], *d = p.ds[it.w];
        it.src = b * s[0] + head * s[1] + l * s[2];
        it.dst = b * d[0] + head * d[1] + l * d[2];
        return it;
    };
    int i = threadIdx.x + blockIdx.y * RNT;
    Item it = item(min(i, items - 1));
    Raw raw = load_unit<DTYPE>(p.src[it.w] + it.src, it.un);
    for (int k = threadIdx.x; k < n * pairs; k += RNT) {
        const int t = quotient(k, p.by_pairs), b = quotient(t0 + t, p.by_L);
        turns[k] = turn_of(p.r, b, t0 + t - b * p.L, k - t * pairs);
    }
    __syncthreads();
    const int step = RNT * gridDim.y;
    while (i < items) {
        float x[2 * N];
        widen<DTYPE>(raw, x);
        const Item now = it;
        i += step;
        if (i < items) {
            it = item(i);
            raw = load_unit<DTYPE>(p.src[it.w] + it.src, it.un);
        }
        turn_unit<DTYPE, HALVES>(x, now.un, turns + now.t * pairs);
        store_unit<DTYPE>(p.dst[now.w] + now.dst, now.un, x);
    }
}

} // namespace

int launch_rope(const RopeParams &p_, int dtype, void *stream)
{
    RopeParams p = p_;
    const int64_t all = (int64_t)p.B * p.L;
    p.units = p.d / (dtype == 0 ? 8 : 16);
    p.per_token = p.H * p.units;
    p.by_token = fast_div((uint32_t)p.per_token);
    p.by_units = fast_div((uint32_t)p.units);
    p.by_pairs = fast_div((uint32_t)(p.r.rot / 2));
    p.by_L = fast_div((uint32_t)p.L);
    // tokens of a workgroup where there are enough (8192 tokens of 40 heads, d 128, us: fp32, one 59.4, four 68.2; bf16, one 34.0, two 32.2,
    // four 33.0; 128 000 tokens of 2 heads, fp32, d 64, two 97.9, 20 38.6); the heads of a
    // token over several workgroups where there are few (8 tokens 3.5 us, in one workgroup each 4.0; 64 tokens 3.7, 4.2)
    p.tokens = tokens_of(all, p.per_token, 2, p.r.rot, TOKENS);
    const int64_t blocks = (all + p.tokens - 1) / p.tokens, rounds = ((int64_t)p.tokens * p.per_token + RNT - 1) / RNT;
    const int64_t parts = blocks >= 512 ? 1 : std::min<int64_t>(rounds, std::max<int64_t>(1, 512 / blocks));
    const size_t lds = sizeof(double2) * (size_t)p.tokens * (size_t)(p.r.rot / 2);
    void (*kernel)(const RopeParams) = p.r.halves ? (dtype == 0 ? rope_kernel<0, true> : dtype == 1 ? rope_kernel<1, true> : rope_kernel<2, true>)
                                                  : (dtype == 0 ? rope_kernel<0, false> : dtype == 1 ? rope_kernel<1, false> : rope_kernel<2, false>);
    hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks, (uint32_t)parts), dim3(RNT), lds, (hipStream_t)stream, p);
    return (int)hipGetLastError();
}

} // namespace intattn
