// New tokens into the paged cache, for gfx950: K rotated, K and V quantized with the cache's scales into their pages, Q rotated
// and quantized with a scale of its own for each token and head (Sec. 2.1, Eq. quant).  Every element is read once and leaves as
// one byte; a large call is bound by HBM, a decoding step's by the latency of one launch.  A workgroup takes a few tokens with
// all their heads (the angles of a token are evaluated once), d / 16 lanes a row, so that the maximum over a row of Q needs
// shuffles alone.
#include "cache_common.h"

namespace intattn {

namespace {

constexpr int ANT = 256;

// nearest integer of the IEEE fp32 quotient, ties to even, clamped
__device__ __forceinline__ int quantized(float x, float s)
{
    return (int)fminf(fmaxf(__builtin_rintf(x / s), -127.0f), 127.0f);
}

template <int D, int DTYPE> __global__ __launch_bounds__(ANT) void append_kernel(const AppendParams p)
{
    constexpr int UNITS = D / 16;
    extern __shared__ double2 turns[]; // [tokens][rot / 2]
    const int pairs = p.r.rot / 2;
    const int64_t all = (int64_t)p.c.B * p.L, t0 = (int64_t)blockIdx.x * p.tokens;
    const int n = (int)min((int64_t)p.tokens, all - t0);
    for (int i = threadIdx.x; i < n * pairs; i += ANT) {
        const int64_t t = t0 + i / pairs;
        turns[i] = turn_of(p.r, (int)(t / p.L), (int)(t % p.L), i % pairs);
    }
    __syncthreads();
    const int heads = p.Hq + 2 * p.c.Hkv, rows = n * heads;
    const int u = threadIdx.x % UNITS;
    for (int row0 = 0; row0 < rows; row0 += ANT / UNITS) {
        const int row = row0 + threadIdx.x / UNITS;
        if (row >= rows) break; // all lanes of a row alike
        const int t = row / heads, h = row % heads;
        const int b = (int)((t0 + t) / p.L), l = (int)((t0 + t) % p.L);
        const int len = cache_len(p.c, b), fresh = new_tokens(p.n_new, b, p.L, len);
        const int which = h < p.Hq ? 0 : h < p.Hq + p.c.Hkv ? 1 : 2, head = h - (which == 0 ? 0 : which == 1 ? p.Hq : p.Hq + p.c.Hkv);
        const bool there = l < fresh;
        const bool rotated = which < 2 && 16 * u < p.r.rot;
        const Unit un = unit_of(u, which < 2 ? p.r.rot : 0, p.r.halves);
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.0f;
        if (there) {
            const Raw16<DTYPE> raw = load_unit<DTYPE>(p.x[which] + b * p.xs[which][0] + head * p.xs[which][1] + l * p.xs[which][2], un);
            widen_unit<DTYPE>(raw, un, rotated, turns + t * pairs, u, x);
        }
        float scale;
        int8_t *dst = nullptr;
        if (which == 0) {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) m = fmaxf(m, __builtin_fabsf(x[i]));
#pragma unroll
            for (int o = 1; o < UNITS; o *= 2) m = fmaxf(m, __shfl_xor(m, o));
            scale = fmaxf(m, 1e-12f) / 127.0f;
            if (u == 0) p.q_scale[((int64_t)b * p.Hq + head) * p.L + l] = there ? scale : 0.0f;
            dst = p.q_out + b * p.qos[0] + head * p.qos[1] + l * p.qos[2];
        } else {
            scale = (which == 1 ? p.c.scale_k : p.c.scale_v)[p.c.per_head ? head : 0];
            const int slot = len - fresh + l;
            if (there) {
                const Slot at = find_slot(p.c, p.c.table + b * p.c.table_stride, slot);
                if (at.page >= 0) {
                    const int64_t *s = which == 1 ? p.c.ks : p.c.vs;
                    dst = (which == 1 ? p.c.k : p.c.v) + at.page * s[0] + head * s[1] + at.at * s[2];
                }
                if (which == 1 && u == 0) {
                    if (p.weight) p.weight[b * p.wst[0] + head * p.wst[1] + slot] = 0.0f;
                    if (p.order) p.order[b * p.ost[0] + head * p.ost[1] + slot] = p.first ? p.first[b] + l : slot;
                }
            }
        }
        if (!dst) continue;
        const bool ok = good_cache_scale(scale);
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t a = ok ? (uint32_t)quantized(x[2 * j], scale) & 0xffu : 0u, c = ok ? (uint32_t)quantized(x[2 * j + 1], scale) & 0xffu : 0u;
            const int i0 = un.halves ? j : 2 * j, i1 = un.halves ? 8 + j : 2 * j + 1; // in memory order
            w[0] |= i0 / 4 == 0 ? a << (8 * (i0 % 4)) : 0u;
            w[1] |= i0 / 4 == 1 ? a << (8 * (i0 % 4)) : 0u;
            w[2] |= i0 / 4 == 2 ? a << (8 * (i0 % 4)) : 0u;
            w[3] |= i0 / 4 == 3 ? a << (8 * (i0 % 4)) : 0u;
            w[0] |= i1 / 4 == 0 ? c << (8 * (i1 % 4)) : 0u;
            w[1] |= i1 / 4 == 1 ? c << (8 * (i1 % 4)) : 0u;
            w[2] |= i1 / 4 == 2 ? c << (8 * (i1 % 4)) : 0u;
            w[3] |= i1 / 4 == 3 ? c << (8 * (i1 % 4)) : 0u;
        }
        *(uint2 *)(dst + un.first) = make_uint2(w[0], w[1]);
        *(uint2 *)(dst + un.second) = make_uint2(w[2], w[3]);
    }
}

} // namespace

int launch_append(const AppendParams &p_, int d, int dtype, void *stream)
{
    AppendParams p = p_;
    p.tokens = 1;
    const int64_t blocks = ((int64_t)p.c.B * p.L + p.tokens - 1) / p.tokens;
    const size_t lds = sizeof(double2) * (size_t)p.tokens * (size_t)(p.r.rot / 2);
    void (*kernel)(const AppendParams) = d == 64 ? (dtype == 0 ? append_kernel<64, 0> : dtype == 1 ? append_kernel<64, 1> : append_kernel<64, 2>)
                                                 : (dtype == 0 ? append_kernel<128, 0> : dtype == 1 ? append_kernel<128, 1> : append_kernel<128, 2>);
    hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(ANT), lds, (hipStream_t)stream, p);
    return (int)hipGetLastError();
}

} // namespace intattn
