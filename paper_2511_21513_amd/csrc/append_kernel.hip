// New tokens into the paged cache, for gfx950: K rotated, K and V quantized with the cache's scales into their pages, Q rotated
// and quantized with a scale of its own for each token and head (Sec. 2.1, Eq. quant).  Every element is read once and leaves as
// one byte; a decoding step's call is bound by the latency of one launch.  A workgroup takes a few tokens with all their heads (the
// angles of a token are evaluated once), 32 bytes of a row to a lane, so that the maximum over a row of Q needs shuffles alone.
#include "cache_common.h"
#include "work_map.h"

namespace intattn {

namespace {

constexpr int ANT = 256;
constexpr int TOKENS = 64; // of a workgroup at most
constexpr int HEAD_BYTES = 32;

// Integers of x: rint of the IEEE fp32 quotient x / s, ties to even, clamped to +-127.  With r the reciprocal of s to one unit in the
// last place, y = fma(x, r, 128) is off the quotient + 128 by less than 2^-15 where that lies in a byte's range, so wherever y is farther
// than 2^-14 from every half-integer both round alike, and the conversion to an unsigned byte rounds to nearest even and saturates: six
// operations an element.  Units with an element nearer than that take the division, and scales whose reciprocal is no normal number.
template <int N> __device__ __forceinline__ void quantize(const float (&x)[N], float s, uint32_t (&w)[N / 4])
{
    const float r = __builtin_amdgcn_rcpf(s);
    float y[N], off = s >= 0x1p-100f && s <= 0x1p100f ? 0.0f : 1.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        y[i] = __builtin_fmaf(x[i], r, 128.0f);
        off = fmaxf(off, __builtin_fabsf(y[i] - __builtin_rintf(y[i])));
    }
    if (off > 0.5f - 6.103515625e-05f) {
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = __builtin_rintf(x[i] / s) + 128.0f;
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        uint32_t q = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) q = __builtin_amdgcn_cvt_pk_u8_f32(fmaxf(y[4 * i + j], 1.0f), j, q); // (-127 the least)
        w[i] = q ^ 0x80808080u;
    }
}

template <int D, int DTYPE, bool HALVES> __global__ __launch_bounds__(ANT) void append_kernel(const AppendParams p)
{
    constexpr int N = HALF<DTYPE>, UNITS = D / (2 * N), ROWS = ANT / UNITS;
    // What the rows of a token, and those of a head, share is formed once (with three strides of each of three tensors in every row the
    // kernel was bound by vector instructions, 390 to a unit, and loads of a row waited behind those of the next).
    struct Token {
        int64_t src[3], dst[3]; // Q, K, V: offset of the row of head 0; dst < 0: nothing is written
        int b, l, slot, order;
        bool there;
    };
    struct Head {
        const uint8_t *src;
        int8_t *dst;
        float scale; // K, V
        int which, head;
    };
    static_assert(sizeof(Head) <= HEAD_BYTES, "room for the heads");
    extern __shared__ char lds[]; // heads, turns [tokens][rot / 2]
    __shared__ Token token[TOKENS];
    Head *const head = (Head *)lds; // HEAD_BYTES apart
    double2 *const turns = (double2 *)(lds + p.turns_at);
    const int pairs = p.r.rot / 2, t0 = blockIdx.x * p.tokens, n = min(p.tokens, p.c.B * p.L - t0), rows = n * p.heads;
    const int u = threadIdx.x % UNITS;
    const Unit plain = unit_of<DTYPE, HALVES>(u, D, 0), turned = unit_of<DTYPE, HALVES>(u, D, p.r.rot);
    for (int h = threadIdx.x; h < p.heads; h += ANT) {
        const int which = h < p.Hq ? 0 : h < p.Hq + p.c.Hkv ? 1 : 2, at = h - (which == 0 ? 0 : which == 1 ? p.Hq : p.Hq + p.c.Hkv);
        Head to;
        to.src = p.x[which] + at * p.xs[which][1];
        to.dst = which == 0 ? p.q_out + at * p.qos[1] : which == 1 ? p.c.k + at * p.c.ks[1] : p.c.v + at * p.c.vs[1];
        to.scale = (which == 2 ? p.c.scale_v : p.c.scale_k)[p.c.per_head && which > 0 ? at : 0];
        to.which = which;
        to.head = at;
        head[h] = to;
    }
    if ((int)threadIdx.x >= ANT - n) { // (other threads than those with the first heads)
        const int i = threadIdx.x - (ANT - n), b = quotient(t0 + i, p.by_L), l = t0 + i - b * p.L;
        const int len = cache_len(p.c, b), fresh = new_tokens(p.n_new, b, p.L, len), slot = len - fresh + l;
        Token to;
        to.b = b;
        to.l = l;
        to.slot = slot;
        to.there = l < fresh;
        to.order = p.first ? p.first[b] + l : slot;
#pragma unroll
        for (int w = 0; w < 3; ++w) to.src[w] = b * p.xs[w][0] + l * p.xs[w][2];
        to.dst[0] = b * p.qos[0] + l * p.qos[2];
        to.dst[1] = to.dst[2] = -1;
        if (to.there) {
            const Slot at = find_slot(p.c, p.c.table + b * p.c.table_stride, slot);
            if (at.page >= 0) {
                to.dst[1] = at.page * p.c.ks[0] + at.at * p.c.ks[2];
                to.dst[2] = at.page * p.c.vs[0] + at.at * p.c.vs[2];
            }
        }
        token[i] = to;
    }
    for (int k = threadIdx.x; k < n * pairs; k += ANT) {
        const int t = quotient(k, p.by_pairs), b = quotient(t0 + t, p.by_L);
        turns[k] = turn_of(p.r, b, t0 + t - b * p.L, k - t * pairs);
    }
    __syncthreads();
    struct Row {
        int t, h, which;
        Raw raw;
    };
    auto ask = [&](int i) {
        Row r;
        r.t = quotient(i, p.by_heads);
        r.h = i - r.t * p.heads;
        r.which = head[r.h].which;
        r.raw = load_unit<DTYPE>(head[r.h].src + token[r.t].src[r.which], r.which < 2 ? turned : plain);
        return r;
    };
    const int step = ROWS * gridDim.y;
    int i = threadIdx.x / UNITS + blockIdx.y * ROWS;
    if (i >= rows) return;
    Row next = ask(i);
    while (i < rows) { // all lanes of a row alike
        const Row r = next;
        const Unit un = r.which < 2 ? turned : plain;
        float x[2 * N];
        widen<DTYPE>(r.raw, x);
        i += step;
        if (i < rows) next = ask(i);
        const Token &at = token[r.t];
        const Head &to = head[r.h];
        if (r.which < 2) turn_unit<DTYPE, HALVES>(x, turned, turns + r.t * pairs);
        float scale = to.scale;
        const int64_t place = at.dst[r.which];
        if (r.which == 0) {
            float m = 0.0f;
#pragma unroll
            for (int j = 0; j < 2 * N; ++j) {
                if (!at.there) x[j] = 0.0f; // padding
                m = fmaxf(m, __builtin_fabsf(x[j]));
            }
#pragma unroll
            for (int o = 1; o < UNITS; o *= 2) m = fmaxf(m, __shfl_xor(m, o));
            scale = fmaxf(m, 1e-12f) / 127.0f;
            if (u == 0) p.q_scale[((int64_t)at.b * p.Hq + to.head) * p.L + at.l] = at.there ? scale : 0.0f;
        } else if (r.which == 1 && u == 0 && at.there) {
            if (p.weight) p.weight[at.b * p.wst[0] + to.head * p.wst[1] + at.slot] = 0.0f;
            if (p.order) p.order[at.b * p.ost[0] + to.head * p.ost[1] + at.slot] = at.order;
        }
        if (place < 0) continue;
        int8_t *const dst = to.dst + place;
        uint32_t w[N / 2];
        quantize<2 * N>(x, scale, w);
        if (!good_cache_scale(scale)) {
#pragma unroll
            for (int j = 0; j < N / 2; ++j) w[j] = 0;
        }
        if constexpr (N == 8) {
            *(uint2 *)(dst + un.first) = make_uint2(w[0], w[1]);
            *(uint2 *)(dst + un.second) = make_uint2(w[2], w[3]);
        } else {
            *(uint32_t *)(dst + un.first) = w[0];
            *(uint32_t *)(dst + un.second) = w[1];
        }
    }
}

} // namespace

template <int D, bool HALVES> static auto append_kernel_of(int dtype)
{
    return dtype == 0 ? append_kernel<D, 0, HALVES> : dtype == 1 ? append_kernel<D, 1, HALVES> : append_kernel<D, 2, HALVES>;
}

int launch_append(const AppendParams &p_, int d, int dtype, void *stream)
{
    AppendParams p = p_;
    const int64_t all = (int64_t)p.c.B * p.L;
    p.heads = p.Hq + 2 * p.c.Hkv;
    p.by_heads = fast_div((uint32_t)p.heads);
    p.by_L = fast_div((uint32_t)p.L);
    p.by_pairs = fast_div((uint32_t)(p.r.rot > 0 ? p.r.rot / 2 : 1));
    // tokens of a workgroup where there are enough (8192 tokens, one, two, four and eight, us: d 128, 48 heads 40.6, 36.8, 38.2, 39.8; d 64,
    // 48 heads 28.7, 25.5, 24.1, 23.0; d 128, 8 heads 18.1, 14.8, 13.1, 12.8; 131 000 tokens, d 64, 3 heads 189, 100, 57.9, 41.9); the heads
    // of a token over several workgroups where there are few (32 tokens of 48 heads 5.4 us, in one workgroup each 6.1)
    const int units = d / (dtype == 0 ? 8 : 16), rows = ANT / units;
    p.tokens = tokens_of(all, p.heads * units, 4, p.r.rot, TOKENS);
    const int64_t blocks = (all + p.tokens - 1) / p.tokens, rounds = ((int64_t)p.tokens * p.heads + rows - 1) / rows;
    const int64_t parts = blocks >= 512 ? 1 : std::min<int64_t>(rounds, std::max<int64_t>(1, 512 / blocks));
    p.turns_at = p.heads * HEAD_BYTES;
    const size_t lds = (size_t)p.turns_at + sizeof(double2) * (size_t)p.tokens * (size_t)(p.r.rot / 2);
    void (*kernel)(const AppendParams) = d == 64 ? (p.r.halves ? append_kernel_of<64, true>(dtype) : append_kernel_of<64, false>(dtype))
                                                 : (p.r.halves ? append_kernel_of<128, true>(dtype) : append_kernel_of<128, false>(dtype));
    hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks, (uint32_t)parts), dim3(ANT), lds, (hipStream_t)stream, p);
    return (int)hipGetLastError();
}

} // namespace intattn
