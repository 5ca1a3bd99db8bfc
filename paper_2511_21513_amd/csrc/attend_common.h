// Device helpers of the kernels that attend over a paged cache: rows and their thresholds, where lanes find their keys, the product
// with V.  Layout of a step of 64 keys: v_mfma_i32_16x16x64_i8 with keys as rows and query rows as columns; lane (n, kb) =
// (lane % 16, lane / 16) gives 16 bytes of a key's row, and the four MFMA tiles take key 4 n + i each, so that lane (n, kb) holds
// the scores of row n for the 16 keys from 16 kb on, in order: exactly the bytes of the P operand of the product with V.  V is
// turned in registers: a lane reads d / 16 channels of its 16 keys, and v_perm makes them rows of keys for each channel.  Neither
// product passes LDS.
#pragma once
#include "cache_common.h"

namespace intattn {

namespace {

constexpr int HIDDEN = (int)0x80000000; // further below any row maximum than any clip threshold

struct RowParams {
    double factor;   // the double after top / c_int
    float unit;      // floating-point output of one step of the accumulator
    int32_t c_int;
    int32_t limit;   // slots that the row sees
    int32_t mult, shift;
};

// c_int, index factor and output of one row, with the host's arithmetic; false where a scale is unusable
__device__ __forceinline__ bool row_params(const AttendParams &p, int b, int head, int t, int kvh, RowParams &rp)
{
    const float sq = p.scale_q[((int64_t)b * p.Hq + head) * p.L + t];
    const float sk = p.c.scale_k[p.c.per_head ? kvh : 0], sv = p.c.scale_v[p.c.per_head ? kvh : 0];
    const float so = p.out_type == 3 && p.scale_out ? p.scale_out[p.out_per_head ? head : 0] : sv;
    bool ok = good_cache_scale(sq) && good_cache_scale(sk) && good_cache_scale(sv) && good_cache_scale(so);
    double c = 1.0;
    if (ok) {
        const double alpha = ((double)sq * (double)sk) / p.sqrt_d;
        c = __builtin_floor(p.clip / alpha + 0.5);
        if (!(c >= 1.0)) c = 1.0;
        if (c > 1073741824.0) c = 1073741824.0;
    }
    rp.c_int = (int32_t)c;
    rp.factor = __builtin_bit_cast(double, (uint64_t)__double_as_longlong((double)p.top / c) + 1ull);
    rp.unit = ok ? (float)((double)sv / 255.0) : 0.0f;
    rp.mult = 0;
    rp.shift = 31;
    if (ok && p.out_type == 3) {
        const double r = (double)sv / (255.0 * (double)so);
        int e = 0;
        const double m = __builtin_frexp(r, &e);
        long long M = __builtin_llround(m * 2147483648.0);
        if (M == 2147483648LL) {
            M = 1073741824LL;
            e += 1;
        }
        const int sh = 31 - e;
        if (!(r > 0.0) || sh < 1 || sh > 62) ok = false;
        else {
            rp.mult = (int32_t)M;
            rp.shift = sh;
        }
    }
    return ok;
}

// the four words that hold byte j of the words w[0 .. 3]
__device__ __forceinline__ void transpose4(const uint32_t w0, const uint32_t w1, const uint32_t w2, const uint32_t w3, uint32_t (&o)[4])
{
    const uint32_t a = __builtin_amdgcn_perm(w1, w0, 0x05010400u), b = __builtin_amdgcn_perm(w1, w0, 0x07030602u);
    const uint32_t c = __builtin_amdgcn_perm(w3, w2, 0x05010400u), d = __builtin_amdgcn_perm(w3, w2, 0x07030602u);
    o[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    o[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    o[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    o[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// Where lanes find their keys.  WHOLE: pages of a multiple of 16 keys, so that 16 keys from a multiple of 16 on lie in one.
// Keys past the end, and keys of pages that are not there, are read from the pool's first row (their probability is 0).
template <int D, bool WHOLE> struct Keys {
    const CacheParams &c;
    const int32_t *row;
    int64_t head_k, head_v;
    int n; // slots in use

    __device__ __forceinline__ Slot at(int slot) const
    {
        if (slot >= n) return Slot{-1, 0};
        const Slot s = find_slot(c, row, slot);
        return s.page < 0 ? Slot{-1, 0} : s;
    }
    // 16 bytes of each of the lane's four keys 4 m + i of the step, channels 16 kb + 64 j on; there[i]: the key's page is there
    __device__ __forceinline__ void load_k(int step, int lane, v4i (&a)[4][D / 64], bool (&there)[4]) const
    {
        const int m = lane & 15, kb = lane >> 4;
        Slot s[4];
        if constexpr (WHOLE) {
            s[0] = at(step * 64 + 4 * m);
#pragma unroll
            for (int i = 1; i < 4; ++i) s[i] = Slot{s[0].page, s[0].at + i};
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = at(step * 64 + 4 * m + i);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            there[i] = s[i].page >= 0;
            const int8_t *at_ = c.k + head_k + max(s[i].page, 0) * c.ks[0] + s[i].at * c.ks[2] + 16 * kb;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) a[i][j] = *(const v4i *)(at_ + 64 * j);
        }
    }
    // d / 16 channels, from d / 16 m on, of the lane's 16 keys
    __device__ __forceinline__ void load_v(int step, int lane, uint32_t (&v)[16][D / 64]) const
    {
        const int m = lane & 15, kb = lane >> 4;
        Slot s = at(step * 64 + 16 * kb + (WHOLE ? 0 : m));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            int page = max(s.page, 0), place = WHOLE ? s.at + i : s.at;
            if constexpr (!WHOLE) {
                page = __shfl(page, (lane & 48) + i);
                place = __shfl(place, (lane & 48) + i);
            }
            const int8_t *at_ = c.v + head_v + page * c.vs[0] + place * c.vs[2] + m * (D / 16);
            if constexpr (D == 128) {
                const uint2 w = *(const uint2 *)at_;
                v[i][0] = w.x;
                v[i][1] = w.y;
            } else {
                v[i][0] = *(const uint32_t *)at_;
            }
        }
    }
};

// P.V of a step: acc[c] is channels d / 16 r + c of MFMA row r.  P_hat is unsigned and the MFMA signed: a byte of 128 or more
// enters as P - 256, and where a wave holds one, 256 = 2 + 127 + 127 times V is added (kernel_common.h).
template <int D> __device__ __forceinline__ void step_pv(const uint32_t (&v)[16][D / 64], const v4i pf, v4i (&acc)[D / 16])
{
    v4i t[D / 16];
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            uint32_t o[4];
            transpose4(v[4 * g][j], v[4 * g + 1][j], v[4 * g + 2][j], v[4 * g + 3][j], o);
#pragma unroll
            for (int c = 0; c < 4; ++c) t[4 * j + c][g] = (int)o[c];
        }
#pragma unroll
    for (int c = 0; c < D / 16; ++c) acc[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(t[c], pf, acc[c], 0, 0, 0);
    if (__any(((pf[0] | pf[1] | pf[2] | pf[3]) & (int)0x80808080u) != 0)) {
        v4i two, big;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            two[g] = (int)(((uint32_t)pf[g] >> 6) & 0x02020202u);
            big[g] = (int)(((uint32_t)two[g] << 6) - ((uint32_t)two[g] >> 1)); // 127 in place of 2
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            acc[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(t[c], two, acc[c], 0, 0, 0);
            acc[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(t[c], big, acc[c], 0, 0, 0);
            acc[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(t[c], big, acc[c], 0, 0, 0);
        }
    }
}

// Q of row `row` of KV head kvh: 16 bytes of each 64 channels
template <int D> __device__ __forceinline__ void load_q(const AttendParams &p, int b, int kvh, int row, int kb, v4i (&qf)[D / 64])
{
#pragma unroll
    for (int j = 0; j < D / 64; ++j) qf[j] = v4i{0, 0, 0, 0};
    if (row < p.rows) {
        const int8_t *at = p.q + b * p.qs[0] + (int64_t)(kvh * p.group + row / p.L) * p.qs[1] + (row % p.L) * p.qs[2] + 16 * kb;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) qf[j] = *(const v4i *)(at + 64 * j);
    }
}

// scores of the lane's row for its 16 keys, sc[ii][i] that of key 16 kb + 4 ii + i; HIDDEN past the row's limit (left: what is left
// of it at the lane's first key) and where the page is not there
template <int D> __device__ __forceinline__ void step_scores(const v4i (&a)[4][D / 64], const bool (&there)[4], const v4i (&qf)[D / 64], int left, int kb, v4i (&sc)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v4i d = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < D / 64; ++j) d = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i][j], qf[j], d, 0, 0, 0);
#pragma unroll
        for (int ii = 0; ii < 4; ++ii) sc[ii][i] = d[ii];
    }
    uint32_t seen[4]; // bit m: key 4 m + i is there
#pragma unroll
    for (int i = 0; i < 4; ++i) seen[i] = ((uint32_t)__ballot(there[i]) & 0xffffu) >> (4 * kb);
#pragma unroll
    for (int ii = 0; ii < 4; ++ii)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[ii][i] = 4 * ii + i < left && ((seen[i] >> ii) & 1u) ? sc[ii][i] : HIDDEN;
}

// the table index of four scores (bytes of the result), and the sum of their entries
__device__ __forceinline__ uint32_t four_indices(const int4 x, int top, const RowParams &rp, const uint8_t *entry, int &sum)
{
    const int sc[4] = {x.x, x.y, x.z, x.w};
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t away = min((uint32_t)top - (uint32_t)sc[i], (uint32_t)rp.c_int);
        const uint32_t idx = (uint32_t)(int)__builtin_fma((double)(int)away, rp.factor, 0.5);
        sum += entry[idx];
        word |= idx << (8 * i);
    }
    return word;
}

// where row `row` of KV head kvh goes
__device__ __forceinline__ uint8_t *out_row(const AttendParams &p, int b, int kvh, int row)
{
    return p.out + b * p.os[0] + (int64_t)(kvh * p.group + row / p.L) * p.os[1] + (row % p.L) * p.os[2];
}

// sums over the 16 lanes of a row of lanes: lane n ends with the sum of their x[n]
__device__ __forceinline__ float scatter_sum16(float (&x)[16], int n)
{
#pragma unroll
    for (int h = 8; h >= 1; h /= 2) {
        const bool up = (n & h) != 0;
#pragma unroll
        for (int j = 0; j < h; ++j) {
            const float send = up ? x[j] : x[j + h], keep = up ? x[j + h] : x[j];
            x[j] = keep + __shfl_xor(send, h);
        }
    }
    return x[0];
}

__device__ __forceinline__ void store_out(const AttendParams &p, const RowParams &rp, uint8_t *at, int ch, int acc)
{
    if (p.out_type == 3) {
        at[ch] = (uint8_t)(int8_t)requant_any(acc, rp.mult, rp.shift);
        return;
    }
    const float x = (float)acc * rp.unit;
    if (p.out_type == 0) ((float *)at)[ch] = x;
    else if (p.out_type == 1) ((uint16_t *)at)[ch] = __builtin_bit_cast(uint16_t, (_Float16)x);
    else ((uint16_t *)at)[ch] = __builtin_bit_cast(uint16_t, (__bf16)x);
}

} // namespace

} // namespace intattn
