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

constexpr int PROB = 68; // bytes of a row's probabilities in LDS: rows start in banks of their own
constexpr int HIDDEN = (int)0x80000000; // further below any row maximum than any clip threshold

struct RowScales {
    float q, k, v, out;
};
__device__ __forceinline__ RowScales row_scales(const AttendParams &p, int b, int head, int t, int kvh)
{
    RowScales s;
    s.q = p.scale_q[((int64_t)b * p.Hq + head) * p.L + t];
    s.k = p.c.scale_k[p.c.per_head ? kvh : 0];
    s.v = p.c.scale_v[p.c.per_head ? kvh : 0];
    s.out = p.out_type == 3 && p.scale_out ? p.scale_out[p.out_per_head ? head : 0] : s.v;
    return s;
}

// c_int, index factor and output of one row, with the host's arithmetic; false where a scale is unusable
__device__ __forceinline__ bool row_params(const AttendParams &p, const RowScales &s, RowParams &rp)
{
    const float sq = s.q, sk = s.k, sv = s.v, so = s.out;
    const bool ok = good_cache_scale(sq) && good_cache_scale(sk) && good_cache_scale(sv) && good_cache_scale(so);
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
        // past a multiplier's range the formula is simple: accumulators, below 2^17, stay below a half, or saturate from 1 on
        if (sh < 1) {
            rp.mult = 1 << 30;
            rp.shift = 1;
        } else if (sh <= 62) {
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

// Where lanes find their keys.  WHOLE: pages of a multiple of 16 keys whose rows follow each other, so that 16 keys from a multiple of 16
// on are one run of 16 d bytes: one look into the table, and offsets that are part of the instruction (with a stride that is not known
// the sixteen addresses of a step of V took 32 registers).  Keys past the end are read where the table says, which does not wait for
// the length, and keys of pages that are not there from the pool's first page (the probability of either is 0); what lies past the last
// slot that a sequence may have is read from its last key, or, where lanes read runs, from the start of its last run, which ends inside
// its page because the page's size is a multiple of the run's.  V that is read once
// is read in whole lines past the caches (8 KiB blocks in no order: 6.1 TB/s, 5.4 through them); half lines of K need the cache.
//
// find_*() asks the table, load_*() for the keys.  They are apart so that a loop can ask for the places of a step before it asks for the
// keys of an earlier one: loads come back in order, and a place asked for last could only be waited for together with every key
// that is on its way.  (Scalar loads, which are counted apart, miss their cache too often: 4.6 -> 6.4 us for the first launch on 700 keys.)
// Every address that is formed for K and V comes from find_k(), find_v(), k_offset() and v_offset(), which the host can call as well.
template <int D, bool WHOLE> struct Keys {
    const CacheParams &c;
    const int32_t *row;
    int64_t head_k, head_v;

    struct Place {
        int entry, at; // of the table, as it is; place in the page
    };
    struct PlaceK {
        Place p[WHOLE ? 1 : 4];
    };
    // of a slot that is a multiple of RUN, a power of two: the first of as many keys that the lane reads from there
    template <int RUN> __host__ __device__ __forceinline__ Place find(int slot) const
    {
        const int last = (c.capacity - 1) & -RUN;
        slot = slot < last ? slot : last;
        const int n = quotient(slot, c.by_page);
        return Place{row[n], slot - n * c.page_size};
    }
    __host__ __device__ __forceinline__ bool there(const Place &p) const { return (uint32_t)p.entry < (uint32_t)c.n_pages; }
    // the lane's four keys 4 m + i of the step
    __host__ __device__ __forceinline__ PlaceK find_k(int step, int lane) const
    {
        PlaceK k;
#pragma unroll
        for (int i = 0; i < (WHOLE ? 1 : 4); ++i) k.p[i] = find<WHOLE ? 4 : 1>(step * 64 + 4 * (lane & 15) + i);
        return k;
    }
    // the lane's sixteen keys from 16 kb on; not WHOLE: key 16 kb + m of them
    __host__ __device__ __forceinline__ Place find_v(int step, int lane) const { return find<WHOLE ? 16 : 1>(step * 64 + 16 * (lane >> 4) + (WHOLE ? 0 : lane & 15)); }

    // bytes from the pool's first to the first 16 (and, 64 further, the second) of key i of the lane's four
    __host__ __device__ __forceinline__ int64_t k_offset(const PlaceK &k, int i, int lane) const
    {
        const Place &p = k.p[WHOLE ? 0 : i];
        const bool is = there(p);
        return head_k + (is ? p.entry : 0) * c.ks[0] + (is ? p.at : 0) * (WHOLE ? D : c.ks[2]) + 16 * (lane >> 4) + (WHOLE ? i * D : 0);
    }
    // and to the lane's channels of the key at this place of this page, which are there; WHOLE: of the first of a run of sixteen, D bytes apart
    __host__ __device__ __forceinline__ int64_t v_offset(int page, int at, int lane) const
    {
        return head_v + page * c.vs[0] + at * (WHOLE ? D : c.vs[2]) + (lane & 15) * (D / 16);
    }

    // 16 bytes of each of the lane's four keys, channels 16 kb + 64 j on; is[i]: the key's page is there
    __device__ __forceinline__ void load_k(const PlaceK &k, int lane, v4i (&a)[4][D / 64], bool (&is)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            is[i] = there(k.p[WHOLE ? 0 : i]);
            const int8_t *from = c.k + k_offset(k, i, lane);
#pragma unroll
            for (int j = 0; j < D / 64; ++j) a[i][j] = *(const v4i *)(from + 64 * j);
        }
    }
    // d / 16 channels, from d / 16 m on, of the lane's 16 keys; ONCE: no other workgroup reads them
    template <bool ONCE = true> __device__ __forceinline__ void load_v(const Place &p, int lane, uint32_t (&v)[16][D / 64]) const
    {
        const bool is = there(p);
        const int page = is ? p.entry : 0, at = is ? p.at : 0;
        const int8_t *const from = c.v + (WHOLE ? v_offset(page, at, lane) : 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int8_t *key = from + i * D;
            if constexpr (!WHOLE) key = from + v_offset(__shfl(page, (lane & 48) + i), __shfl(at, (lane & 48) + i), lane);
            if constexpr (D == 128) {
                v2i w;
                if constexpr (ONCE) w = __builtin_nontemporal_load((const v2i *)key);
                else w = *(const v2i *)key;
                v[i][0] = (uint32_t)w[0];
                v[i][1] = (uint32_t)w[1];
            } else {
                if constexpr (ONCE) v[i][0] = __builtin_nontemporal_load((const uint32_t *)key);
                else v[i][0] = *(const uint32_t *)key;
            }
        }
    }
};
inline bool whole_pages(const CacheParams &c, int d) { return c.page_size % 16 == 0 && c.ks[2] == d && c.vs[2] == d; }

// P.V of a step: acc[c] is channels d / 16 r + c of MFMA row r.  P_hat is unsigned and the MFMA signed: a byte of 128 or more
// enters as P - 256, and where a wave holds one, 256 = 2 + 127 + 127 times V is added (kernel_common.h).
template <int D> __device__ __forceinline__ void step_pv(const uint32_t (&v)[16][D / 64], const v4i pf, v4i (&acc)[D / 16])
{
    const bool big = __any(((pf[0] | pf[1] | pf[2] | pf[3]) & (int)0x80808080u) != 0);
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
        v4i t[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            uint32_t o[4];
            transpose4(v[4 * g][j], v[4 * g + 1][j], v[4 * g + 2][j], v[4 * g + 3][j], o);
#pragma unroll
            for (int c = 0; c < 4; ++c) t[c][g] = (int)o[c];
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[4 * j + c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(t[c], pf, acc[4 * j + c], 0, 0, 0);
        if (big) {
            v4i two, most;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                two[g] = (int)(((uint32_t)pf[g] >> 6) & 0x02020202u);
                most[g] = (int)(((uint32_t)two[g] << 6) - ((uint32_t)two[g] >> 1)); // 127 in place of 2
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                acc[4 * j + c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(t[c], two, acc[4 * j + c], 0, 0, 0);
                acc[4 * j + c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(t[c], most, acc[4 * j + c], 0, 0, 0);
                acc[4 * j + c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(t[c], most, acc[4 * j + c], 0, 0, 0);
            }
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

// Scores of the lane's row for its 16 keys, sc[ii][i] that of key 16 kb + 4 ii + i; HIDDEN past the row's limit (left: what is left
// of it at the lane's first key; lanes without a row give 16 or more, so that the others need not mask) and where the page is not there.
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
    if (__all(there[0] && there[1] && there[2] && there[3] && left >= 16)) return; // nearly all steps
    uint32_t seen[4]; // bit m: key 4 m + i is there
#pragma unroll
    for (int i = 0; i < 4; ++i) seen[i] = ((uint32_t)__ballot(there[i]) & 0xffffu) >> (4 * kb);
#pragma unroll
    for (int ii = 0; ii < 4; ++ii)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[ii][i] = 4 * ii + i < left && ((seen[i] >> ii) & 1u) ? sc[ii][i] : HIDDEN;
}

// the table index of four distances from the row's maximum (bytes of the result), and the sum of their entries
__device__ __forceinline__ uint32_t four_indices(const uint32_t (&away)[4], int c_int, double factor, const uint8_t *entry, int &sum)
{
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t idx = (uint32_t)(int)__builtin_fma((double)(int)min(away[i], (uint32_t)c_int), factor, 0.5);
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

// Workgroup barrier that orders LDS accesses only: global loads requested before it stay in flight across it (__syncthreads() waits
// for them).
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// What a step's key, one for each lane, has drawn from `rows` rows: idx holds the indices of row n's keys 16 kb .. + 15 at (n, kb),
// 16 bytes each, so that a lane's bytes of all rows lie 64 apart.  The wave wrote them itself.
__device__ __forceinline__ float drawn_by(const uint8_t *idx, const float (*share)[64], int rows, int lane)
{
    __builtin_amdgcn_wave_barrier();
    float sum = 0.0f;
#pragma unroll 4
    for (int r = 0; r < rows; ++r) sum += share[r][idx[64 * r + lane]];
    __builtin_amdgcn_wave_barrier();
    return sum;
}

// A key's weight after a call.  `drawn` is added up in one order whichever kernels a call takes, and so whatever else is in it: over the rows
// of a block of 16, and then over the blocks.
__device__ __forceinline__ float new_weight(const AttendParams &p, float old, float drawn) { return __builtin_fmaf(p.decay, old, drawn); }

// N channels of an output row from ch (a multiple of N) on; mult and shift (INT8) or unit of the row's parameters
template <int N> __device__ __forceinline__ void store_out(const AttendParams &p, float unit, int mult, int shift, uint8_t *at, int ch, const int (&acc)[N])
{
    typedef uint8_t V1 __attribute__((ext_vector_type(N)));
    typedef uint16_t V2 __attribute__((ext_vector_type(N)));
    typedef float V4 __attribute__((ext_vector_type(N)));
    if (p.out_type == 3) {
        V1 x;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (uint8_t)(int8_t)requant_any(acc[i], mult, shift);
        *(V1 *)(at + ch) = x;
        return;
    }
    V4 x;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)acc[i] * unit;
    if (p.out_type == 0) {
        *(V4 *)(at + 4 * ch) = x;
        return;
    }
    V2 y;
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = p.out_type == 1 ? __builtin_bit_cast(uint16_t, (_Float16)x[i]) : __builtin_bit_cast(uint16_t, (__bf16)x[i]);
    *(V2 *)(at + 2 * ch) = y;
}

} // namespace

} // namespace intattn
