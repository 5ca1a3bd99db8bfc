// Attention of the newest tokens over a paged INT8 cache (the pipeline of include/intattn.h, steps 1 to 8), for gfx950.
//
// IndexSoftmax needs the exact row maximum before any index and the exact row sum before any probability, so a row's keys are met
// three times; K and V are read once each, because the scores, and then their table indices, stay in LDS (or, past its size, in
// room of the context).  A workgroup takes all keys of a (sequence, KV head) and up to 16 rows of its query heads and tokens at a
// time; its waves take every NW-th step of 64 keys and meet twice, at the maxima and at the sums.
//
// Layout of a step.  v_mfma_i32_16x16x64_i8 with keys as rows and query rows as columns: lane (n, kb) = (lane % 16, lane / 16)
// gives 16 bytes of a key's row, and the four MFMA tiles take key 4 n + i each, so that lane (n, kb) holds the scores of row n
// for the 16 keys from 16 kb on, in order: exactly the bytes of the P operand of the product with V.  V is turned in registers: a lane
// reads d / 16 channels of its 16 keys, and v_perm makes them rows of keys for each channel.  Neither product passes LDS.
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
    const float so = p.out_type == 3 && p.scale_out ? p.scale_out[p.c.per_head ? head : 0] : sv;
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
    rp.unit = (float)((double)sv / 255.0);
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

template <int D, int NW, bool WHOLE> __global__ __launch_bounds__(64 * NW) void attend_kernel(const AttendParams p)
{
    constexpr int KB = D / 64, CT = D / 16, ACC_ROW = D + 1; // (rows of accumulators a bank apart)
    __shared__ RowParams rowp[16];
    __shared__ int wave_max[NW][16], wave_sum[NW][16], acc_sum[16 * ACC_ROW];
    __shared__ uint8_t entry[64], prob[16][64]; // LUT_hat, and P_hat of each index in a row
    __shared__ float share[16][64];             // E / S
    extern __shared__ int4 held[];              // scores of the first lds_steps steps

    const int b = blockIdx.x / p.c.Hkv, kvh = blockIdx.x % p.c.Hkv;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, kb = lane >> 4;
    const int len = cache_len(p.c, b), fresh = new_tokens(p.n_new, b, p.L, len), steps = (len + 63) / 64;
    const Keys<D, WHOLE> keys{p.c, p.c.table + b * p.c.table_stride, kvh * p.c.ks[1], kvh * p.c.vs[1], len};
    const int held_rows = min(p.rows, 16);
    int4 *const spill = (int4 *)(p.scores + blockIdx.x * p.scores_wg);
    // the lane's sixteen scores, then indices, of a step
    auto place = [&](int s) {
        const int at = (s * 4 + kb) * held_rows + n;
        return s < p.lds_steps ? held + 4 * at : spill + 4 * (at - p.lds_steps * 4 * held_rows);
    };
    if (threadIdx.x < 64) entry[threadIdx.x] = (uint8_t)(p.lut[threadIdx.x >> 2] >> (8 * (threadIdx.x & 3)));

    for (int blk = 0; blk < p.blocks; ++blk) {
        const int row = blk * 16 + n;
        if (threadIdx.x < 16) {
            RowParams rp = {1.0, 0.0f, 1, 0, 0, 31};
            if (row < p.rows) {
                const int t = row % p.L;
                if (row_params(p, b, kvh * p.group + row / p.L, t, kvh, rp) && t < fresh) rp.limit = len - fresh + t + 1;
            }
            rowp[n] = rp;
        }
        for (int i = threadIdx.x; i < 16 * ACC_ROW; i += 64 * NW) acc_sum[i] = 0;
        v4i qf[KB];
#pragma unroll
        for (int j = 0; j < KB; ++j) qf[j] = v4i{0, 0, 0, 0};
        if (row < p.rows) {
            const int8_t *at = p.q + b * p.qs[0] + (int64_t)(kvh * p.group + row / p.L) * p.qs[1] + (row % p.L) * p.qs[2] + 16 * kb;
#pragma unroll
            for (int j = 0; j < KB; ++j) qf[j] = *(const v4i *)(at + 64 * j);
        }
        __syncthreads();
        const RowParams rp = rowp[n];
        const bool mine = n < held_rows;

        // Q.K^T and row maxima
        int top = HIDDEN;
        for (int s = wave; s < steps; s += NW) {
            v4i a[4][KB], sc[4];
            bool there[4];
            keys.load_k(s, lane, a, there);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v4i d = {0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < KB; ++j) d = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i][j], qf[j], d, 0, 0, 0);
#pragma unroll
                for (int ii = 0; ii < 4; ++ii) sc[ii][i] = d[ii]; // key 16 kb + 4 ii + i
            }
            uint32_t seen[4]; // bit m: key 4 m + i is there
#pragma unroll
            for (int i = 0; i < 4; ++i) seen[i] = (uint32_t)__ballot(there[i]) & 0xffffu;
            const int left = rp.limit - (s * 64 + 16 * kb);
#pragma unroll
            for (int ii = 0; ii < 4; ++ii)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool see = 4 * ii + i < left && ((seen[i] >> (4 * kb + ii)) & 1u);
                    sc[ii][i] = see ? sc[ii][i] : HIDDEN;
                    top = max(top, sc[ii][i]);
                }
            if (mine) {
                int4 *at = place(s);
#pragma unroll
                for (int ii = 0; ii < 4; ++ii) at[ii] = make_int4(sc[ii][0], sc[ii][1], sc[ii][2], sc[ii][3]);
            }
        }
        top = max(top, __shfl_xor(top, 16));
        top = max(top, __shfl_xor(top, 32));
        if (kb == 0) wave_max[wave][n] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) top = max(top, wave_max[w][n]);

        // indices and row sums
        int sum = 0;
        if (mine) {
            for (int s = wave; s < steps; s += NW) {
                int4 *at = place(s);
                uint32_t word[4];
#pragma unroll
                for (int ii = 0; ii < 4; ++ii) {
                    const int4 x = at[ii];
                    const int sc[4] = {x.x, x.y, x.z, x.w};
                    word[ii] = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t away = min((uint32_t)top - (uint32_t)sc[i], (uint32_t)rp.c_int);
                        const uint32_t idx = (uint32_t)(int)__builtin_fma((double)(int)away, rp.factor, 0.5);
                        sum += entry[idx];
                        word[ii] |= idx << (8 * i);
                    }
                }
                at[0] = make_int4((int)word[0], (int)word[1], (int)word[2], (int)word[3]);
            }
        }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (kb == 0) wave_sum[wave][n] = sum;
        __syncthreads();
        // tables of the rows: a wave fills row after row
        for (int r = wave; r < 16; r += NW) {
            int total = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w) total += wave_sum[w][r];
            const int row_top = __shfl(top, r);
            const uint32_t e = lane <= p.top && row_top != HIDDEN ? entry[lane] : 0u, S = (uint32_t)max(total, 1);
            prob[r][lane] = (uint8_t)prob_u8(e, S, __builtin_amdgcn_rcpf((float)(2u * S)));
            share[r][lane] = (float)e / (float)S;
        }
        __syncthreads();

        // P.V and the keys' weights
        v4i acc[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[c] = v4i{0, 0, 0, 0};
        for (int s = wave; s < steps; s += NW) {
            uint32_t v[16][KB];
            keys.load_v(s, lane, v);
            uint32_t word[4] = {0, 0, 0, 0};
            if (mine) {
                const int4 x = *place(s);
                word[0] = (uint32_t)x.x, word[1] = (uint32_t)x.y, word[2] = (uint32_t)x.z, word[3] = (uint32_t)x.w;
            }
            v4i pf = {0, 0, 0, 0};
            float w[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const uint32_t idx = (word[j / 4] >> (8 * (j & 3))) & 0xffu;
                const uint32_t pr = mine ? prob[n][idx] : 0u;
                pf[j / 4] |= (int)(pr << (8 * (j & 3)));
                w[j] = 0.0f;
                if (p.weight) w[j] = mine ? share[n][idx] : 0.0f;
            }
            step_pv<D>(v, pf, acc);
            if (p.weight) { // uniform
                const float drawn = scatter_sum16(w, n);
                const int slot = s * 64 + 16 * kb + n;
                if (slot < len) {
                    float *to = p.weight_out + b * p.wost[0] + kvh * p.wost[1] + slot;
                    *to = blk == 0 ? p.decay * p.weight[b * p.wst[0] + kvh * p.wst[1] + slot] + drawn : *to + drawn;
                }
            }
        }
        if (mine) {
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) atomicAdd(&acc_sum[n * ACC_ROW + CT * (4 * kb + i) + c], acc[c][i]);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < held_rows * D; i += 64 * NW) {
            const int r = i / D, ch = i % D, g = blk * 16 + r;
            if (g < p.rows) {
                uint8_t *at = p.out + b * p.os[0] + (int64_t)(kvh * p.group + g / p.L) * p.os[1] + (g % p.L) * p.os[2];
                store_out(p, rowp[r], at, ch, acc_sum[r * ACC_ROW + ch]);
            }
        }
        __syncthreads(); // before the next rows' parameters
    }
}

} // namespace

// LDS for the scores of a workgroup; the rest of its steps go to room of the context
static constexpr int HELD_BYTES = 120 * 1024;

static int step_bytes(const AttendParams &p) { return 4 * 64 * (p.rows < 16 ? p.rows : 16); }
static int most_steps(const AttendParams &p) { return (p.c.capacity + 63) / 64; }
static int held_steps(const AttendParams &p)
{
    const int fit = HELD_BYTES / step_bytes(p);
    return fit < most_steps(p) ? fit : most_steps(p);
}

int64_t attend_room(const AttendParams &p, int)
{
    return (int64_t)(most_steps(p) - held_steps(p)) * step_bytes(p) * p.c.B * p.c.Hkv;
}

int launch_attend(const AttendParams &p_, int d, void *room, void *stream)
{
    AttendParams p = p_;
    p.lds_steps = held_steps(p);
    p.scores = (int32_t *)room;
    p.scores_wg = (int64_t)(most_steps(p) - p.lds_steps) * step_bytes(p) / 4;
    const bool whole = p.c.page_size % 16 == 0;
    const size_t lds = (size_t)p.lds_steps * (size_t)step_bytes(p);
    const bool few = most_steps(p) <= 4;
    void (*kernel)(const AttendParams);
    if (d == 64) kernel = few ? (whole ? attend_kernel<64, 4, true> : attend_kernel<64, 4, false>) : (whole ? attend_kernel<64, 8, true> : attend_kernel<64, 8, false>);
    else kernel = few ? (whole ? attend_kernel<128, 4, true> : attend_kernel<128, 4, false>) : (whole ? attend_kernel<128, 8, true> : attend_kernel<128, 8, false>);
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(p.c.B * p.c.Hkv)), dim3(few ? 256 : 512), lds, (hipStream_t)stream, p);
    return (int)hipGetLastError();
}

} // namespace intattn
