// Attention of the newest tokens over a paged INT8 cache (the pipeline of include/intattn.h, steps 1 to 8), for gfx950.
//
// IndexSoftmax needs the exact row maximum before any index and the exact row sum before any probability, so a row's keys are met
// three times; K and V are read once each, because the scores, and then their table indices, stay in LDS (or, past its size, in
// room of the context).  A workgroup takes all keys of a (sequence, KV head) and up to 16 rows of its query heads and tokens at a
// time; its waves take every NW-th step of 64 keys and meet twice, at the maxima and at the sums.
#include "attend_common.h"

namespace intattn {

namespace {

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
        load_q<D>(p, b, kvh, row, kb, qf);
        __syncthreads();
        const RowParams rp = rowp[n];
        const bool mine = n < held_rows;

        // Q.K^T and row maxima
        int top = HIDDEN;
        for (int s = wave; s < steps; s += NW) {
            v4i a[4][KB], sc[4];
            bool there[4];
            keys.load_k(s, lane, a, there);
            step_scores<D>(a, there, qf, rp.limit - (s * 64 + 16 * kb), kb, sc);
#pragma unroll
            for (int ii = 0; ii < 4; ++ii) top = max(top, max(max(sc[ii][0], sc[ii][1]), max(sc[ii][2], sc[ii][3])));
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
                for (int ii = 0; ii < 4; ++ii) word[ii] = four_indices(at[ii], top, rp, entry, sum);
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
            if (g < p.rows) store_out(p, rowp[r], out_row(p, b, kvh, g), ch, acc_sum[r * ACC_ROW + ch]);
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

static bool split_serves(const AttendParams &p) { return p.c.capacity > 1024; }

int64_t attend_room(const AttendParams &p, int d)
{
    if (split_serves(p)) return attend_split_room(p, d, nullptr, nullptr);
    return (int64_t)(most_steps(p) - held_steps(p)) * step_bytes(p) * p.c.B * p.c.Hkv;
}

int launch_attend(const AttendParams &p_, int d, void *room, void *stream)
{
    if (split_serves(p_)) return launch_attend_split(p_, d, room, stream);
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
