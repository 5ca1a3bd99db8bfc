// Attention of the newest tokens over a paged INT8 cache with the keys of a (sequence, KV head) split over workgroups, for gfx950: for long
// sequences, and for batches of any lengths.  IndexSoftmax is exact in the row maximum and the row sum, and partial results of other
// maxima cannot be joined afterwards, so the work is cut at both, each a launch boundary: no workgroup waits for another.
//   scores   Q.K^T of a chunk of keys: INT32 scores to room of the context, a maximum for each row and chunk
//   lookup   the row's maximum; scores become table indices (a byte each, in place), a sum for each row and chunk
//   values   the row's sum; P.V of a chunk; the last workgroup of a KV head's chunks adds them up and writes the rows.  With more than
//            one block of 16 rows a fourth launch does, and a fifth forms the weights.
// K is read once for each 128 rows of a KV head and V once for each 16, and the scores (4 bytes for each row and key against 2 d for a key)
// mostly stay in the caches between the launches where rows are few.  The chunks of all sequences are one grid of small workgroups, which evens out sequences of different lengths.
//
// Scores of a step of 64 keys: [ii][row][kb] of four keys 16 kb + 4 ii each, so that a wave's stores are contiguous; the sixteen
// indices of (row, kb) take the place of its first four scores.
#include "attend_common.h"

#include <algorithm>

namespace intattn {

namespace {

constexpr int SNT = 256, SWAVES = 4;
constexpr int SBLK = 8, SROWS = 16 * SBLK; // rows of a workgroup in the first two launches

struct Group {
    int b, kvh, len, fresh, steps;
};
// of place g in the room
__device__ __forceinline__ Group group_of(const AttendParams &p, int g)
{
    Group r;
    r.b = (p.first + g) / p.c.Hkv;
    r.kvh = (p.first + g) % p.c.Hkv;
    r.len = cache_len(p.c, r.b);
    r.fresh = new_tokens(p.n_new, r.b, p.L, r.len);
    r.steps = (r.len + 63) / 64;
    return r;
}
// slots that a row sees, whatever its scale
__device__ __forceinline__ int row_limit(const AttendParams &p, const Group &g, int row)
{
    const int t = row % p.L;
    return row < p.rows && t < g.fresh ? g.len - g.fresh + t + 1 : 0;
}
__device__ __forceinline__ int4 *step_of(const AttendParams &p, int g, int s) { return (int4 *)p.scores + ((int64_t)g * p.steps + s) * 16 * p.rows; }

template <int D, bool WHOLE, bool ONE> __global__ __launch_bounds__(SNT) void cache_scores_kernel(const AttendParams p)
{
    constexpr int KB = D / 64;
    __shared__ int limit[SROWS], most[SROWS];
    __shared__ v4i q_lds[ONE ? 1 : SBLK][KB][64];
    const int chunk = blockIdx.x, g = blockIdx.y, blk0 = blockIdx.z * SBLK;
    const Group gr = group_of(p, g);
    const int s0 = chunk * p.score_steps, s1 = min(s0 + p.score_steps, gr.steps);
    if (chunk == 0) {
        for (int i = threadIdx.x; i < SROWS && blk0 * 16 + i < p.rows; i += SNT) { // for the other launches
            const int row = blk0 * 16 + i;
            RowParams rp;
            rp.limit = row_params(p, row_scales(p, gr.b, gr.kvh * p.group + row / p.L, row % p.L, gr.kvh), rp);
            p.row_params[(int64_t)g * p.rows + row] = rp;
        }
    }
    if (s0 >= s1) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, kb = lane >> 4;
    const int blocks = ONE ? 1 : min(SBLK, p.blocks - blk0);
    const Keys<D, WHOLE> keys{p.c, p.c.table + gr.b * p.c.table_stride, gr.kvh * p.c.ks[1], gr.kvh * p.c.vs[1]};
    v4i qf[KB];
    if constexpr (ONE) {
        load_q<D>(p, gr.b, gr.kvh, n, kb, qf);
    } else {
        for (int i = wave; i < blocks; i += SWAVES) {
            load_q<D>(p, gr.b, gr.kvh, (blk0 + i) * 16 + n, kb, qf);
#pragma unroll
            for (int j = 0; j < KB; ++j) q_lds[i][j][lane] = qf[j];
        }
    }
    for (int i = threadIdx.x; i < blocks * 16; i += SNT) {
        limit[i] = row_limit(p, gr, blk0 * 16 + i);
        most[i] = HIDDEN;
    }
    __syncthreads();
    typename Keys<D, WHOLE>::PlaceK at = keys.find_k(s0 + wave, lane);
    for (int s = s0 + wave; s < s1; s += SWAVES) {
        v4i a[4][KB];
        bool there[4];
        keys.load_k(at, lane, a, there);
        at = keys.find_k(s + SWAVES, lane);
        int4 *const to = step_of(p, g, s);
        for (int i = 0; i < blocks; ++i) {
            if constexpr (!ONE) {
#pragma unroll
                for (int j = 0; j < KB; ++j) qf[j] = q_lds[i][j][lane];
            }
            const int row = (blk0 + i) * 16 + n;
            v4i sc[4];
            step_scores<D>(a, there, qf, (row < p.rows ? limit[i * 16 + n] : 0x7fffffff) - (s * 64 + 16 * kb), kb, sc);
            int top = HIDDEN;
#pragma unroll
            for (int ii = 0; ii < 4; ++ii) {
                top = max(top, max(max(sc[ii][0], sc[ii][1]), max(sc[ii][2], sc[ii][3])));
                if (row < p.rows) to[(ii * p.rows + row) * 4 + kb] = make_int4(sc[ii][0], sc[ii][1], sc[ii][2], sc[ii][3]);
            }
            top = max(top, __shfl_xor(top, 16));
            top = max(top, __shfl_xor(top, 32));
            if (kb == 0) atomicMax(&most[i * 16 + n], top);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < blocks * 16; i += SNT) {
        const int row = blk0 * 16 + i;
        if (row < p.rows) p.part_max[((int64_t)g * p.score_chunks + chunk) * p.rows + row] = most[i];
    }
}

__global__ __launch_bounds__(SNT) void cache_lookup_kernel(const AttendParams p)
{
    __shared__ RowParams rowp[SROWS];
    __shared__ int most[SROWS], total[SROWS];
    __shared__ uint8_t entry[64];
    const int chunk = blockIdx.x, g = blockIdx.y, row0 = blockIdx.z * SROWS, rows = min(SROWS, p.rows - row0);
    const Group gr = group_of(p, g);
    const int s0 = chunk * p.lookup_steps, s1 = min(s0 + p.lookup_steps, gr.steps);
    if (chunk == 0) // arrivals of the next launch
        for (int i = threadIdx.x; i < (rows + 15) / 16; i += SNT) p.arrived[g * p.blocks + row0 / 16 + i] = 0;
    if (s0 >= s1) return;
    const int per_step = rows * 4, items = (s1 - s0) * per_step, live = (gr.steps + p.score_steps - 1) / p.score_steps;
    // the first scores are asked for before the row's maximum is known
    auto at = [&](int i) {
        const int s = i / per_step;
        return step_of(p, g, s0 + s) + row0 * 4 + (i - s * per_step);
    };
    int4 x[4];
    if ((int)threadIdx.x < items) {
#pragma unroll
        for (int ii = 0; ii < 4; ++ii) x[ii] = at(threadIdx.x)[ii * p.rows * 4];
    }
    if (threadIdx.x < 64) entry[threadIdx.x] = (uint8_t)(p.lut[threadIdx.x >> 2] >> (8 * (threadIdx.x & 3)));
    for (int i = threadIdx.x; i < rows; i += SNT) {
        most[i] = HIDDEN;
        total[i] = 0;
        rowp[i] = p.row_params[(int64_t)g * p.rows + row0 + i];
    }
    lds_barrier();
    for (int i = threadIdx.x; i < rows * live; i += SNT)
        atomicMax(&most[i % rows], p.part_max[((int64_t)g * p.score_chunks + i / rows) * p.rows + row0 + i % rows]);
    lds_barrier();
    for (int i = threadIdx.x; i < items; i += SNT) {
        int4 *const from = at(i);
        if (i >= SNT) {
#pragma unroll
            for (int ii = 0; ii < 4; ++ii) x[ii] = from[ii * p.rows * 4];
        }
        const int r = i % per_step / 4;
        const int top = most[r], c_int = rowp[r].c_int;
        const double factor = rowp[r].factor;
        int sum = 0;
        uint32_t word[4];
#pragma unroll
        for (int ii = 0; ii < 4; ++ii) {
            const uint32_t t = (uint32_t)top, away[4] = {t - (uint32_t)x[ii].x, t - (uint32_t)x[ii].y, t - (uint32_t)x[ii].z, t - (uint32_t)x[ii].w};
            word[ii] = four_indices(away, c_int, factor, entry, sum);
        }
        from[0] = make_int4((int)word[0], (int)word[1], (int)word[2], (int)word[3]);
        atomicAdd(&total[r], sum);
    }
    lds_barrier();
    for (int i = threadIdx.x; i < rows; i += SNT) // a row that sees nothing, or has no scale: 0
        p.part_sum[((int64_t)g * p.lookup_chunks + chunk) * p.rows + row0 + i] = most[i] == HIDDEN || !rowp[i].limit ? 0 : total[i];
}

// P_hat and E / S of each index for 16 rows from row0 on, by the first 256 threads; S = 0: zeros
__device__ __forceinline__ void row_tables(const AttendParams &p, int g, int steps, int row0, uint8_t (*prob)[PROB], float (*share)[64])
{
    if (threadIdx.x >= 256) return;
    const int live = (steps + p.lookup_steps - 1) / p.lookup_steps;
    const int r = threadIdx.x >> 4, part = threadIdx.x & 15, row = row0 + r;
    int sum = 0;
    if (row < p.rows)
        for (int c = part; c < live; c += 16) sum += p.part_sum[((int64_t)g * p.lookup_chunks + c) * p.rows + row];
#pragma unroll
    for (int o = 1; o < 16; o *= 2) sum += __shfl_xor(sum, o);
    const uint32_t S = (uint32_t)max(sum, 1);
    const float inv = __builtin_amdgcn_rcpf((float)(2u * S));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int idx = 4 * part + i;
        const uint32_t e = sum > 0 ? (p.lut[part] >> (8 * i)) & 0xffu : 0u;
        prob[r][idx] = (uint8_t)prob_u8(e, S, inv);
        if (share) share[r][idx] = (float)e / (float)S;
    }
}

// ONE: one block of rows; the last of a KV head's workgroups to arrive adds their accumulators up.
template <int D, int NW, bool WHOLE, bool ONE, bool WEIGHT> __global__ __launch_bounds__(64 * NW) void cache_values_kernel(const AttendParams p)
{
    constexpr int KB = D / 64, CT = D / 16, ACC_ROW = D + 1;
    __shared__ uint8_t prob[16][PROB];
    __shared__ float share[WEIGHT ? 16 : 1][64];
    __shared__ int4 widx[WEIGHT ? NW : 1][64];
    __shared__ int acc_sum[16 * ACC_ROW];
    __shared__ int last;
    const int chunk = blockIdx.x, g = blockIdx.y, blk = blockIdx.z;
    const Group gr = group_of(p, g);
    const int s0 = chunk * p.chunk_steps, s1 = min(s0 + p.chunk_steps, gr.steps);
    if ((chunk > 0 || !ONE) && s0 >= s1) return;
    const int live = max((gr.steps + p.chunk_steps - 1) / p.chunk_steps, 1);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, kb = lane >> 4, row = blk * 16 + n;
    const int rows = min(16, p.rows - blk * 16);
    const Keys<D, WHOLE> keys{p.c, p.c.table + gr.b * p.c.table_stride, gr.kvh * p.c.ks[1], gr.kvh * p.c.vs[1]};
    const bool mine = n < rows;
    const float *const weight = WEIGHT ? p.weight + gr.b * p.wst[0] + gr.kvh * p.wst[1] : nullptr;
    float *const weight_out = WEIGHT ? p.weight_out + gr.b * p.wost[0] + gr.kvh * p.wost[1] : nullptr;

    // what a step reads, requested for two steps at a time
    struct Step {
        uint32_t v[16][KB];
        int4 x;
        float old;
    } st[2];
    typename Keys<D, WHOLE>::Place at[2];
    auto request = [&](int s, int i) {
        Step &to = st[i];
        keys.template load_v<ONE>(at[i], lane, to.v);
        to.x = step_of(p, g, s)[(mine ? row : blk * 16) * 4 + kb];
        if constexpr (WEIGHT) to.old = weight[min(s * 64 + lane, gr.len - 1)];
    };
    const int first = s0 + wave;
#pragma unroll
    for (int i = 0; i < 2; ++i) at[i] = keys.find_v(first + i * NW, lane);
    if (first < s1) {
        request(first, 0);
        if (first + NW < s1) request(first + NW, 1);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) at[i] = keys.find_v(first + (2 + i) * NW, lane);
    row_tables(p, g, gr.steps, blk * 16, prob, WEIGHT ? share : nullptr);
    for (int i = threadIdx.x; i < 16 * ACC_ROW; i += 64 * NW) acc_sum[i] = 0;
    lds_barrier();
    v4i acc[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[c] = v4i{0, 0, 0, 0};
    auto take = [&](int s, const Step &of) {
        const uint32_t word[4] = {(uint32_t)of.x.x, (uint32_t)of.x.y, (uint32_t)of.x.z, (uint32_t)of.x.w};
        v4i pf = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t pr = prob[n][(word[j / 4] >> (8 * (j & 3))) & 0xffu];
            pf[j / 4] |= (int)(pr << (8 * (j & 3)));
        }
        if (!mine) pf = v4i{0, 0, 0, 0};
        step_pv<D>(of.v, pf, acc);
        if constexpr (WEIGHT) {
            if (mine) widx[wave][n * 4 + kb] = of.x;
            const float drawn = drawn_by((const uint8_t *)widx[wave], share, rows, lane);
            if (s * 64 + lane < gr.len) weight_out[s * 64 + lane] = new_weight(p, of.old, drawn);
        }
    };
    for (int s = first; s < s1; s += 2 * NW) {
        if (s != first) {
            request(s, 0);
            if (s + NW < s1) request(s + NW, 1);
#pragma unroll
            for (int i = 0; i < 2; ++i) at[i] = keys.find_v(s + (2 + i) * NW, lane);
        }
        take(s, st[0]);
        if (s + NW < s1) take(s + NW, st[1]);
    }
    if (mine) {
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) atomicAdd(&acc_sum[n * ACC_ROW + CT * (4 * kb + i) + c], acc[c][i]);
    }
    __syncthreads();
    int *const parts = p.part_acc + ((int64_t)g * p.blocks + blk) * p.chunks * 16 * D;
    if constexpr (!ONE) { // for cache_join_kernel
        for (int i = threadIdx.x; i < rows * D / 4; i += 64 * NW) {
            const int *const a = &acc_sum[4 * i / D * ACC_ROW + 4 * i % D];
            *(int4 *)(parts + (int64_t)chunk * 16 * D + 4 * i) = make_int4(a[0], a[1], a[2], a[3]);
        }
        return;
    }
    uint64_t *const part = (uint64_t *)parts;
    constexpr int PART = 16 * D / 2; // pairs of accumulators of a chunk
    if (live > 1) {
        // device-scope stores and loads for what another workgroup reads: they pass the L2 of the XCD
        for (int i = threadIdx.x; i < rows * D / 2; i += 64 * NW) {
            const int *a = &acc_sum[2 * i / D * ACC_ROW + 2 * i % D];
            __hip_atomic_store(part + (int64_t)chunk * PART + i, (uint64_t)(uint32_t)a[0] | ((uint64_t)(uint32_t)a[1] << 32), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) last = (int)atomicAdd((unsigned *)&p.arrived[g * p.blocks + blk], 1u);
        __syncthreads();
        if (last != live - 1) return;
    }
    for (int i = threadIdx.x; i < rows * D / 2; i += 64 * NW) {
        const int r = 2 * i / D, ch = 2 * i % D, out = blk * 16 + r;
        int sum[2] = {acc_sum[r * ACC_ROW + ch], acc_sum[r * ACC_ROW + ch + 1]};
        if (live > 1) {
            sum[0] = sum[1] = 0;
            constexpr int BATCH = 32; // loads in flight
            for (int c = 0; c < live; c += BATCH) {
                uint64_t x[BATCH];
#pragma unroll
                for (int u = 0; u < BATCH; ++u) x[u] = __hip_atomic_load(part + (int64_t)min(c + u, live - 1) * PART + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                for (int u = 0; u < BATCH; ++u) {
                    sum[0] += c + u < live ? (int)(uint32_t)x[u] : 0;
                    sum[1] += c + u < live ? (int)(uint32_t)(x[u] >> 32) : 0;
                }
            }
        }
        const RowParams ro = p.row_params[(int64_t)g * p.rows + out];
        uint8_t *const at = out_row(p, gr.b, gr.kvh, out);
        store_out<2>(p, ro.unit, ro.mult, ro.shift, at, ch, sum);
    }
}

// The rows where a KV head has more than one block of them: the accumulators of all chunks added up, four channels to a thread (the
// last workgroup, on its own, took 41 us for 32 rows of 20006 keys, 8 sequences, 2 KV heads, d 128, apart both take 34 and with V
// through the caches 30.  For one block of four rows of 30011 keys 18.4 apart, 16.7 so).
constexpr int JNT = 64;
template <int D> __global__ __launch_bounds__(JNT) void cache_join_kernel(const AttendParams p)
{
    const int g = blockIdx.y, i = blockIdx.x * JNT + threadIdx.x, row = 4 * i / D, ch = 4 * i % D;
    if (row >= p.rows) return;
    const Group gr = group_of(p, g);
    const int live = (gr.steps + p.chunk_steps - 1) / p.chunk_steps;
    const int *const part = p.part_acc + ((int64_t)g * p.blocks + row / 16) * p.chunks * 16 * D + row % 16 * D + ch;
    const RowParams ro = p.row_params[(int64_t)g * p.rows + row];
    if (p.weight) { // the row's sum for the next launch, by the lanes that have the row
        int total = 0;
        for (int c = ch / 4; c < (gr.steps + p.lookup_steps - 1) / p.lookup_steps; c += D / 4) total += p.part_sum[((int64_t)g * p.lookup_chunks + c) * p.rows + row];
#pragma unroll
        for (int o = 1; o < D / 4; o *= 2) total += __shfl_xor(total, o);
        if (ch == 0) p.row_sum[(int64_t)g * p.rows + row] = total;
    }
    int sum[4] = {0, 0, 0, 0};
    constexpr int BATCH = 16; // loads in flight
    for (int c = 0; c < live; c += BATCH) {
        int4 x[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) x[u] = *(const int4 *)(part + (int64_t)min(c + u, live - 1) * 16 * D);
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            if (c + u >= live) break;
            sum[0] += x[u].x, sum[1] += x[u].y, sum[2] += x[u].z, sum[3] += x[u].w;
        }
    }
    store_out<4>(p, ro.unit, ro.mult, ro.shift, out_row(p, gr.b, gr.kvh, row), ch, sum);
}

// Weights where a KV head has more than 16 rows: a thread for each key, over all rows, E / S of 64 rows at a time in LDS (64
// keys and a quarter of the rows to each wave: 7.0 -> 14.1 us for 32 rows of 20006 keys, 8 sequences, 2 KV heads, and 17.1 -> 12.9 for 224 rows).
__global__ __launch_bounds__(SNT) void cache_weights_kernel(const AttendParams p)
{
    constexpr int AT_ONCE = 64;
    __shared__ float share[AT_ONCE][64];
    const int g = blockIdx.y, slot = blockIdx.x * SNT + threadIdx.x;
    const Group gr = group_of(p, g);
    if ((int)blockIdx.x * SNT >= gr.len) return;
    const bool mine = slot < gr.len;
    float drawn = 0.0f;
    for (int row0 = 0; row0 < p.rows; row0 += AT_ONCE) {
        const int rows = min(AT_ONCE, p.rows - row0);
        __syncthreads();
        for (int i = threadIdx.x; i < rows * (p.top + 1); i += SNT) {
            const int r = i / (p.top + 1), idx = i & p.top, sum = p.row_sum[(int64_t)g * p.rows + row0 + r]; // (2^b entries)
            share[r][idx] = sum > 0 ? (float)((p.lut[idx >> 2] >> (8 * (idx & 3))) & 0xffu) / (float)sum : 0.0f;
        }
        __syncthreads();
        if (mine) {
            const uint8_t *at = (const uint8_t *)(step_of(p, g, slot >> 6) + row0 * 4) + (slot & 63);
            for (int r0 = 0; r0 < rows; r0 += 16) { // a block of rows
                float of_block = 0.0f;
                if (rows - r0 >= 16) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) of_block += share[r0 + r][at[64 * (r0 + r)]];
                } else {
                    for (int r = r0; r < rows; ++r) of_block += share[r][at[64 * r]];
                }
                drawn += of_block;
            }
        }
    }
    if (mine) p.weight_out[gr.b * p.wost[0] + gr.kvh * p.wost[1] + slot] = new_weight(p, p.weight[gr.b * p.wst[0] + gr.kvh * p.wst[1] + slot], drawn);
}

} // namespace

// Steps of a workgroup in each launch, by the number of steps there can be (one row, 32 sequences of 4000 to 12400 keys, and one of
// 30011, d 128, us): scores, short workgroups, 4: 59.0, 9.1; 16: 69.5, 11.0.  Lookup, 8: 12.9, 4.6; 32: 10.2, 5.3.  Values, where
// each workgroup leaves accumulators to be joined, 4: 128, 31.8; 8: 87, 21.2; 16: 73.3, 17.6; 32: 74.4, 22.1.  Lookup of 224 rows of
// 5809 keys, two sequences, 8: 18.5; 1: 8.3.
static void plan(AttendParams &p, int64_t groups)
{
    p.steps = (p.c.capacity + 63) / 64;
    const int64_t all = p.steps * groups;
    // as many steps as leave `workgroups` workgroups, between `least` and what makes `most` chunks of a sequence
    auto steps_of = [&](int64_t workgroups, int64_t least, int64_t most) {
        const int64_t c = std::max(std::max((all + workgroups - 1) / workgroups, least), (p.steps + most - 1) / most);
        return (int32_t)c;
    };
    auto whole = [](int32_t steps) { return (steps + SWAVES - 1) / SWAVES * SWAVES; };
    p.score_steps = whole(steps_of(16384, 4, 256));
    p.lookup_steps = steps_of(1536, p.rows <= 16 ? 8 : std::max(1, 128 / p.rows), 256);
    p.chunk_steps = whole(steps_of(3000, 8, 32));
    p.score_chunks = (p.steps + p.score_steps - 1) / p.score_steps;
    p.lookup_chunks = (p.steps + p.lookup_steps - 1) / p.lookup_steps;
    p.chunks = (p.steps + p.chunk_steps - 1) / p.chunk_steps;
}

// bytes of room for `groups` groups, laid out from `room` on
static int64_t lay_out(AttendParams &p, int d, int64_t groups, void *room)
{
    plan(p, groups);
    int64_t at = 0;
    auto take = [&](int64_t words) {
        int32_t *const m = room ? (int32_t *)room + at : nullptr;
        at += (words + 63) / 64 * 64;
        return m;
    };
    p.scores = take(groups * p.steps * 64 * p.rows);
    p.part_max = take(groups * p.score_chunks * p.rows);
    p.part_sum = take(groups * p.lookup_chunks * p.rows);
    p.part_acc = take(groups * p.blocks * p.chunks * 16 * d);
    p.arrived = take(groups * p.blocks);
    p.row_sum = take(groups * p.rows);
    p.row_params = (RowParams *)take(groups * p.rows * (int64_t)(sizeof(RowParams) / 4));
    return 4 * at;
}

// what all groups need; where that is more than SCORE_ROOM, that much, or what one group needs.  (No less for more rows: reservations.)
int64_t attend_split_room(const AttendParams &p_, int d)
{
    AttendParams p = p_;
    const int64_t all = lay_out(p, d, (int64_t)p.c.B * p.c.Hkv, nullptr);
    return all <= SCORE_ROOM ? all : std::max(SCORE_ROOM, lay_out(p, d, 1, nullptr));
}

// Waves of a workgroup of the third launch: eight where they are no more than CUs, so that each has its keys on their way at once (four
// rows, d 128, 8 KV heads, us with four waves and with eight: 1 x 30011 keys 18.3, 16.4; 1 x 100000 36.5, 31.5; 2 x 8000 13.8, 13.0; in
// more workgroups, 4 x 4000 .. 12400, 19.0, 25.9).
template <int D, bool WHOLE> static void launch_values(const AttendParams &p, uint32_t groups, hipStream_t st)
{
    const dim3 grid((uint32_t)p.chunks, groups, (uint32_t)p.blocks);
    const bool eight = (int64_t)p.chunks * groups * p.blocks <= 256;
    void (*kernel)(const AttendParams);
    if (p.blocks > 1) kernel = eight ? cache_values_kernel<D, 8, WHOLE, false, false> : cache_values_kernel<D, 4, WHOLE, false, false>;
    else if (p.weight) kernel = eight ? cache_values_kernel<D, 8, WHOLE, true, true> : cache_values_kernel<D, 4, WHOLE, true, true>;
    else kernel = eight ? cache_values_kernel<D, 8, WHOLE, true, false> : cache_values_kernel<D, 4, WHOLE, true, false>;
    hipLaunchKernelGGL(kernel, grid, dim3(eight ? 512 : 256), 0, st, p);
}

template <int D, bool WHOLE> static void launch_split_d(const AttendParams &p, uint32_t groups, hipStream_t st)
{
    const uint32_t supers = (uint32_t)((p.rows + SROWS - 1) / SROWS);
    if (p.blocks == 1) hipLaunchKernelGGL((cache_scores_kernel<D, WHOLE, true>), dim3((uint32_t)p.score_chunks, groups, 1), dim3(SNT), 0, st, p);
    else hipLaunchKernelGGL((cache_scores_kernel<D, WHOLE, false>), dim3((uint32_t)p.score_chunks, groups, supers), dim3(SNT), 0, st, p);
    hipLaunchKernelGGL(cache_lookup_kernel, dim3((uint32_t)p.lookup_chunks, groups, supers), dim3(SNT), 0, st, p);
    launch_values<D, WHOLE>(p, groups, st);
    if (p.blocks == 1) return;
    hipLaunchKernelGGL(cache_join_kernel<D>, dim3((uint32_t)((p.rows * D / 4 + JNT - 1) / JNT), groups), dim3(JNT), 0, st, p);
    if (p.weight) hipLaunchKernelGGL(cache_weights_kernel, dim3((uint32_t)((p.c.capacity + SNT - 1) / SNT), groups), dim3(SNT), 0, st, p);
}

int launch_attend_split(const AttendParams &p_, int d, void *room, void *stream)
{
    AttendParams p = p_;
    const bool whole = whole_pages(p.c, d);
    hipStream_t st = (hipStream_t)stream;
    const int64_t all = (int64_t)p.c.B * p.c.Hkv, bytes = attend_split_room(p, d);
    int64_t at_once = all; // groups whose room that is
    for (int64_t need; at_once > 1 && (need = lay_out(p, d, at_once, nullptr)) > bytes;) at_once = std::max<int64_t>(1, std::min(at_once - 1, at_once * bytes / need));
    lay_out(p, d, at_once, room); // (one layout for all parts: fewer groups may be cut into more chunks, and need more)
    for (int64_t first = 0; first < all; first += at_once) {
        const int64_t n = std::min(at_once, all - first);
        p.first = (int32_t)first;
        if (d == 64) whole ? launch_split_d<64, true>(p, (uint32_t)n, st) : launch_split_d<64, false>(p, (uint32_t)n, st);
        else whole ? launch_split_d<128, true>(p, (uint32_t)n, st) : launch_split_d<128, false>(p, (uint32_t)n, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    return (int)hipSuccess;
}

} // namespace intattn
