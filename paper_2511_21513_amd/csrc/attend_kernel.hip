// Attention of the newest tokens over a paged INT8 cache (the pipeline of include/intattn.h, steps 1 to 8), for gfx950.
//
// IndexSoftmax needs the exact row maximum before any index and the exact row sum before any probability, so a row's keys are met
// three times; each 16 rows read K and V once, because the scores, and then their table indices, stay in LDS.  Steps whose scores do not
// fit have room for their indices there, and K of these is read again for them: with 32 sequences of 4000 to 12400 keys, 8 KV heads of
// four rows and d 128, 137 us, 4.1 TB/s of the bytes that have to move (the three launches of attend_split.hip 144).  A workgroup
// takes all keys of a (sequence, KV head) and up to 16 rows of its query heads and tokens (what several blocks of rows draw from the
// keys is added up by a second launch); its waves take every NW-th step of 64 keys and meet at the maxima and at the sums.
#include "attend_common.h"

#include <algorithm>

namespace intattn {

namespace {

template <int D, int NW, bool WHOLE> __global__ __launch_bounds__(64 * NW) void attend_kernel(const AttendParams p)
{
    using Place = typename Keys<D, WHOLE>::Place;
    using PlaceK = typename Keys<D, WHOLE>::PlaceK;
    constexpr int KB = D / 64, CT = D / 16, ACC_ROW = D + 1; // (rows of accumulators a bank apart)
    __shared__ RowParams rowp[16];
    __shared__ int row_max[16], row_sum[16], acc_sum[16 * ACC_ROW];
    __shared__ uint8_t entry[64], prob[16][PROB]; // LUT_hat, and P_hat of each index in a row
    __shared__ float share[16][64];             // E / S
    // of each lane that has a row, for step after step: sixteen scores, then indices in the place of the first four; from step
    // p.held_steps on, indices alone
    extern __shared__ int4 held[];
    __shared__ int4 widx[NW][64];               // indices of a wave's step

    const int group = p.first + blockIdx.x, b = group / p.c.Hkv, kvh = group % p.c.Hkv, blk = blockIdx.y;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, kb = lane >> 4;
    const Keys<D, WHOLE> keys{p.c, p.c.table + b * p.c.table_stride, kvh * p.c.ks[1], kvh * p.c.vs[1]};
    // (asked for before the length is known, and the scales before keys that a wait for them would have to wait for as well)
    const int row = blk * 16 + n, head = kvh * p.group + row / p.L, t = row % p.L;
    RowScales scales;
    if (threadIdx.x < 16 && row < p.rows) scales = row_scales(p, b, head, t, kvh);
    const PlaceK first_k = keys.find_k(wave, lane);
    const Place first_v = keys.find_v(wave, lane);
    const int len = cache_len(p.c, b), fresh = new_tokens(p.n_new, b, p.L, len), steps = (len + 63) / 64;
    const int held_rows = min(p.rows, 16);
    // weights: the only block of rows writes them, of several each what its rows draw to a plane of its own
    const float *const weight = p.weight && p.blocks == 1 ? p.weight + b * p.wst[0] + kvh * p.wst[1] : nullptr;
    float *const weight_out = !p.weight ? nullptr
                              : p.blocks == 1 ? p.weight_out + b * p.wost[0] + kvh * p.wost[1]
                                              : p.drawn + ((int64_t)blockIdx.x * p.blocks + blk) * p.c.capacity;
    const int held_to = min(steps, p.held_steps);
    auto place = [&](int s) { // the lane's
        const int i = (s * 4 + kb) * held_rows + n;
        return held + (s < held_to ? 4 * i : i + 3 * held_to * 4 * held_rows);
    };
    if (steps == 0) { // no keys: zeros
        const int none[4] = {0, 0, 0, 0};
        const int end = min(blk * 16 + 16, p.rows);
        for (int i = blk * 4 * D + threadIdx.x; i < end * D / 4; i += 64 * NW) store_out<4>(p, 0.0f, 0, 31, out_row(p, b, kvh, 4 * i / D), 4 * i % D, none);
        return;
    }
    if (threadIdx.x < 64) entry[threadIdx.x] = (uint8_t)(p.lut[threadIdx.x >> 2] >> (8 * (threadIdx.x & 3)));

    // K and V of the wave's first step are on their way while the rows' parameters are formed.  (Further steps are asked for one at a time;
    // the number of waves keeps keys on their way.  Places of a step asked for ahead of it: 102 and 100 us for 256 workgroups of 8192 keys,
    // 116 and 117 for 1024 of up to 6000, and registers spilled for pages that are not whole runs.)
    v4i a[4][KB], qf[KB];
    bool there[4];
    uint32_t v[16][KB];
    float old;
    auto ask_v = [&](int s, const Place &from) {
        keys.load_v(from, lane, v);
        old = weight ? weight[min(s * 64 + lane, len - 1)] : 0.0f; // uniform
    };
    keys.load_k(first_k, lane, a, there);
    ask_v(wave, first_v);
    load_q<D>(p, b, kvh, row, kb, qf);
    if (threadIdx.x < 16) {
        RowParams rp = {1.0, 0.0f, 1, 0, 0, 31};
        if (row < p.rows && row_params(p, scales, rp) && t < fresh) rp.limit = len - fresh + t + 1;
        rowp[n] = rp;
        row_max[n] = HIDDEN;
        row_sum[n] = 0;
    }
    for (int i = threadIdx.x; i < 16 * ACC_ROW; i += 64 * NW) acc_sum[i] = 0;
    lds_barrier();
    const bool mine = n < held_rows;
    const int limit = mine ? rowp[n].limit : 0x7fffffff;

    // Q.K^T and row maxima
    int top = HIDDEN;
    for (int s = wave; s < steps;) {
        v4i sc[4];
        step_scores<D>(a, there, qf, limit - (s * 64 + 16 * kb), kb, sc);
#pragma unroll
        for (int ii = 0; ii < 4; ++ii) top = max(top, max(max(sc[ii][0], sc[ii][1]), max(sc[ii][2], sc[ii][3])));
        if (mine && s < held_to) {
            int4 *at = place(s);
#pragma unroll
            for (int ii = 0; ii < 4; ++ii) at[ii] = make_int4(sc[ii][0], sc[ii][1], sc[ii][2], sc[ii][3]);
        }
        s += NW;
        if (s < steps) keys.load_k(keys.find_k(s, lane), lane, a, there);
    }
    top = max(top, __shfl_xor(top, 16));
    top = max(top, __shfl_xor(top, 32));
    if (kb == 0 && mine) atomicMax(&row_max[n], top);
    lds_barrier();

    // indices and row sums: sixteen scores of a row to a thread, whichever wave they came from, so that all lanes have work
    // (by the lanes that hold the rows it took 20 us of 115 at four rows and 8192 keys)
    for (int i = threadIdx.x; i < held_to * 4 * held_rows; i += 64 * NW) {
        const int r = i % held_rows;
        int4 *const at = held + 4 * i;
        const int c_int = rowp[r].c_int;
        const uint32_t row_top = (uint32_t)row_max[r];
        const double factor = rowp[r].factor;
        int sum = 0;
        uint32_t word[4];
#pragma unroll
        for (int ii = 0; ii < 4; ++ii) {
            const int4 x = at[ii];
            const uint32_t away[4] = {row_top - (uint32_t)x.x, row_top - (uint32_t)x.y, row_top - (uint32_t)x.z, row_top - (uint32_t)x.w};
            word[ii] = four_indices(away, c_int, factor, entry, sum);
        }
        at[0] = make_int4((int)word[0], (int)word[1], (int)word[2], (int)word[3]);
        atomicAdd(&row_sum[r], sum);
    }
    if (held_to < steps) {
        const int c_int = rowp[n].c_int;
        const uint32_t row_top = (uint32_t)row_max[n];
        const double factor = rowp[n].factor;
        int sum = 0;
        PlaceK at = keys.find_k(held_to + wave, lane);
        for (int s = held_to + wave; s < steps; s += NW) {
            v4i sc[4];
            keys.load_k(at, lane, a, there);
            at = keys.find_k(s + NW, lane);
            step_scores<D>(a, there, qf, limit - (s * 64 + 16 * kb), kb, sc);
            if (!mine) continue;
            uint32_t word[4];
#pragma unroll
            for (int ii = 0; ii < 4; ++ii) {
                const uint32_t away[4] = {row_top - (uint32_t)sc[ii][0], row_top - (uint32_t)sc[ii][1], row_top - (uint32_t)sc[ii][2], row_top - (uint32_t)sc[ii][3]};
                word[ii] = four_indices(away, c_int, factor, entry, sum);
            }
            *place(s) = make_int4((int)word[0], (int)word[1], (int)word[2], (int)word[3]);
        }
        if (mine) atomicAdd(&row_sum[n], sum);
    }
    lds_barrier();
    // tables of the rows
    for (int i = threadIdx.x; i < held_rows * (p.top + 1); i += 64 * NW) {
        const int r = i / (p.top + 1), idx = i & p.top; // (2^b entries)
        const uint32_t e = row_max[r] != HIDDEN ? entry[idx] : 0u, S = (uint32_t)max(row_sum[r], 1);
        prob[r][idx] = (uint8_t)prob_u8(e, S, __builtin_amdgcn_rcpf((float)(2u * S)));
        if (weight_out) share[r][idx] = (float)e / (float)S;
    }
    lds_barrier();

    // P.V and the keys' weights
    v4i acc[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[c] = v4i{0, 0, 0, 0};
    for (int s = wave; s < steps;) {
        uint32_t word[4] = {0, 0, 0, 0};
        if (mine) {
            const int4 x = *place(s);
            word[0] = (uint32_t)x.x, word[1] = (uint32_t)x.y, word[2] = (uint32_t)x.z, word[3] = (uint32_t)x.w;
        }
        v4i pf = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t pr = prob[n][(word[j / 4] >> (8 * (j & 3))) & 0xffu];
            pf[j / 4] |= (int)(pr << (8 * (j & 3)));
        }
        if (!mine) pf = v4i{0, 0, 0, 0};
        step_pv<D>(v, pf, acc);
        if (weight_out) { // uniform
            if (mine) widx[wave][n * 4 + kb] = make_int4((int)word[0], (int)word[1], (int)word[2], (int)word[3]);
            const float drawn = drawn_by((const uint8_t *)widx[wave], share, held_rows, lane);
            const int slot = s * 64 + lane;
            if (slot < len) weight_out[slot] = new_weight(p, old, drawn);
        }
        s += NW;
        if (s < steps) ask_v(s, keys.find_v(s, lane));
    }
    if (mine && wave < steps) {
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) atomicAdd(&acc_sum[n * ACC_ROW + CT * (4 * kb + i) + c], acc[c][i]);
    }
    lds_barrier();
    for (int i = threadIdx.x; i < held_rows * D / 4; i += 64 * NW) {
        const int r = 4 * i / D, ch = 4 * i % D, g = blk * 16 + r;
        const int *const a = &acc_sum[r * ACC_ROW + ch], four[4] = {a[0], a[1], a[2], a[3]};
        if (g < p.rows) store_out<4>(p, rowp[r].unit, rowp[r].mult, rowp[r].shift, out_row(p, b, kvh, g), ch, four);
    }
}

// Weights where a KV head has several blocks of rows: what they have drawn, block by block.
__global__ __launch_bounds__(256) void attend_weights_kernel(const AttendParams p)
{
    const int group = p.first + blockIdx.y, b = group / p.c.Hkv, kvh = group % p.c.Hkv, slot = blockIdx.x * 256 + threadIdx.x;
    if (slot >= cache_len(p.c, b)) return;
    const float *const of = p.drawn + (int64_t)blockIdx.y * p.blocks * p.c.capacity + slot;
    float drawn = 0.0f;
#pragma unroll 8
    for (int blk = 0; blk < p.blocks; ++blk) drawn += of[(int64_t)blk * p.c.capacity];
    p.weight_out[b * p.wost[0] + kvh * p.wost[1] + slot] = new_weight(p, p.weight[b * p.wst[0] + kvh * p.wst[1] + slot], drawn);
}

} // namespace

// LDS for the scores of a workgroup (beside 30 KB of sixteen waves): all of them, or those of as many steps as leave room for the indices
// of the others
static constexpr int HELD_BYTES = 130 * 1024;

static int most_steps(const AttendParams &p) { return (p.c.capacity + 63) / 64; }
static int step_rows(const AttendParams &p) { return 4 * (p.rows < 16 ? p.rows : 16); }
static int held_steps(const AttendParams &p)
{
    const int more = HELD_BYTES / (16 * step_rows(p)) - most_steps(p); // 48 bytes more for each that is held
    return more < 0 ? -1 : std::min(most_steps(p), more / 3);
}
static int held_bytes(const AttendParams &p) { return 16 * step_rows(p) * (most_steps(p) + 3 * held_steps(p)); }

// Whether the keys are split over workgroups: where not even the indices fit LDS, or where a model of both times, in us, says so.  One
// launch takes 8, a third or half for each step of the longest sequence in its workgroup (more where pages are not whole runs of 16
// keys) and a little for its rows, or what all bytes take through the chip (one price for a step, whether LDS holds its scores or K is
// read again).  Three take 17 and what all bytes need.  Both have further launches for more than one block of rows.  (8 KV heads of
// four rows, d 128, one launch against the sum of three: 1 x 700 keys 10.0 and 15, 1 x 2048 18.0 and 17.3, 8 x 1024 13 and 21, 8 x 4096 35 and 30, 12 x 4096 36 and 35, 16 x 4096 37 and 48, 16 x 8192 75 and 83,
// 32 x 8192 102 and 141;
// one KV head of 32 rows, d 64, 32 x 1 .. 4380 keys 30 and 28.)
static bool split_serves(const AttendParams &p, int d, bool weight)
{
    if (held_steps(p) < 0) return true;
    const double steps = most_steps(p), all = steps * p.c.B * p.c.Hkv * p.blocks, size = d / 128.0;
    const double step = ((steps <= 32 ? 0.35 : 0.48) * size + 0.0065 * std::min(p.rows, 16)) * (whole_pages(p.c, d) ? 1.0 : 1.3);
    const double one = 8.0 + (p.blocks > 1 && weight ? 4.0 : 0.0) + std::max(steps * step, 0.0031 * all * size);
    const double three = 17.0 + (p.blocks > 1 ? weight ? 15.0 : 6.0 : 0.0) + 0.0035 * all * size;
    return three < one;
}

// room: what each block of rows draws, [group][block][capacity]; of a launch that takes `groups` groups
static int64_t drawn_room(const AttendParams &p, int64_t groups, bool weight) { return weight && p.blocks > 1 ? 4 * groups * p.blocks * p.c.capacity : 0; }

// groups from p.first on
template <int D, bool WHOLE> static void launch_waves(const AttendParams &p_, int64_t n, void *stream)
{
    AttendParams p = p_;
    p.held_steps = held_steps(p);
    const int steps = most_steps(p);
    const int64_t groups = n * p.blocks;
    // One wave where there are few steps and the workgroups are many (1856 of 43 keys 29.3 us with four, 13.0 with one, 8 of 30 keys 7.4, 8.0;
    // 2000 of up to 120 20.2, 17.0, of up to 250 24.9, 22.2, 800 of them 15.1, 17.6).  Four for up to four steps (8 of 250 keys 8.0, with
    // eight 8.3; 800 of 100 .. 250 15.1, 19.2; of five steps, 8 of 500 keys, 10.0, 9.2).  Sixteen from sixteen steps on for the only
    // workgroup of a compute unit (eight and sixteen, us: 64 of 1024 keys 14.3, 13.1; 256 of up to 2000 25.1, 23.7; 8 of 700 11.0, 11.8);
    // eight where there are more and LDS holds two of them, so that one has keys on their way while the other looks up indices (512 of up
    // to 3700 keys 66.9, with sixteen 73.6).  Two steps of a wave on their way, for which registers are left with eight waves, took 42.4 us
    // for 128 of 4096 keys, sixteen waves 36.7; 101.7 and 101.4 for 256 of 8192; 89.5 and 80.4 for 280 of 2044 .. 6132.
    const bool two = groups > 256 && 2 * (held_bytes(p) + 22400) <= 160 * 1024;
    const int waves = steps <= (groups >= 1536 ? 4 : groups > 512 ? 1 : 0) ? 1 : steps <= 4 ? 4 : steps >= 16 && !two ? 16 : 8;
    void (*kernel)(const AttendParams) = waves == 1   ? attend_kernel<D, 1, WHOLE>
                                         : waves == 4 ? attend_kernel<D, 4, WHOLE>
                                         : waves == 8 ? attend_kernel<D, 8, WHOLE>
                                                      : attend_kernel<D, 16, WHOLE>;
    hipLaunchKernelGGL(kernel, dim3((uint32_t)n, (uint32_t)p.blocks), dim3((uint32_t)(64 * waves)), (uint32_t)held_bytes(p),
                       (hipStream_t)stream, p);
    if (p.weight && p.blocks > 1)
        hipLaunchKernelGGL(attend_weights_kernel, dim3((uint32_t)((p.c.capacity + 255) / 256), (uint32_t)n), dim3(256), 0, (hipStream_t)stream, p);
}

static int64_t room_of(const AttendParams &p, int d, bool weight)
{
    return split_serves(p, d, weight) ? attend_split_room(p, d) : std::min(drawn_room(p, (int64_t)p.c.B * p.c.Hkv, weight), SCORE_ROOM);
}

int64_t attend_room(const AttendParams &p, int d) { return room_of(p, d, p.weight); }

int64_t attend_room_upto(const AttendParams &p_, int d)
{
    AttendParams p = p_;
    int64_t most = 0;
    for (p.blocks = 1; p.blocks <= p_.blocks; ++p.blocks) { // (the choice differs between numbers of blocks)
        p.rows = std::min(p_.rows, 16 * p.blocks);
        most = std::max(most, std::max(room_of(p, d, false), room_of(p, d, true)));
    }
    return most;
}

int launch_attend(const AttendParams &p_, int d, void *room, void *stream)
{
    if (split_serves(p_, d, p_.weight)) return launch_attend_split(p_, d, room, stream);
    AttendParams p = p_;
    p.drawn = (float *)room;
    const bool whole = whole_pages(p.c, d);
    // the groups whose room that is: one needs less than SCORE_ROOM (256 blocks, and no more keys than LDS has indices for)
    const int64_t all = (int64_t)p.c.B * p.c.Hkv, each = drawn_room(p, 1, p.weight), at_once = each > 0 ? std::min(all, SCORE_ROOM / each) : all;
    for (int64_t first = 0; first < all; first += at_once) {
        const int64_t n = std::min(at_once, all - first);
        p.first = (int32_t)first;
        if (d == 64) whole ? launch_waves<64, true>(p, n, stream) : launch_waves<64, false>(p, n, stream);
        else whole ? launch_waves<128, true>(p, n, stream) : launch_waves<128, false>(p, n, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    return (int)hipSuccess;
}

} // namespace intattn
