// Eviction from a paged cache by accumulated attention weight, for gfx950.  Two launches: a workgroup for each (sequence, KV head)
// finds the keys that leave and pairs the gaps among the first `keep` slots with the keys that stay behind them; then rows are
// moved, by as many workgroups as there are rows.  Filling gaps moves at most as many rows as leave (keeping the order would move
// nearly all of them), and no slot is both read and written: gaps lie below keep, the keys that fill them at or above it.
//
// The choice is a radix selection over keys of 64 bits: whether the key is held, its weight as an ordered integer, its order.  A pass
// counts a digit of 11 bits (the first takes the weight's exponent and a bit of the fraction, so that weights of all sizes spread over the
// bins) and narrows down the (len - keep)-th smallest; once 256 keys are left, mostly after one pass, they are compared with each other.
// Of equal keys the lowest slots leave.  No sort, and nothing depends on the order in which atomics arrive, because they count.  Each
// wave owns a run of slots; up to 16384 keys wait in LDS between the passes, more are formed again.  Bound by the instructions and waits
// of one workgroup's passes over its keys.
#include "cache_common.h"

namespace intattn {

namespace {

constexpr int EHOLD = 16384; // slots whose keys LDS holds
constexpr int BINS = 2048, FEW = 256;

// NaN above every weight, -0 as 0; orders are at least 0
__device__ __forceinline__ uint64_t sort_key(float w, int order, int sink, int newest)
{
    uint32_t u = __float_as_uint(w + 0.0f);
    u = w != w ? 0xffffffffu : (u >> 31) ? ~u : u | 0x80000000u;
    const uint64_t held = order < sink || order >= newest;
    return (held << 63) | ((uint64_t)u << 31) | (uint32_t)max(order, 0);
}

// sum over the workgroup of what its waves give (the same for all lanes of a wave), and of the waves before; `slots` is free
// after the next barrier
template <int EWAVES> __device__ __forceinline__ int sum_of_waves(int mine, int *slots, int &before)
{
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) slots[wave] = mine;
    __syncthreads();
    int all = 0;
    before = 0;
#pragma unroll
    for (int w = 0; w < EWAVES; ++w) {
        before += w < wave ? slots[w] : 0;
        all += slots[w];
    }
    return all;
}

// ENT threads; HOLD: keys in LDS
template <int ENT, bool HOLD> __global__ __launch_bounds__(ENT) void evict_select_kernel(const EvictParams p)
{
    constexpr int EWAVES = ENT / 64, PER = BINS / ENT;
    __shared__ int bins[BINS], sums[3][EWAVES], chosen[3], n_few;
    __shared__ uint64_t few[FEW], chosen_key;
    extern __shared__ uint64_t key_of[]; // HOLD: of slot s0 + 64 i at i ENT + thread
    const int b = blockIdx.x / p.c.Hkv, kvh = blockIdx.x % p.c.Hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int len = cache_len(p.c, b);
    const int rounds = (len + ENT - 1) / ENT, s0 = wave * rounds * 64 + lane; // slots s0 + 64 i of this thread
    const float *const weight = p.weight + b * p.wst[0] + kvh * p.wst[1];
    const int32_t *const order = p.order ? p.order + b * p.ost[0] + kvh * p.ost[1] : nullptr; // null: the slot
    float *const weight_out = p.weight_out + b * p.wost[0] + kvh * p.wost[1];
    int32_t *const order_out = p.order_out ? p.order_out + b * p.oost[0] + kvh * p.oost[1] : nullptr;
    const int newest = (int)max((int64_t)(p.total ? p.total[b] : len) - p.recent, (int64_t)-0x7fffffff - 1);
    const bool copy_w = weight_out != weight, copy_o = order_out && order_out != order;

    for (int i = tid; i < BINS; i += ENT) bins[i] = 0;
    // Keys to LDS (behind the last: above any), and planes of their own take what lies below keep as it is; gaps are filled by the
    // next launch.
    if (HOLD || copy_w || copy_o) {
        constexpr int AT_ONCE = 8; // loads of a thread in flight
        const int under = min(len, p.keep);
        for (int i0 = 0; i0 < rounds; i0 += AT_ONCE) {
            float w[AT_ONCE];
            int o[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int from = min(s0 + 64 * (i0 + u), len - 1);
                w[u] = weight[from];
                o[u] = order ? order[from] : from;
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int s = s0 + 64 * (i0 + u);
                if (i0 + u >= rounds) break;
                if constexpr (HOLD) key_of[(i0 + u) * ENT + tid] = s < len ? sort_key(w[u], o[u], p.sink, newest) : ~0ull;
                if (copy_w && s < under) weight_out[s] = w[u];
                if (copy_o && s < under) order_out[s] = o[u];
            }
        }
    }
    bool lost = false;
    const int32_t *row = p.c.table + b * p.c.table_stride;
    if (len > p.keep)
        for (int i = tid; i <= quotient(len - 1, p.c.by_page); i += ENT) lost |= (uint32_t)row[i] >= (uint32_t)p.c.n_pages;
    const bool stays = len <= p.keep || __syncthreads_or(lost);
    if (kvh == 0 && tid == 0) p.count[p.c.B * p.c.Hkv + b] = stays ? len : p.keep;
    if (stays) {
        for (int s = p.keep + tid; s < len; s += ENT) {
            if (copy_w) weight_out[s] = weight[s];
            if (copy_o) order_out[s] = order[s];
        }
        if (tid == 0) p.count[blockIdx.x] = 0;
        return;
    }

    // f(slot, key) for each slot of the thread
    auto each = [&](auto f) {
        constexpr int AT_ONCE = 4; // keys on their way
        for (int i0 = 0; i0 < rounds; i0 += AT_ONCE) {
            uint64_t k[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int i = min(i0 + u, rounds - 1), s = s0 + 64 * i, from = min(s, len - 1);
                if constexpr (HOLD) k[u] = key_of[i * ENT + tid];
                else k[u] = s < len ? sort_key(weight[from], order ? order[from] : from, p.sink, newest) : ~0ull;
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (i0 + u < rounds) f(s0 + 64 * (i0 + u), k[u]);
        }
    };

    // prefix: the first digits of the leave-th smallest key; leave: how many keys with that prefix leave
    uint64_t prefix = 0;
    int leave = len - p.keep, shift = 64, before = 0;
    bool whole = false; // every key with the prefix leaves
    while (shift > 0 && !whole) {
        const int digit = min(shift, 11), above = shift;
        shift -= digit;
        if (above < 64) {
            for (int i = tid; i < BINS; i += ENT) bins[i] = 0;
            __syncthreads();
            each([&](int, uint64_t k) {
                if ((k >> above) == prefix) atomicAdd(&bins[(uint32_t)(k >> shift) & ((1u << digit) - 1u)], 1);
            });
        } else {
            each([&](int, uint64_t k) { atomicAdd(&bins[(uint32_t)(k >> 53)], 1); });
        }
        __syncthreads();
        int some[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) sum += some[i] = bins[PER * tid + i];
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int up = __shfl_up(upto, o);
            if (lane >= o) upto += up;
        }
        sum_of_waves<EWAVES>(__shfl(upto, 63), sums[0], before);
        int count = before + upto - sum;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (count < leave && leave <= count + some[i]) {
                chosen[0] = PER * tid + i;
                chosen[1] = leave - count;
                chosen[2] = some[i];
            }
            count += some[i];
        }
        if (tid == 0) n_few = 0;
        __syncthreads();
        prefix = (prefix << digit) | (uint64_t)chosen[0];
        leave = chosen[1];
        whole = chosen[2] == leave;
        if (whole || shift == 0 || chosen[2] > FEW) continue;
        // few enough to compare each with all
        each([&](int, uint64_t k) {
            if ((k >> shift) == prefix) few[atomicAdd(&n_few, 1)] = k;
        });
        __syncthreads();
        constexpr int TEAM = ENT / FEW; // lanes to a key
        if (tid / TEAM < n_few) {
            const uint64_t mine = few[tid / TEAM];
            int less = 0, same = 0;
#pragma unroll 4
            for (int i = tid % TEAM; i < n_few; i += TEAM) {
                const uint64_t k = few[i];
                less += k < mine;
                same += k == mine;
            }
#pragma unroll
            for (int o = 1; o < TEAM; o *= 2) {
                less += __shfl_xor(less, o);
                same += __shfl_xor(same, o);
            }
            if (less < leave && leave <= less + same) {
                chosen_key = mine;
                chosen[1] = leave - less;
                chosen[2] = same;
            }
        }
        __syncthreads();
        shift = 0;
        prefix = chosen_key;
        leave = chosen[1];
        whole = chosen[2] == leave;
    }

    // Who leaves: keys below `least`, and of those on it (only where not all of them do) the first `leave` in the order of slots.
    // Gaps below keep and keys from keep on that stay are counted by the waves, then numbered and listed.
    const uint64_t least = whole ? ((prefix << shift) | ((1ull << shift) - 1ull)) + 1ull : prefix; // (whole: 0 if that was the greatest key)
    const bool all = whole && least == 0;
    int equals = 0;
    if (!whole) {
        each([&](int, uint64_t k) { equals += __popcll(__ballot(k == least)); });
        sum_of_waves<EWAVES>(equals, sums[0], equals);
    }
    const uint64_t below = (1ull << lane) - 1ull;
    auto leaves = [&](uint64_t k, int &seen) { // seen: equal keys before this round
        bool gone = all || k < least;
        if (!whole) {
            const uint64_t m = __ballot(k == least);
            gone |= k == least && seen + __popcll(m & below) < leave;
            seen += __popcll(m);
        }
        return gone;
    };
    int gaps = 0, movers = 0, seen = equals;
    each([&](int s, uint64_t k) {
        const bool gone = leaves(k, seen);
        gaps += __popcll(__ballot(gone && s < p.keep));
        movers += __popcll(__ballot(!gone && s < len && s >= p.keep));
    });
    const int all_gaps = sum_of_waves<EWAVES>(gaps, sums[1], gaps);
    sum_of_waves<EWAVES>(movers, sums[2], movers);
    int32_t *const to = p.moves + (int64_t)blockIdx.x * 2 * p.max_moves, *const from = to + p.max_moves;
    seen = equals;
    each([&](int s, uint64_t k) {
        const bool gone = leaves(k, seen), gap = gone && s < p.keep, mover = !gone && s < len && s >= p.keep;
        const uint64_t mg = __ballot(gap), mm = __ballot(mover);
        if (gap) to[gaps + __popcll(mg & below)] = s;
        if (mover) from[movers + __popcll(mm & below)] = s;
        gaps += __popcll(mg);
        movers += __popcll(mm);
    });
    if (tid == 0) p.count[blockIdx.x] = all_gaps;
}

// Rows to their gaps: 2 d / 16 lanes a key, K then V.  Bound by reads and writes of single rows in no order: 218 000 of them, 128 bytes of
// K and of V each, in 34 us, 3.3 TB/s (through the caches 37; four moves of a thread in flight 39).
template <int D> __global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams p)
{
    constexpr int LANES = D / 8; // of 16 bytes
    const int bh = blockIdx.y, b = bh / p.c.Hkv, kvh = bh % p.c.Hkv, n = p.count[bh];
    if (blockIdx.x == 0 && kvh == 0 && threadIdx.x == 0) p.lens_out[b] = p.count[p.c.B * p.c.Hkv + b];
    const int32_t *to = p.moves + (int64_t)bh * 2 * p.max_moves, *from = to + p.max_moves, *row = p.c.table + b * p.c.table_stride;
    const int part = threadIdx.x % LANES;
    const bool value = part >= LANES / 2;
    const int64_t *st = value ? p.c.vs : p.c.ks;
    int8_t *base = (value ? p.c.v : p.c.k) + kvh * st[1] + 16 * (part % (LANES / 2));
    for (int i = blockIdx.x * (256 / LANES) + threadIdx.x / LANES; i < n; i += gridDim.x * (256 / LANES)) {
        const int dst = to[i], src = from[i];
        const Slot a = find_slot(p.c, row, src), z = find_slot(p.c, row, dst);
        const v4i x = __builtin_nontemporal_load((const v4i *)(base + a.page * st[0] + a.at * st[2]));
        if (part == 0) {
            const float w = p.weight[b * p.wst[0] + kvh * p.wst[1] + src];
            p.weight_out[b * p.wost[0] + kvh * p.wost[1] + dst] = w;
            if (p.order_out) p.order_out[b * p.oost[0] + kvh * p.oost[1] + dst] = p.order[b * p.ost[0] + kvh * p.ost[1] + src];
        }
        __builtin_nontemporal_store(x, (v4i *)(base + z.page * st[0] + z.at * st[2]));
    }
}

} // namespace

static int32_t most_moves(const EvictParams &p)
{
    const int64_t leave = (int64_t)p.c.capacity - p.keep;
    return (int32_t)(leave < 0 ? 0 : leave < p.keep ? leave : p.keep);
}

int64_t evict_room(const EvictParams &p)
{
    return 4 * ((int64_t)p.c.B * p.c.Hkv * (1 + 2 * (int64_t)most_moves(p)) + p.c.B);
}

int launch_evict(const EvictParams &p_, void *room, void *stream)
{
    EvictParams p = p_;
    p.max_moves = most_moves(p);
    p.count = (int32_t *)room;
    p.moves = p.count + (int64_t)p.c.B * p.c.Hkv + p.c.B;
    const int groups = p.c.B * p.c.Hkv;
    // a workgroup of 512 threads up to 4096 slots: its barriers are cheaper
    const bool few = p.c.capacity <= 4096, hold = p.c.capacity <= EHOLD;
    const int threads = few ? 512 : 1024;
    const size_t lds = hold ? (size_t)(p.c.capacity + threads - 1) / threads * threads * 8 : 0;
    void (*select)(const EvictParams) = few ? evict_select_kernel<512, true> : hold ? evict_select_kernel<1024, true> : evict_select_kernel<1024, false>;
    hipLaunchKernelGGL(select, dim3((uint32_t)groups), dim3((uint32_t)threads), (uint32_t)lds, (hipStream_t)stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (int)e;
    const int rows = 2048 / p.d, fit = (p.max_moves + rows - 1) / rows; // moves of a workgroup at a time, and workgroups for all
    hipLaunchKernelGGL(p.d == 64 ? evict_move_kernel<64> : evict_move_kernel<128>, dim3((uint32_t)(fit < 1 ? 1 : fit < 64 ? fit : 64), (uint32_t)groups),
                       dim3(256), 0, (hipStream_t)stream, p);
    return (int)hipGetLastError();
}

} // namespace intattn
