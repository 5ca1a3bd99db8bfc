// Eviction from a paged cache by accumulated attention weight, for gfx950.  Two launches: a workgroup for each (sequence, KV head)
// finds the keys that leave and pairs the gaps among the first `keep` slots with the keys that stay behind them; then rows are
// moved, by as many workgroups as there are rows.  Filling gaps moves at most as many rows as leave (keeping the order would move
// nearly all of them), and no slot is both read and written: gaps lie below keep, the keys that fill them at or above it.
//
// The choice narrows down an interval of keys of 64 bits (whether the key is held, its weight as an ordered integer, its order) that has
// the (len - keep)-th smallest in it.  It starts at the least and the greatest weight of the keys that are not held; a pass counts the
// keys in 2048 equal parts of the interval, so that weights of all sizes spread over the parts, and once 256 keys are left, mostly
// after one pass, they are compared with each other.  Of equal keys the lowest slots leave.  No sort, and nothing depends on the order in
// which atomics arrive, because they count.  Each wave owns a run of slots; up to 24576 keys wait in registers between the passes, more
// are formed again (16 sequences of 7000 to 10001 keys, 8 KV heads, 17.5 us, with the keys in LDS 19.2; 4 of 20000 25, formed again 46).
// Bound by the instructions and waits of one workgroup's passes over its keys.
#include "cache_common.h"

namespace intattn {

namespace {

constexpr int BINS = 2048, FEW = 256;

constexpr uint64_t HELD = 1ull << 63;

// NaN above every weight, -0 as 0; orders are at least 0
__device__ __forceinline__ uint64_t sort_key(float w, int order, int sink, int newest)
{
    uint32_t u = __float_as_uint(w + 0.0f);
    u = w != w ? 0xffffffffu : (u >> 31) ? ~u : u | 0x80000000u;
    const bool held = order < sink || order >= newest;
    return (held ? HELD : 0) | ((uint64_t)u << 31) | (uint32_t)max(order, 0);
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

// ENT threads; MOST: rounds of them whose keys registers hold, 0: none
template <int ENT, int MOST> __global__ __launch_bounds__(ENT) void evict_select_kernel(const EvictParams p)
{
    constexpr int EWAVES = ENT / 64, PER = BINS / ENT;
    constexpr bool HOLD = MOST > 0;
    __shared__ int bins[BINS], sums[3][EWAVES], chosen[3], n_few;
    __shared__ uint32_t least_weight[EWAVES], most_weight[EWAVES]; // of the keys of a wave that are not held
    __shared__ int free_keys[EWAVES];                              // and how many they are
    __shared__ uint64_t few[FEW], chosen_key;
    __shared__ unsigned long long first_key, last_key;
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
    uint32_t lightest = 0xffffffffu, heaviest = 0;
    int are_free = 0;
    auto range = [&](uint64_t k) {
        const bool out = k >= HELD;
        are_free += !out;
        lightest = min(lightest, out ? 0xffffffffu : (uint32_t)(k >> 31));
        heaviest = max(heaviest, out ? 0u : (uint32_t)(k >> 31));
    };
    // The keys (behind the last: above any), and planes of their own take what lies below keep as it is; gaps are filled by the
    // next launch.
    constexpr int AT_ONCE = 8; // loads of a thread in flight
    constexpr int BATCHES = HOLD ? MOST / AT_ONCE : 1; // that are told apart, because registers have no index
    uint64_t key[HOLD ? MOST : 1];
    const int under = min(len, p.keep);
#pragma unroll BATCHES
    for (int i0 = 0; i0 < (HOLD ? MOST : rounds); i0 += AT_ONCE) {
        if (i0 >= rounds) break;
        float w[AT_ONCE];
        int o[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            if (i0 + u >= rounds) break;
            const int from = min(s0 + 64 * (i0 + u), len - 1);
            w[u] = weight[from];
            o[u] = order ? order[from] : from;
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int s = s0 + 64 * (i0 + u);
            if (i0 + u >= rounds) break;
            const uint64_t k = s < len ? sort_key(w[u], o[u], p.sink, newest) : ~0ull;
            range(k);
            if constexpr (HOLD) key[i0 + u] = k;
            if (copy_w && s < under) weight_out[s] = w[u];
            if (copy_o && s < under) order_out[s] = o[u];
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        lightest = min(lightest, (uint32_t)__shfl_xor((int)lightest, o));
        heaviest = max(heaviest, (uint32_t)__shfl_xor((int)heaviest, o));
        are_free += __shfl_xor(are_free, o);
    }
    if (lane == 0) {
        least_weight[wave] = lightest;
        most_weight[wave] = heaviest;
        free_keys[wave] = are_free;
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

    // f(slot, key, round) for each slot of the thread
    auto each = [&](auto f) {
        if constexpr (HOLD) {
#pragma unroll
            for (int i = 0; i < MOST; ++i) {
                if (i >= rounds) break;
                f(s0 + 64 * i, key[i], i);
            }
        } else {
            for (int i0 = 0; i0 < rounds; i0 += AT_ONCE) {
                uint64_t k[AT_ONCE];
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u) {
                    const int s = s0 + 64 * min(i0 + u, rounds - 1), from = min(s, len - 1);
                    k[u] = s < len ? sort_key(weight[from], order ? order[from] : from, p.sink, newest) : ~0ull;
                }
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u)
                    if (i0 + u < rounds) f(s0 + 64 * (i0 + u), k[u], i0 + u);
            }
        }
    };

    // lo .. hi has the leave-th smallest of the keys from lo on
    int leave = len - p.keep, before = 0;
    are_free = 0;
#pragma unroll
    for (int w = 0; w < EWAVES; ++w) {
        lightest = min(lightest, least_weight[w]);
        heaviest = max(heaviest, most_weight[w]);
        are_free += free_keys[w];
    }
    const bool held_leave = leave > are_free; // (then all others do)
    uint64_t lo = held_leave ? HELD : (uint64_t)lightest << 31, hi = held_leave ? ~0ull : ((uint64_t)heaviest << 31) | 0x7fffffffull;
    if (held_leave) leave -= are_free;
    bool whole = false; // every key of the interval leaves
    for (bool again = false; lo < hi && !whole; again = true) {
        if (again) { // to the keys in it: equal weights (zeros, say) leave the orders alone
            for (int i = tid; i < BINS; i += ENT) bins[i] = 0;
            if (tid == 0) {
                first_key = ~0ull;
                last_key = 0;
            }
            __syncthreads();
            uint64_t first = ~0ull, last = 0;
            each([&](int, uint64_t k, int) {
                const bool in = k >= lo && k <= hi;
                first = in && k < first ? k : first;
                last = in && k > last ? k : last;
            });
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                const uint64_t f = __shfl_xor((unsigned long long)first, o), l = __shfl_xor((unsigned long long)last, o);
                first = f < first ? f : first;
                last = l > last ? l : last;
            }
            if (lane == 0) {
                atomicMin(&first_key, (unsigned long long)first);
                atomicMax(&last_key, (unsigned long long)last);
            }
            __syncthreads();
            lo = first_key;
            hi = last_key;
            if (lo == hi) break;
        }
        const int shift = max(0, 64 - (int)__clzll(hi - lo) - 11);
        each([&](int, uint64_t k, int) {
            if (k >= lo && k <= hi) atomicAdd(&bins[(uint32_t)((k - lo) >> shift)], 1);
        });
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
        lo += (uint64_t)chosen[0] << shift;
        hi = lo + min(hi - lo, ((uint64_t)1 << shift) - 1); // (of one type: of two, min is that of doubles)
        leave = chosen[1];
        whole = chosen[2] == leave;
        if (whole || lo == hi || chosen[2] > FEW) continue;
        // few enough to compare each with all (going on bit by bit in the registers of each wave took 6.3 us for 190 keys, this 2.5)
        each([&](int, uint64_t k, int) {
            if (k >= lo && k <= hi) few[atomicAdd(&n_few, 1)] = k;
        });
        __syncthreads();
        constexpr int TEAM = ENT / FEW; // lanes to a key
        if (tid / TEAM < n_few) {
            const uint64_t mine = few[tid / TEAM];
            int less = 0, same = 0;
#pragma unroll 8
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
        lo = hi = chosen_key;
        leave = chosen[1];
        whole = chosen[2] == leave;
    }

    // Who leaves: keys below `least`, and of those on it (only where not all of them do) the first `leave` in the order of slots.
    // Gaps below keep and keys from keep on that stay are counted by the waves, then numbered and listed.
    const uint64_t least = whole ? hi + 1ull : lo; // (whole: 0 if that was the greatest key there is)
    const bool all = whole && least == 0;
    int equals = 0;
    if (!whole) {
        each([&](int, uint64_t k, int) { equals += __popcll(__ballot(k == least)); });
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
    uint32_t is_gap = 0, is_mover = 0; // of the thread, a bit for each round (HOLD: at most 24 of them)
    each([&](int s, uint64_t k, int i) {
        const bool gone = leaves(k, seen), gap = gone && s < p.keep, mover = !gone && s < len && s >= p.keep;
        is_gap |= (uint32_t)gap << (i & 31);
        is_mover |= (uint32_t)mover << (i & 31);
        gaps += __popcll(__ballot(gap));
        movers += __popcll(__ballot(mover));
    });
    const int all_gaps = sum_of_waves<EWAVES>(gaps, sums[1], gaps);
    sum_of_waves<EWAVES>(movers, sums[2], movers);
    int32_t *const to = p.moves + (int64_t)blockIdx.x * 2 * p.max_moves, *const from = to + p.max_moves;
    auto list = [&](int s, bool gap, bool mover) {
        const uint64_t mg = __ballot(gap), mm = __ballot(mover);
        if (gap) to[gaps + __popcll(mg & below)] = s;
        if (mover) from[movers + __popcll(mm & below)] = s;
        gaps += __popcll(mg);
        movers += __popcll(mm);
    };
    if constexpr (HOLD) {
        for (int i = 0; i < rounds; ++i) list(s0 + 64 * i, (is_gap >> i) & 1u, (is_mover >> i) & 1u);
    } else {
        seen = equals;
        each([&](int s, uint64_t k, int) {
            const bool gone = leaves(k, seen);
            list(s, gone && s < p.keep, !gone && s < len && s >= p.keep);
        });
    }
    if (tid == 0) p.count[blockIdx.x] = all_gaps;
}

// Rows to their gaps.  A workgroup looks up the places of 64 moves at once, and then moves their rows, 2 d / 16 lanes to a row of K and
// one of V, with all loads of a lane on their way together.  Bound by reads and writes of single rows in no order: 218 000 of them, 128
// bytes of K and of V each, in 27 us, 4.1 TB/s (a row to 16 lanes, each looking up its own places: 34 us).
constexpr int MOVES = 64; // of a workgroup of 256 threads: four jobs to each
template <int D> __global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams p)
{
    constexpr int LANES = D / 8, ROWS = 256 / LANES, EACH = MOVES / ROWS; // lanes (of 16 bytes) to a move, moves at once, of a lane
    __shared__ int64_t place[2][2][MOVES]; // [K, V][to, from]
    const int bh = blockIdx.y, b = bh / p.c.Hkv, kvh = bh % p.c.Hkv, n = p.count[bh];
    if (blockIdx.x == 0 && kvh == 0 && threadIdx.x == 0) p.lens_out[b] = p.count[p.c.B * p.c.Hkv + b];
    const int32_t *const to = p.moves + (int64_t)bh * 2 * p.max_moves, *const from = to + p.max_moves, *const row = p.c.table + b * p.c.table_stride;
    const int part = threadIdx.x % LANES, value = part >= LANES / 2;
    int8_t *const base = value ? p.c.v + kvh * p.c.vs[1] + 16 * (part - LANES / 2) : p.c.k + kvh * p.c.ks[1] + 16 * part;
    const int i0 = blockIdx.x * MOVES, some = min(MOVES, n - i0), m = threadIdx.x % MOVES, job = threadIdx.x / MOVES;
    if (some <= 0) return;
    if (m < some) {
        if (job < 2) {
            const Slot s = find_slot(p.c, row, (job == 0 ? to : from)[i0 + m]);
            place[0][job][m] = s.page * p.c.ks[0] + s.at * p.c.ks[2];
            place[1][job][m] = s.page * p.c.vs[0] + s.at * p.c.vs[2];
        } else if (job == 2) {
            p.weight_out[b * p.wost[0] + kvh * p.wost[1] + to[i0 + m]] = p.weight[b * p.wst[0] + kvh * p.wst[1] + from[i0 + m]];
        } else if (p.order_out) {
            p.order_out[b * p.oost[0] + kvh * p.oost[1] + to[i0 + m]] = p.order[b * p.ost[0] + kvh * p.ost[1] + from[i0 + m]];
        }
    }
    __syncthreads();
    v4i x[EACH];
    const int first = threadIdx.x / LANES;
#pragma unroll
    for (int u = 0; u < EACH; ++u) x[u] = __builtin_nontemporal_load((const v4i *)(base + place[value][1][min(first + u * ROWS, some - 1)]));
#pragma unroll
    for (int u = 0; u < EACH; ++u)
        if (first + u * ROWS < some) __builtin_nontemporal_store(x[u], (v4i *)(base + place[value][0][first + u * ROWS]));
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
    // 512 threads where few slots leave more of them idle, and where a compute unit gets more than one workgroup, which it then holds at once
    // (1024 threads and 512, us: 32 workgroups of 1150 keys 11.2, 9.8, of 4000 11.0, 10.7, 8 of 8000 16.7, 17.5; 480 of 1100 21.1, 13.7, of
    // 4000 27.7, 18.8, of 6000 29.2, 22.0, of 8000 28.5, 24.0)
    const bool half = p.c.capacity <= (groups > 256 ? 24 * 512 : 8 * 512);
    void (*select)(const EvictParams) = evict_select_kernel<1024, 0>;
    if (half) select = p.c.capacity <= 8 * 512 ? evict_select_kernel<512, 8> : evict_select_kernel<512, 24>;
    else if (p.c.capacity <= 24 * 1024) select = evict_select_kernel<1024, 24>;
    const int threads = half ? 512 : 1024;
    hipLaunchKernelGGL(select, dim3((uint32_t)groups), dim3((uint32_t)threads), 0, (hipStream_t)stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (int)e;
    const int fit = (p.max_moves + MOVES - 1) / MOVES;
    hipLaunchKernelGGL(p.d == 64 ? evict_move_kernel<64> : evict_move_kernel<128>, dim3((uint32_t)(fit < 1 ? 1 : fit), (uint32_t)groups), dim3(256), 0,
                       (hipStream_t)stream, p);
    return (int)hipGetLastError();
}

} // namespace intattn
