// Eviction from a paged cache by accumulated attention weight, for gfx950.  Two launches: a workgroup for each (sequence, KV head)
// finds the keys that leave and pairs the gaps among the first `keep` slots with the keys that stay behind them; then rows are
// moved, by as many workgroups as there are rows.  Filling gaps moves at most as many rows as leave (keeping the order would move
// nearly all of them), and no slot is both read and written: gaps lie below keep, the keys that fill them at or above it.
//
// The choice is a radix selection: the key of a slot is 64 bits, its weight as an ordered integer above its order, and eight
// passes at most over its digits of 8 bits find the (len - keep)-th smallest; the slot decides between equal keys.  No sort, and
// nothing depends on the order in which atomics arrive (they count).
#include "cache_common.h"

namespace intattn {

namespace {

constexpr int ENT = 1024, EWAVES = ENT / 64;

// weight above order, ordered as unsigned integers; NaN above everything
__device__ __forceinline__ uint64_t sort_key(float w, int order)
{
    uint32_t u = __float_as_uint(w + 0.0f); // (-0 as 0)
    u = (u >> 31) ? ~u : u | 0x80000000u;
    if (w != w) u = 0xffffffffu;
    return ((uint64_t)u << 32) | ((uint32_t)order ^ 0x80000000u);
}

struct HeadKeys {
    const float *weight;
    const int32_t *order; // null: the slot
    int sink, newest;     // orders below sink or from newest on are held
    __device__ __forceinline__ int order_of(int slot) const { return order ? order[slot] : slot; }
    __device__ __forceinline__ uint64_t key(int slot, bool &held) const
    {
        const int o = order_of(slot);
        held = o < sink || o >= newest;
        return sort_key(weight[slot], o);
    }
};

// number of threads below this one whose flag is set, and of all; two barriers
__device__ __forceinline__ int rank_of(bool flag, int *waves, int &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t m = __ballot(flag);
    if (lane == 0) waves[wave] = __popcll(m);
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < EWAVES; ++w) {
        before += w < wave ? waves[w] : 0;
        total += waves[w];
    }
    __syncthreads();
    return before + __popcll(m & ((1ull << lane) - 1ull));
}

__global__ __launch_bounds__(ENT) void evict_select_kernel(const EvictParams p)
{
    __shared__ int bins[256], waves[EWAVES], chosen[2];
    const int b = blockIdx.x / p.c.Hkv, kvh = blockIdx.x % p.c.Hkv, tid = threadIdx.x;
    const int len = cache_len(p.c, b);
    const int32_t *row = p.c.table + b * p.c.table_stride;
    bool lost = false;
    if (len > p.keep)
        for (int i = tid; i <= quotient(len - 1, p.c.by_page); i += ENT) lost |= (uint32_t)row[i] >= (uint32_t)p.c.n_pages;
    const bool stays = len <= p.keep || __syncthreads_or(lost);
    const int fresh_len = stays ? len : p.keep;
    if (kvh == 0 && tid == 0) p.count[p.c.B * p.c.Hkv + b] = fresh_len;

    const int64_t total = p.total ? (int64_t)p.total[b] : (int64_t)len;
    const int64_t newest = total - p.recent;
    const HeadKeys keys{p.weight + b * p.wst[0] + kvh * p.wst[1], p.order ? p.order + b * p.ost[0] + kvh * p.ost[1] : nullptr, p.sink,
                        (int)max(newest, (int64_t)-0x7fffffff - 1)};
    float *const weight_out = p.weight_out + b * p.wost[0] + kvh * p.wost[1];
    int32_t *const order_out = p.order_out ? p.order_out + b * p.oost[0] + kvh * p.oost[1] : nullptr;
    if (stays) {
        for (int s = tid; s < len; s += ENT) {
            if (weight_out != keys.weight) weight_out[s] = keys.weight[s];
            if (order_out && order_out != keys.order) order_out[s] = keys.order[s];
        }
        if (tid == 0) p.count[blockIdx.x] = 0;
        return;
    }

    // whether the keys that are not held are enough; the class that the last key to leave is in, and its number there
    int leave = len - p.keep;
    if (tid == 0) waves[0] = 0;
    __syncthreads();
    int free_keys = 0;
    for (int s = tid; s < len; s += ENT) {
        const int o = keys.order_of(s);
        free_keys += !(o < keys.sink || o >= keys.newest);
    }
    if (free_keys) atomicAdd(&waves[0], free_keys);
    __syncthreads();
    const bool into_held = waves[0] < leave;
    if (into_held) leave -= waves[0];
    __syncthreads();

    // prefix: the first digits of the leave-th smallest key of the class; leave: how many keys with that prefix leave
    uint64_t prefix = 0;
    int shift = 64;
    bool whole = false; // every key with the prefix leaves
    while (shift > 0 && !whole) {
        shift -= 8;
        for (int i = tid; i < 256; i += ENT) bins[i] = 0;
        __syncthreads();
        for (int s = tid; s < len; s += ENT) {
            bool held;
            const uint64_t k = keys.key(s, held);
            if (held == into_held && (shift == 56 || (k >> (shift + 8)) == prefix)) atomicAdd(&bins[(k >> shift) & 0xff], 1);
        }
        __syncthreads();
        if (tid < 64) { // four bins a lane
            int four[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += four[i] = bins[4 * tid + i];
            int before = sum;
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                const int up = __shfl_up(before, o);
                if (tid >= o) before += up;
            }
            before -= sum;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (before < leave && leave <= before + four[i]) {
                    chosen[0] = 4 * tid + i;
                    chosen[1] = leave - before;
                }
                before += four[i];
            }
        }
        __syncthreads();
        prefix = (prefix << 8) | (uint64_t)chosen[0];
        leave = chosen[1];
        whole = bins[chosen[0]] == leave;
        __syncthreads();
    }

    // who leaves, in the order of slots; gaps below keep and keys from keep on that stay are numbered and listed
    int32_t *const to = p.moves + (int64_t)blockIdx.x * 2 * p.max_moves, *const from = to + p.max_moves;
    int gaps = 0, movers = 0, equals = 0;
    for (int s0 = 0; s0 < len; s0 += ENT) {
        const int s = s0 + tid;
        bool gone = false, equal = false;
        float w = 0.0f;
        int o = 0;
        if (s < len) {
            bool held;
            const uint64_t k = keys.key(s, held);
            const uint64_t front = shift ? k >> shift : k;
            gone = held == into_held ? front < prefix || (whole && front == prefix) : into_held;
            equal = held == into_held && !whole && front == prefix;
            w = keys.weight[s];
            o = keys.order_of(s);
        }
        int n;
        if (!whole) { // equal keys: the first `leave` of them (uniform)
            const int r = equals + rank_of(equal, waves, n);
            gone |= equal && r < leave;
            equals += n;
        }
        const bool gap = gone && s < p.keep, mover = s < len && !gone && s >= p.keep;
        const int g = gaps + rank_of(gap, waves, n);
        gaps += n;
        const int m = movers + rank_of(mover, waves, n);
        movers += n;
        if (gap) to[g] = s;
        if (mover) from[m] = s;
        if (s < p.keep && s < len && !gone) {
            if (weight_out != keys.weight) weight_out[s] = w;
            if (order_out && order_out != keys.order) order_out[s] = o;
        }
    }
    if (tid == 0) p.count[blockIdx.x] = gaps;
}

// Rows to their gaps: 2 d / 16 lanes a key, K then V.
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
        *(int4 *)(base + z.page * st[0] + z.at * st[2]) = *(const int4 *)(base + a.page * st[0] + a.at * st[2]);
        if (part == 0) {
            p.weight_out[b * p.wost[0] + kvh * p.wost[1] + dst] = p.weight[b * p.wst[0] + kvh * p.wst[1] + src];
            if (p.order_out) p.order_out[b * p.oost[0] + kvh * p.oost[1] + dst] = p.order[b * p.ost[0] + kvh * p.ost[1] + src];
        }
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
    hipLaunchKernelGGL(evict_select_kernel, dim3((uint32_t)groups), dim3(ENT), 0, (hipStream_t)stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (int)e;
    const int rows = 2048 / p.d; // moves of a workgroup at a time
    const int blocks = p.max_moves <= 0 ? 1 : (p.max_moves + rows - 1) / rows < 64 ? (p.max_moves + rows - 1) / rows : 64;
    hipLaunchKernelGGL(p.d == 64 ? evict_move_kernel<64> : evict_move_kernel<128>, dim3((uint32_t)blocks, (uint32_t)groups), dim3(256), 0,
                       (hipStream_t)stream, p);
    return (int)hipGetLastError();
}

} // namespace intattn
