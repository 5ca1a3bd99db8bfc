// Parameters of the kernels around the paged cache.  Not part of the public ABI (that is include/intattn.h).
#pragma once
#include <stdint.h>

#include "params.h"

namespace intattn {

// Bytes of room for scores that a call may ask for: with more (sequence, KV head) groups than that serves, the launches take some groups after
// the others (one group may need more: 2.1 GiB with 4096 rows of 131 071 keys)
constexpr int64_t SCORE_ROOM = 1ll << 30;

struct CacheParams {
    int8_t *k, *v;
    int64_t ks[3], vs[3];      // bytes between pages, heads, keys
    const int32_t *table;
    int64_t table_stride;
    const int32_t *lens;
    const float *scale_k, *scale_v;
    int32_t B, Hkv;
    int32_t n_pages, page_size, capacity; // capacity: the most slots a sequence is taken to have
    int32_t per_head;
    FastDiv by_page;           // of slot numbers by page_size
};

struct RotaryParams {
    const int32_t *pos;
    int64_t ps[3];
    const double *freq;
    int32_t rot, halves, inverse;
    uint32_t axis[32];         // four axes of pairs to a word
};

struct RopeParams {
    const uint8_t *src[2];
    uint8_t *dst[2];
    int64_t ss[2][3], ds[2][3];
    int32_t H0, H;             // heads of the first tensor, of both
    int32_t B, L, d;
    int32_t tokens;            // of a workgroup
    int32_t units, per_token;  // 32-byte units of a row, of a token
    FastDiv by_token, by_units, by_pairs, by_L;
    RotaryParams r;
};

struct AppendParams {
    CacheParams c;
    const uint8_t *x[3];       // q, k, v
    int64_t xs[3][3];
    int32_t Hq, L, heads;      // heads: of Q, K and V
    int32_t tokens;            // of a workgroup
    int32_t turns_at;          // bytes of LDS in front of the turns
    FastDiv by_heads, by_L, by_pairs;
    const int32_t *n_new;
    int8_t *q_out;
    int64_t qos[3];
    float *q_scale;
    float *weight;
    int32_t *order;
    const int32_t *first;
    int64_t wst[2], ost[2];
    RotaryParams r;
};

// What the kernels need of a row of a KV head
struct RowParams {
    double factor;   // the double after top / c_int
    float unit;      // floating-point output of one step of the accumulator
    int32_t c_int;
    int32_t limit;   // slots that the row sees (attend_split.hip: whether its scales are usable)
    int32_t mult, shift;
};

struct AttendParams {
    CacheParams c;
    const int8_t *q;
    int64_t qs[3];
    const float *scale_q;
    const int32_t *n_new;
    uint8_t *out;
    int64_t os[3];
    const float *scale_out;
    int32_t out_per_head;
    const float *weight;
    float *weight_out;
    int64_t wst[2], wost[2];
    float decay;
    int32_t Hq, L, group;      // group = Hq / Hkv
    int32_t rows, blocks;      // group * L rows of a KV head, in blocks of 16
    int32_t first;             // (sequence, KV head) whose part of the room is the first: that of the launch's first workgroups
    int32_t out_type;
    int32_t top;
    double clip, sqrt_d;
    uint32_t lut[16];
    // one launch: steps of 64 keys whose scores LDS holds; room for what blocks of rows draw from the keys, if there are several
    int32_t held_steps;
    float *drawn;
    // keys split over workgroups (attend_split.hip): steps of a sequence of capacity slots, and for each launch the steps of a
    // workgroup and the workgroups of a sequence.  Room: scores [group][steps][4][rows][16], maxima and sums [group][chunks of that
    // launch][rows], accumulators [group][block of rows][chunks][16][d], arrivals [group][block of rows], sums and parameters
    // [group][rows]; a group is a (sequence, KV head) from `first` on
    int32_t steps, score_steps, score_chunks, lookup_steps, lookup_chunks, chunk_steps, chunks;
    int32_t *scores, *part_max, *part_sum, *part_acc, *arrived, *row_sum;
    RowParams *row_params;
};

struct EvictParams {
    CacheParams c;
    int32_t keep, sink, recent;
    const float *weight;
    float *weight_out;
    const int32_t *order;
    int32_t *order_out;
    int64_t wst[2], wost[2], ost[2], oost[2];
    const int32_t *total;
    int32_t *lens_out;
    int32_t *count;            // room: moves of each (sequence, KV head), and then the new length of each sequence
    int32_t *moves;            // room: [B * Hkv][2][max_moves], the slots to fill and the slots to fill them from
    int32_t max_moves, d;
};

int launch_rope(const RopeParams &p, int dtype, void *stream);
int launch_append(const AppendParams &p, int d, int dtype, void *stream);
// bytes of room that launch_attend needs for these parameters
int64_t attend_room(const AttendParams &p, int d);
// and for any with at most as many rows, with weights or without
int64_t attend_room_upto(const AttendParams &p, int d);
int launch_attend(const AttendParams &p, int d, void *room, void *stream);
int64_t attend_split_room(const AttendParams &p, int d);
int launch_attend_split(const AttendParams &p, int d, void *room, void *stream);
int64_t evict_room(const EvictParams &p);
int launch_evict(const EvictParams &p, void *room, void *stream);

} // namespace intattn
