// The context behind the C ABI and what its entry points share.  Not part of the public ABI (that is include/intattn.h).
#pragma once
#include <hip/hip_runtime.h>

#include <string>
#include <vector>

#include "../../include/intattn.h"
#include "params.h"

using namespace intattn;

// Pinned host staging for small host-to-device uploads (per-head tables): the bytes are copied here
// first, so the asynchronous copy never reads memory that the caller, or a returning function, owns.
struct Staging {
    unsigned char *host = nullptr;
    hipEvent_t done = nullptr;
    bool pending = false;
};
constexpr size_t STAGING_BYTES = 65536;

struct intattn_ctx {
    int device = 0;
    int lut_bits = 5;
    double clip = 6.6;
    int variant = 0;
    uint8_t lut[64] = {0};
    // device-side per-head tables (allocated on first per-head call, grown on demand)
    HeadParams *d_hp = nullptr;
    float *d_alpha = nullptr, *d_svso = nullptr;
    int table_cap = 0;
    // kernel workspace (row max and row sum between the two launches; partial results of the split-key kernels), grown on demand
    int32_t *d_ws = nullptr;
    size_t ws_cap = 0; // in int32 elements
    // room of the key-split launches, apart from the workspace: a smaller problem may need more of it than a larger one, and
    // captured launches keep the pointers they were recorded with, so an outgrown piece stays until the context goes
    int32_t *d_split = nullptr, *split_outgrown[KEY_SPLIT_PIECES] = {nullptr};
    int n_split_outgrown = 0;
    size_t split_cap = 0; // in int32 elements
    bool split_fixed = false; // a reservation could not have it all: what is there now is all there will be
    HeadParams *d_rowtab = nullptr; // parameters per block of query rows (scale_mode 2), grown on demand
    uint32_t *d_dec_state = nullptr; // fused split-key kernel: DEC_STATE_WORDS per (batch, KV head) group, zero between launches
    size_t dec_state_groups = 0;
    size_t rowtab_cap = 0;
    int32_t *d_status = nullptr; // per head: what the last derivation on the device found (intattn_dynamic_status)
    int status_cap = 0, status_n = 0;
    float *d_amax = nullptr; // scratch of the quantizer: partial max|X| per workgroup of its first pass
    int64_t amax_cap = 0;
    // parameters derived from the host scales of the last call (the search for index-map constants costs
    // microseconds per head; serving loops pass the same scales again and again)
    std::vector<uint32_t> dv_key;
    std::vector<HeadParams> dv_hp;
    std::vector<float> dv_alpha, dv_svso;
    int dv_mode = 0;
    std::vector<HeadParams> hp_host;  // what d_hp currently holds
    std::vector<float> alpha_host, svso_host;
    Staging stage[2];
    int stage_next = 0;
    // room of the cache operators; what it outgrows stays until the context goes, like the key-split launches'
    void *d_cache_room = nullptr;
    size_t cache_room_bytes = 0;
    std::vector<void *> cache_room_outgrown;
    std::string err;
};

namespace intattn {

// Records msg on the context (without one: as the text of the last failed intattn_create on this thread) and returns code.
int fail(intattn_ctx *ctx, int code, const std::string &msg);
int hip_fail(intattn_ctx *ctx, hipError_t e, const char *what);

// Scoped "make ctx->device current", restoring the caller's device afterwards.
struct DeviceGuard {
    int prev = -1;
    bool changed = false;
    hipError_t status = hipSuccess;
    explicit DeviceGuard(int dev)
    {
        status = hipGetDevice(&prev);
        if (status == hipSuccess && prev != dev) {
            status = hipSetDevice(dev);
            changed = (status == hipSuccess);
        }
    }
    ~DeviceGuard()
    {
        if (changed) (void)hipSetDevice(prev);
    }
};

} // namespace intattn
