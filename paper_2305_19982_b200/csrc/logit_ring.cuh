// What the roles of the ring kernel on rows of logits share: its shared memory and its cursors.
#pragma once

#include "bulk_copy.cuh"
#include "policy_plan.h"
#include "softmax_rows.cuh"

namespace adama {

// The slice of a row's units that CTA `rank` of 2^log_size takes (units < 2^29, so 32 bits hold it).
__device__ __forceinline__ void slice_of(int units, int rank, int log_size, int &from, int &count) {
    from = (int)(((unsigned)units * (unsigned)rank) >> log_size);
    count = (int)(((unsigned)units * (unsigned)(rank + 1)) >> log_size) - from;
}

// Sums of one thread over its rows; in double, so that their order does not show in fp32.
struct Sums {
    double v[4] = {0.0, 0.0, 0.0, 0.0};

    __device__ __forceinline__ void add(double w, float a, float b, float c, float d) {
        v[0] += w * a;
        v[1] += w * b;
        v[2] += w * c;
        v[3] += w * d;
    }
};

// What the gradient of a row needs.
struct Verdict {
    float top, unit, per_e, x_target;
    int64_t target;
    int writer;  // the thread that writes the target's element, or -1
};

// Two of each, for even and odd live rows: nobody is more than one row ahead.
template <typename Cut>
struct RingShared {
    alignas(128) unsigned char stage[Cut::kStages][Cut::kStageBytes];
    alignas(16) float4 peer[2][kMaxCluster];  // {top, sum, x_target} of the cluster's CTAs
    Verdict verdict[2];
    float2 slots[2][Cut::kWarps];             // {top, sum} of the warps
    unsigned long long full[Cut::kStages], empty[Cut::kStages], joined[2], peered[2], ready[2];
    double sums[1][4];
    int last, give_up;
};
static_assert(sizeof(RingShared<Cut512>) + 128 <= 232448 && sizeof(RingShared<Cut640>) + 128 <= 232448, "shared memory of a CTA");
static_assert(2 * (sizeof(RingShared<Cut256>) + 128 + 1024) <= 233472 &&
                  4 * (sizeof(RingShared<Cut128>) + 128 + 1024) <= 233472 &&
                  8 * (sizeof(RingShared<Cut64>) + 128 + 1024) <= 233472,
              "shared memory of an SM");

// Place in the ring: a stage, and the parity of the barrier phase that its current use completes.
template <int STAGES>
struct Cursor {
    uint32_t slot = 0, parity = 0;

    __device__ __forceinline__ void advance() {
        if (++slot == STAGES) {
            slot = 0;
            parity ^= 1;
        }
    }
};

__device__ __forceinline__ Stats join2(const Stats &a, const Stats &b, float k) {
    const float top = fmaxf(a.top, b.top);
    const Stats p = raised(a, top, k), q = raised(b, top, k);
    return {top, p.sum + q.sum, 0.f};
}

}  // namespace adama
