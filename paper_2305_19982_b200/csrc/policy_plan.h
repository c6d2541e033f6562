// Which form of the kernels on rows of logits takes a call: plain host code, without CUDA, so that its
// rules can be tested for any card.
#pragma once

#include <stdint.h>

namespace adama {

constexpr int kMaxCluster = 8;  // CTAs that may share a row
constexpr int kRowUnits = 8;    // 16-byte units of a lane where a warp holds a row in registers: rows of up to 4 KB

// How a ring in shared memory is cut: WORK threads compute, a stage holds two units of each, PER_SM such
// CTAs share an SM.
template <int WORK, int STAGES, int PER_SM>
struct RingCut {
    static constexpr int kWork = WORK, kStages = STAGES, kPerSm = PER_SM;
    static constexpr int kEach = 2;                              // units of a stage that a thread takes
    static constexpr int kWarps = WORK / 32, kThreads = WORK + 64;
    static constexpr int kProducerWarp = kWarps, kScalarWarp = kWarps + 1;
    static constexpr int kStageUnits = kEach * WORK, kStageBytes = 16 * kStageUnits;
    static constexpr int kSliceUnits = STAGES / 2 * kStageUnits;  // largest slice of which two fit

    // stages of a slice times their units, in percent of the slice
    static int fill_cost(int64_t slice) {
        return (int)((slice + kStageUnits - 1) / kStageUnits * kStageUnits * 100 / slice);
    }
};
// The shorter the slice, the fewer threads to it and the more CTAs to an SM: a row's joins and barriers
// then cost fewer warps, and other rows' work hides its latencies (24390 x 8200 bf16: 250 us with 512
// threads, 160 with 256, 134 with 128; 48828 x 4096: 151 with 128, 132 with 64; 8333 x 24000: 139 with 512, 131 with 256).
using Cut640 = RingCut<640, 11, 1>;  // 11 stages of 20 KB: slices of up to 6400 units
using Cut512 = RingCut<512, 14, 1>;  // 14 of 16 KB: 7168
using Cut256 = RingCut<256, 13, 2>;  // 13 of 8 KB: 3072
using Cut128 = RingCut<128, 13, 4>;  // 13 of 4 KB: 1536
using Cut64 = RingCut<64, 13, 8>;    // 13 of 2 KB: 768

enum PolicyForm { kFormRows, kForm64, kForm128, kForm256, kForm512, kForm640, kFormLong };

// The cut of a whole SM: a stage that a row fills in part costs nearly as much as a full one, so the cut
// that fills better: 8192 x 50257 bf16 (6282 units, 114 % with Cut512, 102 % with Cut640) 259 and 251 us,
// 4096 of them with odd pitches 159 and 147; 8192 x 32000 (4000 units, 102 % and 128 %) 160 and 168 us.  On
// a tie the deeper ring.
inline PolicyForm whole_sm_cut(int64_t slice) {
    return Cut640::fill_cost(slice) < Cut512::fill_cost(slice) ? kForm640 : kForm512;
}

struct PolicyPlan {
    PolicyForm form;
    int cluster;    // CTAs that share a row
    bool one_turn;  // one row to a cluster: its ring has to hold one slice, not two
};

// `units` 16-byte units to a row.  resident(form, cluster, &most) gives the number of clusters of that form
// which run at a time; it returns 0, or an error that ends the planning and is returned.
template <typename Resident>
int plan_policy(int64_t units, int64_t rows, int sm_count, Resident resident, PolicyPlan &plan) {
    plan = {kFormRows, 1, false};
    if (units <= 32 * kRowUnits) return 0;
    // As few CTAs to a row as hold two of its slices.  Few rows are dealt out at once, one to a cluster as
    // large as that and the row's length allow, which then has to hold one slice (33 x 131072 fp32: 10.0 us
    // with 4 CTAs to a row, 10.9 with 8 in three turns).  A second row would wait in such a ring for ever:
    // what is asked about is the cut that will be launched.
    while (plan.cluster < kMaxCluster && (units + plan.cluster - 1) / plan.cluster > Cut512::kSliceUnits) plan.cluster *= 2;
    constexpr int64_t kHeld640 = Cut640::kStages * Cut640::kStageUnits, kHeld512 = Cut512::kStages * Cut512::kStageUnits;
    for (int c = kMaxCluster; c >= 1 && !plan.one_turn; c /= 2) {
        const int64_t slice = (units + c - 1) / c;
        if (rows * c > sm_count || slice > (kHeld640 < kHeld512 ? kHeld640 : kHeld512)) continue;
        if (c > 1 && units < (int64_t)c * Cut512::kWork) continue;
        int most = 0;
        const int e = resident(whole_sm_cut(slice), c, &most);
        if (e != 0) return e;
        if (rows <= most) {
            plan.cluster = c;
            plan.one_turn = true;
        }
    }
    const int64_t slice = (units + plan.cluster - 1) / plan.cluster;
    if (plan.one_turn) {
        plan.form = whole_sm_cut(slice);
    } else if (slice <= Cut64::kSliceUnits) {
        plan.form = kForm64;
    } else if (slice <= Cut128::kSliceUnits) {
        plan.form = kForm128;
    } else if (plan.cluster == 1 && slice <= Cut256::kSliceUnits) {
        // (only whole rows: the halves of 6250 x 32000 in clusters take 131 us, whole rows with Cut512 124)
        plan.form = kForm256;
    } else if (slice <= Cut640::kSliceUnits && whole_sm_cut(slice) == kForm640) {
        plan.form = kForm640;
    } else {
        plan.form = slice <= Cut512::kSliceUnits ? kForm512 : kFormLong;
    }
    return 0;
}

// Log-probabilities of many long rows: warps to a row, 4 or 8, one row to a CTA, of which `resident4` and
// `resident8` fit an SM at a time (fp32 10 and 5; bf16 12 and 6 with entropy, 16 and 8 without).  The rows of
// an SM take whole turns of that many; the smaller CTAs wait less at a row's end, the larger ones waste
// less of a last turn that is not full.  So 8 where that leaves fewer places unused, up to two turns of the
// smaller ones; then turns no longer tell.  With entropy, us with 4 / 8 warps, fp32 of 128256: 740 rows 65.6 /
// 57.4, 800 68.2 / 78.5, 1480 109.2 / 109.5, 1600 150.9 / 133.2, 2048 166.3 / 151.3, 2368 177.9 / 184.4; bf16 of
// 50257: 592 rows 17.8 / 15.7, 1024 23.1 / 25.4, 1480 29.7 / 31.8, 2048 43.3 / 41.0, 4096 70.9 / 72.3.  Of 189 such
// points (444 to 4096 rows of 13000 to 128256) the choice costs 0.3 % over the better of the two on average, at
// most 8 % (3000 fp32 rows: 251.0 and 232.6); without entropy 0.4 % and 8 %.  16 warps are faster still at some
// points (1600 and 3000 of those rows: 119.9 and 216.9) and slower at most.
inline int warps_to_a_row(int64_t rows, int sm_count, int resident4, int resident8) {
    const int64_t per_sm = (rows + sm_count - 1) / sm_count;
    const auto places = [&](int resident) { return (per_sm + resident - 1) / resident * resident; };
    return per_sm <= 2 * resident4 && places(resident8) < places(resident4) ? 8 : 4;
}

}  // namespace adama
