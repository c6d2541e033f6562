// Token log-probabilities, the clipped policy loss with its gradient, and (the part of a row that is no entry's; the entries'
// is in distill.cuh) the divergence from a teacher with its gradient, from rows of logits.
// With z = s*x (s = logit_scale) a row's lse = log sum_j exp(z_j), p_j = exp(z_j - lse),
// logp = z_target - lse, entropy = lse - sum_j p_j z_j.  For a row with weight w:
//     r = exp(logp - old),  pg = -min(r*A, clamp(r, 1-cl, 1+ch)*A),  d = ref - logp,
//     kl = exp(d) - d - 1,  loss += w*(pg + beta*kl)
//     dlogits_j = w*s*c*([j = target] - p_j),  c = -(r*A while r*A <= the clamped product) + beta*(1 - exp(d))
// A row is read once (loss: and its gradient written once).  Beside HBM the exponentials count, one per
// element for the statistics and one for the gradient, at 16 per clock and SM.  Log-probabilities of 4096 rows
// of 50304 bf16 with entropy: 69 us = 5.98 TB/s; loss and gradient of 8192 rows of 50257, a quarter of them
// masked: 252 us = 5.7 TB/s, of 6103 rows of 32768, which fill the ring's stages, 119 us = 5.9 TB/s; the
// log-probability of one row of 50257 fp32: 3.9 us.  Distillation of 4096 x 50257 bf16 from 64 entries, a quarter masked:
// 150 us = 4.8 TB/s, of 24 x 32000 fp32 10.3 us, in three kernels.

#include "adama_device.cuh"
#include "bulk_copy.cuh"
#include "chained.cuh"
#include "distill.cuh"
#include "logit_ring.cuh"
#include "row_writer.cuh"

#include <type_traits>

namespace adama {
namespace {

constexpr int kThreads = 512;  // that work on rows, in every kernel here
constexpr int kWarps = kThreads / 32;

// Barrier of the W warps that share a row: group g of the CTA.
template <int W>
__device__ __forceinline__ void group_sync(int g) {
    if (W == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + g), "n"(W * 32) : "memory");
}

// Union over the W warps of a group, in every thread; `slots` (W of them) are the group's own, and
// are free again after the caller's next group_sync.
template <int W, bool ENT>
__device__ __forceinline__ Stats group_join(Stats s, float k, Stats *slots, int g) {
    s = warp_join<ENT>(s, k);
    if (W == 1) return s;
    const int lane = threadIdx.x % 32;
    if (lane == 0) slots[threadIdx.x / 32 % W] = s;
    group_sync<W>(g);
    const Stats none = {-CUDART_INF_F, 0.f, 0.f};
    return warp_join<ENT>(lane < W ? slots[lane] : none, k);
}

// In natural units: the rounding of k does not show but through the sum.
__device__ __forceinline__ float logp_of(float x_target, const Stats &s, float log_sum, float scale) {
    return fmaf(scale, x_target - s.top, -log_sum);
}

__device__ __forceinline__ void store_peer(const Stats *slot, uint32_t rank, const Stats &s) {
    store12(shared_addr(slot), rank, s.top, s.sum, s.wsum);
}

// ---- token log-probabilities -----------------------------------------------------------------

// W warps to a row (or to the slice of a row that a cluster of CTAs shares), ROWS rows to a CTA, kLoads
// units of each thread in flight.  4096 x 50304: 69.5 us with 4 warps, 76.7 with 2; 70.5 with 8 units in
// flight; 94 when CTAs of 16 warps walked the rows.
constexpr int kLoads = 4;

template <typename T, int W, int ROWS, bool ENT, bool CLUSTER>
__global__ void __launch_bounds__(32 * W * ROWS)
token_logprobs_kernel(const LogprobArgs a, float k, int log_cluster) {
    constexpr int kGroupThreads = 32 * W;
    __shared__ Stats shared[W * ROWS], peers[kMaxCluster];
    const int g = threadIdx.x / kGroupThreads, t = threadIdx.x % kGroupThreads;
    const int rank = CLUSTER ? (int)cluster_rank() : 0;
    const int64_t row = CLUSTER ? blockIdx.x >> log_cluster : (int64_t)blockIdx.x * ROWS + g;
    if (row >= a.rows) return;  // a whole group
    const int64_t target = a.targets[row];
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    float logp = 0.f, lse = 0.f, entropy = 0.f;
    if (target >= 0) {
        if (CLUSTER) cluster_arrive();
        const bool inside = target < a.vocab;
        const float x_target = inside ? widen(x[target]) : CUDART_NAN_F;
        const RowShape shape = row_shape(x, (int)a.vocab);
        const uint4 *body = reinterpret_cast<const uint4 *>(x + shape.head);
        const bool has_extra = rank == 0 && t < shape.head + shape.tail;
        const float x_extra = has_extra ? widen(x[extra_index<T>(shape, t)]) : -CUDART_INF_F;
        int i = t, end = shape.units;
        if (CLUSTER) {
            slice_of(shape.units, rank, log_cluster, i, end);
            end += i;
            i += t;
        }
        Running<ENT> run;
        for (; i + (kLoads - 1) * kGroupThreads < end; i += kLoads * kGroupThreads) {
            uint4 u[kLoads];
#pragma unroll
            for (int j = 0; j < kLoads; ++j) u[j] = ld_unit_ro(body + i + j * kGroupThreads);
            run.template add_units<T>(u, k);
        }
        {
            uint4 u[kLoads - 1];  // what is left, loaded together
#pragma unroll
            for (int j = 0; j < kLoads - 1; ++j) {
                u[j] = nothing<T>();
                if (i + j * kGroupThreads < end) u[j] = ld_unit_ro(body + i + j * kGroupThreads);
            }
            run.template add_units<T>(u, k);
        }
        run.add_one(x_extra, k);
        Stats s = group_join<W, ENT>(run.stats(), k, shared + g * W, g);
        if (CLUSTER) {  // to the first CTA's shared memory
            cluster_wait();  // it has begun
            if (t == 0) store_peer(&peers[rank], 0, s);
            __syncwarp();  // the cluster's barrier is for whole warps
            cluster_sync();
            if (rank != 0) return;
            const Stats none = {-CUDART_INF_F, 0.f, 0.f};
            const int lane = t % 32;
            s = warp_join<ENT>(lane < 1 << log_cluster ? peers[lane] : none, k);
        }
        const float log_sum = logf(s.sum), scale = (float)a.scale;
        lse = fmaf(s.top, scale, log_sum);
        logp = logp_of(x_target, s, log_sum, scale);
        if (ENT) entropy = log_sum - CUDART_LN2_F * (s.wsum / s.sum);
        if (!inside && t == 0) record_bad_target(a.status, row);
    }
    if (t == 0 && rank == 0) {
        a.logp[row] = logp;
        if (a.lse) a.lse[row] = lse;
        if (ENT) a.entropy[row] = entropy;
    }
}

// ---- policy loss: parts shared by its forms ---------------------------------------------------

// What a row brings beside its logits.
struct RowIn {
    int64_t target;
    float weight, old, adv, ref;

    __device__ __forceinline__ bool live() const { return weight != 0.f && target >= 0; }
};
__device__ __forceinline__ RowIn row_in(const PolicyArgs &a, int64_t row) {
    RowIn r;
    r.target = a.targets[row];
    r.weight = a.weights[row];
    r.old = a.old_logp[row];
    r.adv = a.advantages[row];
    r.ref = a.ref_logp ? a.ref_logp[row] : 0.f;
    return r;
}

// Whether a row is read at all, in two steps: what decides it can be loaded ahead.
struct PolicyMask {
    float weight = 0.f;
    int64_t target = -1;

    __device__ __forceinline__ bool live() const { return weight != 0.f && target >= 0; }
};
__device__ __forceinline__ PolicyMask row_mask(const PolicyArgs &a, int64_t row) {
    PolicyMask m;
    m.weight = a.weights[row];
    m.target = a.targets[row];
    return m;
}
struct DistillMask {
    float weight = 0.f;

    __device__ __forceinline__ bool live() const { return weight != 0.f; }
};
__device__ __forceinline__ DistillMask row_mask(const DistillArgs &a, int64_t row) { return {a.weights[row]}; }

// The same of a distilled row, as the kernels for any loss see it: no target, but the teacher's mass.
struct DistillIn {
    int64_t target = -1;
    float weight = 0.f, mass = 0.f;

    __device__ __forceinline__ bool live() const { return weight != 0.f; }
};
__device__ __forceinline__ DistillIn row_in(const DistillArgs &a, int64_t row) { return {-1, a.weights[row], a.masses[row].x}; }

template <typename Args>
constexpr bool kDistill = std::is_same<Args, DistillArgs>::value;

// exp(d) - d - 1, and exp(d) - 1.  Policies that are close have d of 1e-5 to 1e-2 and a KL of d^2/2: the
// difference of exp(d) and d + 1 would leave noise of 6e-8 there.  Below 1/2 the exponential series without its
// first two terms is summed instead (the first one left out is 2e-8 of the sum); from 1/2 on the
// difference costs 1.2e-6 at most.
__device__ __forceinline__ float kl_of(float d, float &less_one) {
    if (fabsf(d) < 0.5f) {
        float q = 1.f / 40320.f;
        q = fmaf(q, d, 1.f / 5040.f);
        q = fmaf(q, d, 1.f / 720.f);
        q = fmaf(q, d, 1.f / 120.f);
        q = fmaf(q, d, 1.f / 24.f);
        q = fmaf(q, d, 1.f / 6.f);
        q = fmaf(q, d, 0.5f);
        const float kl = d * d * q;
        less_one = d + kl;
        return kl;
    }
    less_one = expf(d) - 1.f;
    return less_one - d;
}

// One row's loss terms and its gradient: dlogits_j = unit*[j = target] + per_e*2^(k*(x_j - top)).
struct RowOut {
    float logp, pg, kl, cut, unit, per_e;
};
__device__ __forceinline__ RowOut row_out(const PolicyArgs &a, const RowIn &in, const Stats &s, float x_target) {
    RowOut o;
    o.logp = logp_of(x_target, s, logf(s.sum), a.scale);
    const float r = expf(o.logp - in.old);
    // no advantage, no loss, also where the ratio overflows (a NaN ratio is seen to below)
    const float plain = in.adv == 0.f ? 0.f : r * in.adv;
    const float clipped = in.adv == 0.f ? 0.f : fminf(fmaxf(r, a.ratio_min), a.ratio_max) * in.adv;
    const bool cut = plain > clipped;
    o.pg = -(cut ? clipped : plain);
    o.cut = cut ? 1.f : 0.f;
    float slope = cut ? 0.f : -plain;
    o.kl = 0.f;
    if (a.ref_logp) {
        float less_one;  // exp(d) - 1
        o.kl = kl_of(in.ref - o.logp, less_one);
        if (a.kl_coef != 0.f) slope -= a.kl_coef * less_one;  // a KL that is only watched may be infinite
    }
    if (r != r) o.pg = slope = r;  // a NaN log-probability stays visible
    o.unit = in.weight * slope * a.scale;
    o.per_e = __fdividef(-o.unit, s.sum);  // 2 ulp; sum >= 1 or NaN
    return o;
}

__device__ __forceinline__ RowOut row_out(const DistillArgs &a, const DistillIn &in, const Stats &s, float) {
    return {0.f, 0.f, 0.f, 0.f, 0.f, per_e_of(a, in.mass, in.weight, s.sum)};
}

__device__ __forceinline__ void add_terms(Sums &sums, const PolicyArgs &a, const RowIn &in, const RowOut &o) {
    sums.add(in.weight, o.pg + (a.ref_logp && a.kl_coef != 0.f ? a.kl_coef * o.kl : 0.f), o.pg, o.kl, o.cut);
}

// The leaders' sums -> the CTA's in the workspace -> stats, by the last CTA, in the CTAs' order.  All
// THREADS call it; thread LEADER*i holds the sums of leader i.  CTA `index` of `count` that have sums.
template <int THREADS, int LEADER, typename Args>
__device__ __forceinline__ void finish_stats(const Args &a, const Sums &s, double (*slots)[4], volatile int *last,
                                             int t, unsigned index, unsigned count) {
    static_assert(THREADS / 32 <= kWarps, "slots");
    constexpr int kLeaders = THREADS / LEADER;
    Workspace *ws = static_cast<Workspace *>(a.workspace);
    const auto sync = []() { asm volatile("bar.sync 0, %0;" ::"n"(THREADS) : "memory"); };
    if (t % LEADER == 0)
        for (int i = 0; i < 4; ++i) slots[t / LEADER][i] = s.v[i];
    if (kLeaders > 1) sync();
    else __syncwarp();
    double sum = 0.0;
    if (t < 4) {
        for (int w = 0; w < kLeaders; ++w) sum += slots[w][t];
        if (count == 1) a.stats[t] = (float)sum;
    }
    if (count == 1) return;
    if (t < 32) {
        if (t < 4) ws->part[4 * index + t] = sum;
        __syncwarp();
        if (t == 0) {  // this thread's fences cover the warp's stores before and, past the barrier, the CTA's loads behind
            __threadfence();
            const bool mine = atomicAdd(&ws->ticket, 1u) == count - 1;
            if (mine) __threadfence();
            *last = mine;
        }
    }
    sync();
    if (!*last) return;
    sum = 0.0;  // threads of one remainder mod 4 add up the same of the four sums
    for (unsigned i = t; i < 4 * count; i += THREADS) sum += __ldcg(&ws->part[i]);
    for (int o = 16; o >= 4; o >>= 1) sum += __shfl_down_sync(0xffffffffu, sum, o);
    if (t % 32 < 4) slots[t / 32][t % 32] = sum;
    sync();
    if (t < 4) {
        sum = 0.0;
        for (int w = 0; w < THREADS / 32; ++w) sum += slots[w][t];
        a.stats[t] = (float)sum;
    }
    if (t == 0) ws->ticket = 0;
}

// ---- rows that fit a warp's registers -----------------------------------------------------------

// One row at a time to a warp, 32 warps to an SM hide its latencies: 100000 x 2000 bf16 144 us (75 % of a
// copy's rate), 333333 x 600 246 us (44 %).  What holds these back is no floor: all 32 lanes compute the row's
// loss terms (a logarithm, two exponentials, a division) once per row, and a lane's eight units leave 64
// registers too few (72 to 104 bytes spilled).
template <typename T, typename O>
__global__ void __launch_bounds__(kThreads, 2)
policy_loss_rows_kernel(const PolicyArgs a, float k) {
    __shared__ double sums[kWarps][4];
    __shared__ int last;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    Sums acc;
    for (int64_t row = (int64_t)blockIdx.x * kWarps + warp; row < a.rows; row += (int64_t)gridDim.x * kWarps) {
        const RowIn in = row_in(a, row);
        O *y = static_cast<O *>(a.dlogits) + row * a.ld_dlogits;
        if (!in.live()) {
            if (lane == 0 && a.logp) a.logp[row] = 0.f;
            if (a.dlogits) fill_zeros(y, a.vocab, lane, 32);
            continue;
        }
        const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
        const RowShape shape = row_shape(x, (int)a.vocab);
        const uint4 *body = reinterpret_cast<const uint4 *>(x + shape.head);
        const bool has_extra = lane < shape.head + shape.tail, inside = in.target < a.vocab;
        const int extra = has_extra ? extra_index<T>(shape, lane) : 0;
        const float x_target = inside ? widen(x[in.target]) : CUDART_NAN_F;
        uint4 u[kRowUnits];
#pragma unroll
        for (int i = 0; i < kRowUnits; ++i)
            if (lane + 32 * i < shape.units) u[i] = ld_unit(body + lane + 32 * i);
        const float x_extra = has_extra ? widen(x[extra]) : 0.f;
        Running<false> run;
#pragma unroll
        for (int i = 0; i < kRowUnits; ++i) {
            if (lane + 32 * i < shape.units) {
                const uint4 one[1] = {u[i]};
                run.template add_units<T>(one, k);
            }
        }
        if (has_extra) run.add_one(x_extra, k);
        const Stats s = warp_join<false>(run.stats(), k);
        __syncwarp();  // the gradient may replace the logits: no lane writes before all have read (a join alone orders no memory)
        const RowOut o = row_out(a, in, s, x_target);
        if (lane == 0) {
            add_terms(acc, a, in, o);
            if (!inside) record_bad_target(a.status, row);
            if (a.logp) a.logp[row] = o.logp;
        }
        if (!a.dlogits) continue;
        const RowWriter<T, O> out(y, shape, s.top, o.unit, o.per_e, k);
        O *p = y + shape.head + lane * kUnit<T>;
        if (out.shift == 0) {
#pragma unroll
            for (int i = 0; i < kRowUnits; ++i)
                if (lane + 32 * i < shape.units) out.put(u[i], p + 32 * i * kUnit<T>);
        } else {
#pragma unroll
            for (int i = 0; i < kRowUnits; ++i) {
                const int at = lane + 32 * i;
                if (at < shape.units)
                    out.put_shifted(u[i], ld_unit(body + (at + 1 < shape.units ? at + 1 : at)), p + 32 * i * kUnit<T>, at == 0,
                                    at + 1 == shape.units);
            }
        }
        if (has_extra) y[extra] = out.value(x_extra, extra == in.target);
        if (inside && lane == out.writer_of(shape, in.target, 0, shape.units, 32)) y[in.target] = out.value(x_target, true);
    }
    finish_stats<kThreads, 32>(a, acc, sums, &last, threadIdx.x, blockIdx.x, gridDim.x);
}

// The same for distillation: the warp's lanes hold the entries, too.  100000 x 2000 bf16 from 64 entries 231 us (50 % of a copy's
// rate), 333333 x 600 from 20 entries 387 (30 %): a warp does a row's loads, two exchanges, teacher's side, loss terms and
// stores one after the other, and 64 registers to a thread are too few here as well (128 to 152 bytes spilled).
template <typename T, typename O>
__global__ void __launch_bounds__(kThreads, 2)
distill_rows_kernel(const DistillArgs a, float k) {
    __shared__ double sums[kWarps][4];
    __shared__ int last;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    Sums acc;
    for (int64_t row = (int64_t)blockIdx.x * kWarps + warp; row < a.rows; row += (int64_t)gridDim.x * kWarps) {
        const float weight = a.weights[row];
        O *y = static_cast<O *>(a.dlogits) + row * a.ld_dlogits;
        if (weight == 0.f) {
            if (lane == 0 && a.loss) a.loss[row] = 0.f;
            if (a.dlogits) fill_zeros(y, a.vocab, lane, 32);
            continue;
        }
        const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
        const RowShape shape = row_shape(x, (int)a.vocab);
        const uint4 *body = reinterpret_cast<const uint4 *>(x + shape.head);
        const bool has_extra = lane < shape.head + shape.tail;
        const int extra = has_extra ? extra_index<T>(shape, lane) : 0;
        RawEntries raw = {};
        load_entries(a, row, lane, raw);
        uint4 u[kRowUnits];
#pragma unroll
        for (int i = 0; i < kRowUnits; ++i)
            if (lane + 32 * i < shape.units) u[i] = ld_unit(body + lane + 32 * i);
        const float x_extra = has_extra ? widen(x[extra]) : 0.f;
        Entries en = entries_of(a, raw, a.teacher_lse ? a.teacher_lse[row] : 0.f, lane);
        float x_at[kTopEach];
#pragma unroll
        for (int e = 0; e < kTopEach; ++e) x_at[e] = in_use(a, e) ? widen(x[max(en.id[e], 0)]) : 0.f;
        if (any_twice(a, en)) join_twice(en.id, en.p, en.own);
        Running<false> run;
#pragma unroll
        for (int i = 0; i < kRowUnits; ++i) {
            if (lane + 32 * i < shape.units) {
                const uint4 one[1] = {u[i]};
                run.template add_units<T>(one, k);
            }
        }
        if (has_extra) run.add_one(x_extra, k);
        const Stats s = warp_join<false>(run.stats(), k);
        const float per_e = per_e_of(a, en.mass, weight, s.sum), log_sum = logf(s.sum), inv = 1.f / s.sum;
        float kl = en.inner, cross = 0.f, held = 0.f, g[kTopEach];
#pragma unroll
        for (int e = 0; e < kTopEach; ++e)
            if (in_use(a, e) && en.id[e] >= 0) {
                const EntryTerms o = entry_terms(x_at[e], en.p[e], en.own[e], en.mass, a.scale, weight * a.scale, s.top, log_sum, inv, k);
                cross += o.cross;
                held += o.held;
                g[e] = o.g;
            }
        kl += cross;
        if (en.bad) kl = cross = held = CUDART_NAN_F;
        __syncwarp();  // the gradient may replace the logits: no lane writes before all have read
        acc.add(weight, kl, cross, held, lane == 0 ? en.mass : 0.f);
        if (a.loss) {
            kl = warp_sum(kl);
            if (lane == 0) a.loss[row] = kl;
        }
        if (lane == 0 && en.bad) record_bad_target(a.status, row);
        if (!a.dlogits) continue;
        if (per_e == 0.f) {
            fill_zeros(y, a.vocab, lane, 32);
        } else {
            const RowWriter<T, O> out(y, shape, s.top, 0.f, per_e, k);
            O *p = y + shape.head + lane * kUnit<T>;
            if (out.shift == 0) {
#pragma unroll
                for (int i = 0; i < kRowUnits; ++i)
                    if (lane + 32 * i < shape.units) out.put(u[i], p + 32 * i * kUnit<T>);
            } else {
#pragma unroll
                for (int i = 0; i < kRowUnits; ++i) {
                    const int at = lane + 32 * i;
                    if (at < shape.units)
                        out.put_shifted(u[i], ld_unit(body + (at + 1 < shape.units ? at + 1 : at)), p + 32 * i * kUnit<T>, at == 0,
                                        at + 1 == shape.units);
                }
            }
            if (has_extra) y[extra] = out.value(x_extra, false);
        }
        __syncwarp();  // the entries' elements are written over
#pragma unroll
        for (int e = 0; e < kTopEach; ++e)
            if (in_use(a, e) && en.id[e] >= 0) y[en.id[e]] = narrow<O>(g[e]);
    }
    sum_lanes(acc);
    finish_stats<kThreads, 32>(a, acc, sums, &last, threadIdx.x, blockIdx.x, gridDim.x);
}

// ---- longer rows: a ring in shared memory ------------------------------------------------------
// A row, or its slice where a cluster of CTAs shares one, is brought to shared memory by bulk copies,
// in stages; the statistics are taken from the stages as they arrive, then the gradient is computed
// from the same stages, each of which is refilled as soon as it has been used: every logit crosses the
// HBM bus once.  The warps that compute take row i+1's statistics BEFORE they write row i's gradient:
// between a row's statistics and its gradient lie the joins over warps and CTAs and the loss itself,
// which one warp of its own does meanwhile, and nobody waits for them.  The ring therefore holds two
// rows (slices).  One more warp issues the copies.

template <typename T, typename O, typename Cut, typename Args>
__global__ void __launch_bounds__(Cut::kThreads, Cut::kPerSm)
policy_loss_ring_kernel(const Args a, float k, int log_cluster) {
    constexpr int kStages = Cut::kStages, kStageUnits = Cut::kStageUnits, kRingWork = Cut::kWork, kEach = Cut::kEach;
    extern __shared__ unsigned char raw[];
    RingShared<Cut> &sh = *reinterpret_cast<RingShared<Cut> *>((reinterpret_cast<uintptr_t>(raw) + 127) & ~(uintptr_t)127);
    const int t = threadIdx.x, lane = t % 32, warp = t / 32;
    const int cluster = 1 << log_cluster;
    const int rank = cluster > 1 ? (int)cluster_rank() : 0;
    const int64_t first = blockIdx.x >> log_cluster, step = gridDim.x >> log_cluster;
    if (t == 0) {
        for (int i = 0; i < kStages; ++i) {
            barrier_init(shared_addr(&sh.full[i]), 1);
            barrier_init(shared_addr(&sh.empty[i]), Cut::kWarps);
        }
        for (int i = 0; i < 2; ++i) {
            barrier_init(shared_addr(&sh.joined[i]), Cut::kWarps);
            barrier_init(shared_addr(&sh.peered[i]), 1);
            barrier_init(shared_addr(&sh.ready[i]), 1);
        }
        sh.give_up = 0;
        barrier_init_fence();
    }
    __syncthreads();
    if (cluster > 1) cluster_sync();  // the peers' barriers are ready before the first message

    if (warp == Cut::kProducerWarp) {
        if (lane == 0) {
            Cursor<kStages> c;
            uint32_t issued = 0;  // stages, up to kStages
            for (int64_t row = first; row < a.rows && !*(volatile int *)&sh.give_up; row += step) {
                if (!row_mask(a, row).live()) continue;
                const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
                const RowShape shape = row_shape(x, (int)a.vocab);
                int from, count;
                slice_of(shape.units, rank, log_cluster, from, count);
                const unsigned char *src = reinterpret_cast<const unsigned char *>(x + shape.head) + (size_t)from * 16;
                for (int at = 0; at < count; at += kStageUnits, c.advance()) {
                    const uint32_t full = shared_addr(&sh.full[c.slot]);
                    // used before: wait until that use, of the other parity, is over
                    if (issued == kStages && !barrier_wait(shared_addr(&sh.empty[c.slot]), c.parity ^ 1, &sh.give_up)) break;
                    const uint32_t bytes = 16u * (uint32_t)(count - at < kStageUnits ? count - at : kStageUnits);
                    barrier_expect(full, bytes);
                    bulk_load(shared_addr(sh.stage[c.slot]), src + (size_t)at * 16, bytes, full);
                    if (issued < kStages) ++issued;
                }
            }
            if (*(volatile int *)&sh.give_up) {  // copies in flight end before the CTA does
                int none = 0;
                for (uint32_t i = 0; i < issued; ++i) {  // backwards from the last one issued
                    if (c.slot == 0) c.parity ^= 1;
                    c.slot = c.slot ? c.slot - 1 : kStages - 1;
                    barrier_wait(shared_addr(&sh.full[c.slot]), c.parity, &none);
                }
                report_expired_wait(&sh.give_up, a.status, kWaitPolicyRing);
            }
        }
    } else if (warp == Cut::kScalarWarp) {
        if constexpr (kDistill<Args>) {
            let_next_start();
            wait_for_previous();  // for the teacher's masses; the others need nothing that was not there before that kernel
        }
        Sums acc;
        uint32_t n = 0;  // live rows
        decltype(row_in(a, first)) next = {};
        if (first < a.rows) next = row_in(a, first);
        for (int64_t row = first; row < a.rows; row += step) {
            const auto in = next;
            if (row + step < a.rows) next = row_in(a, row + step);
            if (!in.live()) {
                if constexpr (!kDistill<Args>) {
                    if (lane == 0 && rank == 0 && a.logp) a.logp[row] = 0.f;
                }
                continue;
            }
            const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
            const RowShape shape = row_shape(x, (int)a.vocab);
            int from, count;
            slice_of(shape.units, rank, log_cluster, from, count);
            const int b = n & 1;
            const uint32_t parity = n >> 1 & 1;
            const bool inside = !kDistill<Args> && in.target < a.vocab, has_extra = rank == 0 && lane < shape.head + shape.tail;
            const int extra = has_extra ? extra_index<T>(shape, lane) : 0;
            // the gradient may replace the logits: what is read here travels with this CTA's message,
            // before which nobody writes
            float x_target = rank == 0 && inside ? widen(x[in.target]) : CUDART_NAN_F;
            const float x_extra = has_extra ? widen(x[extra]) : -CUDART_INF_F;
            Running<false> run;
            run.add_one(x_extra, k);
            barrier_wait(shared_addr(&sh.joined[b]), parity, &sh.give_up);
            const Stats none = {-CUDART_INF_F, 0.f, 0.f};
            Stats s = none;
            if (lane < Cut::kWarps) s = {sh.slots[b][lane].x, sh.slots[b][lane].y, 0.f};
            s = warp_join<false>(join2(s, run.stats(), k), k);
            if (cluster > 1) {
                const uint32_t bar = shared_addr(&sh.peered[b]);
                if (lane == 0) barrier_expect(bar, 16u * cluster);
                if (lane < cluster) send16(shared_addr(&sh.peer[b][rank]), bar, lane, s.top, s.sum, x_target, 0.f);
                barrier_wait(bar, parity, &sh.give_up);
                float4 q = make_float4(-CUDART_INF_F, 0.f, 0.f, 0.f);
                if (lane < cluster) q = sh.peer[b][lane];
                x_target = __shfl_sync(0xffffffffu, q.z, 0);
                s = warp_join<false>({q.x, q.y, 0.f}, k);
            }
            const RowOut o = row_out(a, in, s, x_target);
            O *y = static_cast<O *>(a.dlogits) + row * a.ld_dlogits;
            const RowWriter<T, O> out(y, shape, s.top, o.unit, o.per_e, k);
            __syncwarp();  // all lanes have read x_target, which the verdict's readers may overwrite
            if (lane == 0) {
                const int writer = inside ? out.writer_of(shape, in.target, from, count, kRingWork) : -1;
                sh.verdict[b] = {s.top, o.unit, o.per_e, x_target, in.target, writer};
                barrier_arrive(shared_addr(&sh.ready[b]));
                if constexpr (kDistill<Args>) {
                    if (rank == 0) a.row_stats[row] = make_float2(s.top, s.sum);
                } else if (rank == 0) {
                    add_terms(acc, a, in, o);
                    if (a.logp) a.logp[row] = o.logp;
                    if (!inside) record_bad_target(a.status, row);
                }
            }
            if (has_extra && a.dlogits) {
                if (kDistill<Args> && o.per_e == 0.f) y[extra] = narrow<O>(0.f);
                else y[extra] = out.value(x_extra, extra == in.target);
            }
            ++n;
        }
        if (lane == 0) report_expired_wait(&sh.give_up, a.status, kWaitPolicyRing);
        __syncwarp();
        if constexpr (!kDistill<Args>) {
            if (rank == 0) finish_stats<32, 32>(a, acc, sh.sums, &sh.last, lane, (unsigned)first, (unsigned)step);
        }
    } else {
        Cursor<kStages> c;
        uint32_t n = 0;              // live rows whose statistics have been taken
        int64_t due = -1;            // the row whose gradient is to be written next
        Cursor<kStages> due_at;
        RowShape shape = {0, 0, 0};  // the due row's, and its slice
        int from = 0, count = 0;
        const auto write_due = [&]() {
            const int b = (n - 1) & 1;
            const bool ok = barrier_wait(shared_addr(&sh.ready[b]), (n - 1) >> 1 & 1, &sh.give_up);
            const Verdict q = sh.verdict[b];
            O *y = static_cast<O *>(a.dlogits) + due * a.ld_dlogits;
            const RowWriter<T, O> out(y, shape, q.top, q.unit, q.per_e, k);
            Cursor<kStages> at_stage = due_at;
            const unsigned zero = (unsigned)log_cluster >> 8;  // which the compiler does not know
            // A stage is given back when it has been read, not when its loads have been issued: a load that is still on its way
            // when the arrival is seen would find the stage filled anew.  So it is given back behind the stores of what was
            // read, or as soon as that has come, by an arrival whose address depends on it: a vote, since one lane arrives
            // for all of the warp, and lanes may run apart.  (4096 x 50257 bf16 distilled: 151 us so, 157 behind the stores.)
            // A stage is given back when it has been read, not when its loads have been issued: a load that is still on its way
            // when the arrival is seen would find the stage filled anew.  So it is given back behind the stores of what was
            // read, or as soon as that has come, by an arrival whose address depends on it.  One lane arrives for its warp, and
            // lanes may run apart, so it is a vote of all lanes that the address depends on.  (8192 x 50257 bf16: 252 us, 261
            // behind the stores; 252 with the arriving lane's own words alone.)
            const auto release = [&](unsigned nothing = 0u) {
                __syncwarp();
                if (lane == 0) barrier_arrive(shared_addr(&sh.empty[at_stage.slot]) + nothing);
            };
            const auto once_read = [&](unsigned read) { return (unsigned)__any_sync(0xffffffffu, (read & zero) != 0u); };  // 0
            O *p = y + shape.head + (int64_t)(from + t) * kUnit<T>;
            bool skip = !a.dlogits || !ok;
            if constexpr (kDistill<Args>) {
                if (!skip && q.per_e == 0.f) {  // a row without entries, whatever its logits
                    fill_zeros(y + shape.head + (int64_t)from * kUnit<T>, (int64_t)count * kUnit<T>, t, kRingWork);
                    skip = true;
                }
            }
            if (skip) {
                for (int at = 0; at < count; at += kStageUnits, at_stage.advance()) release();
                return;
            }
            if (out.shift == 0) {
                int at = 0;
                for (; count - at >= 2 * kStageUnits; at += 2 * kStageUnits, p += 2 * kStageUnits * kUnit<T>) {
                    uint4 u[2 * kEach];
                    Cursor<kStages> second = at_stage;
                    second.advance();
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint4 *units = reinterpret_cast<const uint4 *>(sh.stage[j ? second.slot : at_stage.slot]) + t;
#pragma unroll
                        for (int i = 0; i < kEach; ++i) u[j * kEach + i] = units[i * kRingWork];
                    }
                    unsigned read = 0;
#pragma unroll
                    for (int i = 0; i < 2 * kEach; ++i) read ^= u[i].x;
                    const unsigned nothing = once_read(read);
                    release(nothing);
                    at_stage.advance();
                    release(nothing);
                    at_stage.advance();
#pragma unroll
                    for (int i = 0; i < 2 * kEach; ++i) out.put(u[i], p + i * kRingWork * kUnit<T>);
                }
                for (; at < count; at += kStageUnits, at_stage.advance(), p += kStageUnits * kUnit<T>) {
                    const uint4 *units = reinterpret_cast<const uint4 *>(sh.stage[at_stage.slot]) + t;
                    if (count - at >= kStageUnits) {
                        uint4 u[kEach];
                        unsigned read = 0;
#pragma unroll
                        for (int i = 0; i < kEach; ++i) u[i] = units[i * kRingWork];
#pragma unroll
                        for (int i = 0; i < kEach; ++i) read ^= u[i].x;
                        const unsigned nothing = once_read(read);
                        release(nothing);
#pragma unroll
                        for (int i = 0; i < kEach; ++i) out.put(u[i], p + i * kRingWork * kUnit<T>);
                    } else {
#pragma unroll 1
                        for (int i = 0; i < count - at - t; i += kRingWork) out.put(units[i], p + i * kUnit<T>);
                        release();
                    }
                }
            } else {
                for (int at = 0; at < count; at += kStageUnits, p += kStageUnits * kUnit<T>) {
                    const uint4 *units = reinterpret_cast<const uint4 *>(sh.stage[at_stage.slot]);
                    const int slot = at_stage.slot + 1 == kStages ? 0 : at_stage.slot + 1;
                    // the row's next stage: nobody releases it before this one
                    const uint4 *after = reinterpret_cast<const uint4 *>(sh.stage[slot]);
#pragma unroll 1
                    for (int i = t; i < kStageUnits && at + i < count; i += kRingWork) {
                        const bool last = at + i + 1 == count;
                        const uint4 *next = i + 1 < kStageUnits ? units + i + 1 : after;
                        out.put_shifted(units[i], last ? units[i] : *next, p + (i - t) * kUnit<T>, at + i == 0, last);
                    }
                    release();
                    at_stage.advance();
                }
            }
            if (t == q.writer) y[q.target] = out.value(q.x_target, true);
        };
        decltype(row_mask(a, first)) next;
        if (first < a.rows) next = row_mask(a, first);
        for (int64_t row = first; row < a.rows; row += step) {
            const bool live = next.live();
            if (row + step < a.rows) next = row_mask(a, row + step);
            const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
            const RowShape new_shape = row_shape(x, (int)a.vocab);
            int new_from, new_count;
            slice_of(new_shape.units, rank, log_cluster, new_from, new_count);
            if (!live) {
                if (a.dlogits) {  // the first CTA's part has the row's head, the last one's its tail
                    const int64_t begin = rank == 0 ? 0 : new_shape.head + (int64_t)new_from * kUnit<T>;
                    const int64_t end =
                        rank == cluster - 1 ? a.vocab : new_shape.head + (int64_t)(new_from + new_count) * kUnit<T>;
                    fill_zeros(static_cast<O *>(a.dlogits) + row * a.ld_dlogits + begin, end - begin, t, kRingWork);
                }
                continue;
            }
            const Cursor<kStages> begin = c;
            Running<false> run;
            int at = 0;
            for (; new_count - at >= 2 * kStageUnits; at += 2 * kStageUnits) {
                uint4 u[2 * kEach];
#pragma unroll
                for (int j = 0; j < 2; ++j, c.advance()) {
                    barrier_wait(shared_addr(&sh.full[c.slot]), c.parity, &sh.give_up);
                    const uint4 *units = reinterpret_cast<const uint4 *>(sh.stage[c.slot]) + t;
#pragma unroll
                    for (int i = 0; i < kEach; ++i) u[j * kEach + i] = units[i * kRingWork];
                }
                run.template add_units<T>(u, k);
            }
            for (; at < new_count; at += kStageUnits, c.advance()) {
                barrier_wait(shared_addr(&sh.full[c.slot]), c.parity, &sh.give_up);
                const int here = new_count - at;
                const uint4 *units = reinterpret_cast<const uint4 *>(sh.stage[c.slot]) + t;
                if (here <= kRingWork) {
                    if (t < here) {
                        const uint4 u[1] = {units[0]};
                        run.template add_units<T>(u, k);
                    }
                } else if (t < here) {
                    uint4 u[kEach];
#pragma unroll
                    for (int i = 0; i < kEach; ++i) u[i] = t + i * kRingWork < here ? units[i * kRingWork] : nothing<T>();
                    run.template add_units<T>(u, k);
                }
            }
            const Stats s = warp_join<false>(run.stats(), k);
            if (lane == 0) {
                sh.slots[n & 1][warp] = make_float2(s.top, s.sum);
                barrier_arrive(shared_addr(&sh.joined[n & 1]));
            }
            if (due >= 0) write_due();
            due = row;
            shape = new_shape;
            from = new_from;
            count = new_count;
            due_at = begin;
            ++n;
        }
        if (due >= 0) write_due();
        if (lane == 0) report_expired_wait(&sh.give_up, a.status, kWaitPolicyRing);
    }
    if (cluster > 1) {
        __syncwarp();
        cluster_sync();  // no CTA ends while a peer may still send to it
    }
}

// ---- rows that no cluster's shared memory holds: read twice --------------------------------------

template <typename T, typename O>
__global__ void __launch_bounds__(kThreads)
policy_loss_long_kernel(const PolicyArgs a, float k) {
    __shared__ Stats shared[kWarps];
    __shared__ double sums[kWarps][4];
    __shared__ int last;
    const int t = threadIdx.x;
    Sums acc;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const RowIn in = row_in(a, row);
        const bool live = in.live();
        const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
        const RowShape shape = row_shape(x, (int)a.vocab);
        const uint4 *body = reinterpret_cast<const uint4 *>(x + shape.head);
        const bool has_extra = t < shape.head + shape.tail;
        const int extra = has_extra ? extra_index<T>(shape, t) : 0;
        float x_extra = 0.f, x_target = CUDART_NAN_F, top = 0.f;
        RowOut o = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (live) {
            const bool inside = in.target < a.vocab;
            if (inside) x_target = widen(x[in.target]);
            if (has_extra) x_extra = widen(x[extra]);
            Running<false> run;
            for (int i = t; i < shape.units; i += kThreads) {
                const uint4 u[1] = {ld_unit(body + i)};
                run.template add_units<T>(u, k);
            }
            if (has_extra) run.add_one(x_extra, k);
            const Stats s = group_join<kWarps, false>(run.stats(), k, shared, 0);
            top = s.top;
            o = row_out(a, in, s, x_target);
            if (t == 0) {
                add_terms(acc, a, in, o);
                if (!inside) record_bad_target(a.status, row);
            }
        }
        if (t == 0 && a.logp) a.logp[row] = o.logp;
        if (a.dlogits) {
            O *y = static_cast<O *>(a.dlogits) + row * a.ld_dlogits;
            if (live) {
                const RowWriter<T, O> out(y, shape, top, o.unit, o.per_e, k);
                O *p = y + shape.head;
                if (out.shift == 0) {
                    for (int i = t; i < shape.units; i += kThreads) out.put(ld_unit(body + i), p + (int64_t)i * kUnit<T>);
                } else {
                    for (int i = t; i < shape.units; i += kThreads)
                        out.put_shifted(ld_unit(body + i), ld_unit(body + (i + 1 < shape.units ? i + 1 : i)),
                                        p + (int64_t)i * kUnit<T>, i == 0, i + 1 == shape.units);
                }
                if (has_extra) y[extra] = out.value(x_extra, extra == in.target);
                if (in.target < a.vocab && t == out.writer_of(shape, in.target, 0, shape.units, kThreads))
                    y[in.target] = out.value(x_target, true);
            } else {
                fill_zeros(y, a.vocab, t, kThreads);
            }
        }
        group_sync<kWarps>(0);  // the slots are used again
    }
    finish_stats<kThreads, kThreads>(a, acc, sums, &last, t, blockIdx.x, gridDim.x);
}

// The same for distillation.
template <typename T, typename O>
__global__ void __launch_bounds__(kThreads)
distill_long_kernel(const DistillArgs a, float k) {
    __shared__ Stats shared[kWarps];
    const int t = threadIdx.x;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const DistillIn in = row_in(a, row);
        const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
        O *y = static_cast<O *>(a.dlogits) + row * a.ld_dlogits;
        if (!in.live()) {
            if (a.dlogits) fill_zeros(y, a.vocab, t, kThreads);
            continue;
        }
        const RowShape shape = row_shape(x, (int)a.vocab);
        const uint4 *body = reinterpret_cast<const uint4 *>(x + shape.head);
        const bool has_extra = t < shape.head + shape.tail;
        const int extra = has_extra ? extra_index<T>(shape, t) : 0;
        const float x_extra = has_extra ? widen(x[extra]) : 0.f;
        Running<false> run;
        for (int i = t; i < shape.units; i += kThreads) {
            const uint4 u[1] = {ld_unit(body + i)};
            run.template add_units<T>(u, k);
        }
        if (has_extra) run.add_one(x_extra, k);
        const Stats s = group_join<kWarps, false>(run.stats(), k, shared, 0);
        const RowOut o = row_out(a, in, s, 0.f);
        if (t == 0) a.row_stats[row] = make_float2(s.top, s.sum);
        group_sync<kWarps>(0);  // the slots are used again
        if (!a.dlogits) continue;
        if (o.per_e == 0.f) {
            fill_zeros(y, a.vocab, t, kThreads);
            continue;
        }
        const RowWriter<T, O> out(y, shape, s.top, 0.f, o.per_e, k);
        O *p = y + shape.head;
        if (out.shift == 0) {
            for (int i = t; i < shape.units; i += kThreads) out.put(ld_unit(body + i), p + (int64_t)i * kUnit<T>);
        } else {
            for (int i = t; i < shape.units; i += kThreads)
                out.put_shifted(ld_unit(body + i), ld_unit(body + (i + 1 < shape.units ? i + 1 : i)),
                                p + (int64_t)i * kUnit<T>, i == 0, i + 1 == shape.units);
        }
        if (has_extra) y[extra] = out.value(x_extra, false);
    }
}

// ---- a distilled row's entries, before and after the row -----------------------------------------

constexpr int kEntryWarps = 8;  // a row to each at a time

template <typename T>
__global__ void __launch_bounds__(32 * kEntryWarps)
distill_teacher_kernel(const DistillArgs a) {
    let_next_start();
    const int lane = threadIdx.x % 32;
    const int64_t row = (int64_t)blockIdx.x * kEntryWarps + threadIdx.x / 32;
    if (row >= a.rows) return;
    RawEntries raw = {};
    load_entries(a, row, lane, raw);  // whether the row counts or not: its weight is not waited for
    const float lse = a.teacher_lse ? a.teacher_lse[row] : 0.f;
    if (a.weights[row] == 0.f) return;
    const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
    T x_at[kTopEach];
#pragma unroll
    for (int e = 0; e < kTopEach; ++e) {
        x_at[e] = narrow<T>(0.f);
        if (in_use(a, e)) x_at[e] = x[min(max(raw.id[e], (int64_t)0), a.vocab - 1)];  // (used where there is an entry)
    }
    Entries en = entries_of(a, raw, lse, lane);
    if (any_twice(a, en)) join_twice(en.id, en.p, en.own);
#pragma unroll
    for (int e = 0; e < kTopEach; ++e)
        if (32 * e + lane < a.top)
            a.entries[row * a.top + 32 * e + lane] = make_float4(widen(x_at[e]), en.p[e], en.own[e], __int_as_float(en.id[e]));
    const float inner = warp_sum(en.inner);
    if (lane == 0) {
        a.masses[row] = make_float2(en.mass, inner);
        if (en.bad) record_bad_target(a.status, row);
    }
}

template <typename O>
__global__ void __launch_bounds__(32 * kEntryWarps)
distill_entries_kernel(const DistillArgs a, float k) {
    __shared__ double sums[kEntryWarps][4];
    __shared__ int last;
    wait_for_previous();
    const int lane = threadIdx.x % 32;
    Sums acc;
    for (int64_t row = (int64_t)blockIdx.x * kEntryWarps + threadIdx.x / 32; row < a.rows; row += (int64_t)gridDim.x * kEntryWarps) {
        const float weight = a.weights[row];
        float4 q[kTopEach];  // (what a row without weight left there is not used)
#pragma unroll
        for (int e = 0; e < kTopEach; ++e)
            if (in_use(a, e)) q[e] = a.entries[row * a.top + min(32 * e + lane, a.top - 1)];
        const float2 of_row = a.row_stats[row], of_teacher = a.masses[row];
        if (weight == 0.f) {
            if (lane == 0 && a.loss) a.loss[row] = 0.f;
            continue;
        }
        const float log_sum = logf(of_row.y), inv = 1.f / of_row.y, mass = of_teacher.x;
        O *y = static_cast<O *>(a.dlogits) + row * a.ld_dlogits;
        float cross = 0.f, held = 0.f;
#pragma unroll
        for (int e = 0; e < kTopEach; ++e)
            if (32 * e + lane < a.top) {
                const int id = __float_as_int(q[e].w);
                if (id >= 0) {
                    const EntryTerms o = entry_terms(q[e].x, q[e].y, q[e].z, mass, a.scale, weight * a.scale, of_row.x, log_sum, inv, k);
                    cross += o.cross;
                    held += o.held;
                    if (a.dlogits) y[id] = narrow<O>(o.g);
                }
            }
        if (mass != mass) cross = held = mass;
        const float kl = cross + (lane == 0 ? of_teacher.y : 0.f);
        acc.add(weight, kl, cross, held, lane == 0 ? mass : 0.f);
        if (a.loss) {
            const float all = warp_sum(kl);
            if (lane == 0) a.loss[row] = all;
        }
    }
    sum_lanes(acc);
    finish_stats<32 * kEntryWarps, 32>(a, acc, sums, &last, threadIdx.x, blockIdx.x, gridDim.x);
}

// ---- launches --------------------------------------------------------------------------------------

constexpr double kLog2e = 1.4426950408889634074;

unsigned grid_of(int64_t work, int64_t cap) {
    if (cap > kWorkspaceParts / 4) cap = kWorkspaceParts / 4;
    return (unsigned)(work < 1 ? 1 : work < cap ? work : cap);
}

template <typename T, int W, int ROWS>
cudaError_t logprobs_groups(const LogprobArgs &a, float k, cudaStream_t stream) {
    const unsigned grid = (unsigned)((a.rows + ROWS - 1) / ROWS);
    if (a.entropy) token_logprobs_kernel<T, W, ROWS, true, false><<<grid, 32 * W * ROWS, 0, stream>>>(a, k, 0);
    else token_logprobs_kernel<T, W, ROWS, false, false><<<grid, 32 * W * ROWS, 0, stream>>>(a, k, 0);
    return cudaGetLastError();
}

// CTAs of W warps, one row to each, that fit an SM.  Asked for once per device.
template <typename T, int W, bool ENT>
cudaError_t logprobs_resident(int *out) {
    static std::atomic<int> known[64];
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    int m = device < 64 ? known[device].load() : 0;
    if (m == 0) {
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&m, token_logprobs_kernel<T, W, 1, ENT, false>, 32 * W, 0);
        if (e != cudaSuccess) return e;
        if (m < 1) m = 1;
        if (device < 64) known[device].store(m);
    }
    *out = m;
    return cudaSuccess;
}

int log2_of(int n) {
    int l = 0;
    while (1 << l < n) ++l;
    return l;
}

template <typename T>
cudaError_t logprobs_cluster(const LogprobArgs &a, float k, int cluster, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.rows * cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim = {(unsigned)cluster, 1, 1};
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return a.entropy ? cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, kWarps, 1, true, true>, a, k, log2_of(cluster))
                     : cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, kWarps, 1, false, true>, a, k, log2_of(cluster));
}

template <typename T>
cudaError_t logprobs(const LogprobArgs &a, int sm_count, cudaStream_t stream) {
    const float k = (float)(a.scale * kLog2e);
    const int64_t units = a.vocab / kUnit<T>;
    if (units <= 32 * kRowUnits) return logprobs_groups<T, 1, 4>(a, k, stream);
    // Warps to a row, us with 4 / 8 / 16.  Short rows: 592 x 9000 bf16 4.8 / 5.5 / 6.0, 74 of them 3.6 / 3.2 / 3.1.
    const int64_t per_sm = a.rows / sm_count;
    if (units <= 3 * kThreads)
        return per_sm < 1 ? logprobs_groups<T, 8, 1>(a, k, stream) : logprobs_groups<T, 4, 1>(a, k, stream);
    // Few long rows: a cluster of CTAs to each while there are fewer rows than SMs and work for their threads
    // (20 x 50257 bf16 4.5 with 8 CTAs, 5.4 with 1; 20 x 20000 3.9 and 3.6), then 16 warps (296 x 131072
    // fp32 50.7 / 31.3 / 24.9).
    if (per_sm < 3 && units > 6 * kThreads) {
        int cluster = 1;
        if (units >= 8 * kThreads)
            while (cluster < kMaxCluster && a.rows * cluster * 2 <= sm_count && units >= cluster * 2 * kThreads) cluster *= 2;
        return cluster > 1 ? logprobs_cluster<T>(a, k, cluster, stream) : logprobs_groups<T, kWarps, 1>(a, k, stream);
    }
    int resident4 = 0, resident8 = 0;
    cudaError_t e = a.entropy ? logprobs_resident<T, 4, true>(&resident4) : logprobs_resident<T, 4, false>(&resident4);
    if (e == cudaSuccess) e = a.entropy ? logprobs_resident<T, 8, true>(&resident8) : logprobs_resident<T, 8, false>(&resident8);
    if (e != cudaSuccess) return e;
    return warps_to_a_row(a.rows, sm_count, resident4, resident8) == 8 ? logprobs_groups<T, 8, 1>(a, k, stream)
                                                                       : logprobs_groups<T, 4, 1>(a, k, stream);
}

template <typename T, typename O>
void launch_rows(const PolicyArgs &a, float k, unsigned grid, cudaStream_t stream) {
    policy_loss_rows_kernel<T, O><<<grid, kThreads, 0, stream>>>(a, k);
}
template <typename T, typename O>
void launch_rows(const DistillArgs &a, float k, unsigned grid, cudaStream_t stream) {
    distill_rows_kernel<T, O><<<grid, kThreads, 0, stream>>>(a, k);
}
template <typename T, typename O>
void launch_long(const PolicyArgs &a, float k, unsigned grid, cudaStream_t stream) {
    policy_loss_long_kernel<T, O><<<grid, kThreads, 0, stream>>>(a, k);
}
template <typename T, typename O>
void launch_long(const DistillArgs &a, float k, unsigned grid, cudaStream_t stream) {
    distill_long_kernel<T, O><<<grid, kThreads, 0, stream>>>(a, k);
}

template <typename T, typename O, typename Cut, typename Args>
struct RingLaunch {
    static constexpr int kBytes = (int)sizeof(RingShared<Cut>) + 128;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];

    RingLaunch(int cluster, int64_t clusters, cudaStream_t stream) {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim = {(unsigned)cluster, 1, 1};
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // distillation: behind its first kernel
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3((unsigned)(clusters * cluster));
        cfg.blockDim = dim3(Cut::kThreads);
        cfg.dynamicSmemBytes = kBytes;
        cfg.stream = stream;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
    RingLaunch(const RingLaunch &) = delete;  // cfg points at attr

    static cudaError_t prepare() {
        static std::atomic<unsigned long long> ready{0};
        return allow_shared(policy_loss_ring_kernel<T, O, Cut, Args>, kBytes, ready);
    }
    // Clusters that run at a time.  A GPC's SMs need not be a multiple of the cluster's (132 of 148 SMs
    // take part in clusters of 4, 120 in clusters of 8), and a cluster that waits for its turn would leave
    // its share of the rows to the end.  Asked for once per device.
    static cudaError_t resident(int cluster, int sm_count, int *out) {
        static std::atomic<int> known[64][4];
        const int most = kWorkspaceParts / 4;  // each CTA's sums have a place there
        *out = sm_count * Cut::kPerSm < most ? sm_count * Cut::kPerSm : most;
        if (cluster == 1) return cudaSuccess;
        int device = 0;
        cudaError_t e = cudaGetDevice(&device);
        if (e != cudaSuccess) return e;
        std::atomic<int> *slot = device < 64 ? &known[device][log2_of(cluster)] : nullptr;
        int m = slot ? slot->load() : 0;
        if (m == 0) {
            e = prepare();
            if (e != cudaSuccess) return e;
            RingLaunch l(cluster, sm_count * Cut::kPerSm / cluster, nullptr);
            e = cudaOccupancyMaxActiveClusters(&m, policy_loss_ring_kernel<T, O, Cut, Args>, &l.cfg);
            if (e != cudaSuccess) return e;
            if (m < 1) m = 1;
            if (slot) slot->store(m);
        }
        *out = m;
        return cudaSuccess;
    }
    static cudaError_t launch(const Args &a, float k, int cluster, int sm_count, cudaStream_t stream) {
        int most = 0;
        cudaError_t e = prepare();
        if (e == cudaSuccess) e = resident(cluster, sm_count, &most);
        if (e != cudaSuccess) return e;
        RingLaunch l(cluster, a.rows < 1 ? 1 : a.rows < most ? a.rows : most, stream);
        if (kDistill<Args> && a.rows > 0) l.cfg.numAttrs = 2;
        return cudaLaunchKernelEx(&l.cfg, policy_loss_ring_kernel<T, O, Cut, Args>, a, k, log2_of(cluster));
    }
};

// A loss and its gradient: the policy loss's arguments or the distillation's.
template <typename T, typename O, typename Args>
cudaError_t loss(const Args &a, int sm_count, cudaStream_t stream) {
    const float k = (float)(a.scale_exact * kLog2e);
    PolicyPlan plan;
    const int e = plan_policy(a.vocab / kUnit<T>, a.rows, sm_count, [&](PolicyForm form, int cluster, int *most) {
        return (int)(form == kForm640 ? RingLaunch<T, O, Cut640, Args>::resident(cluster, sm_count, most)
                                      : RingLaunch<T, O, Cut512, Args>::resident(cluster, sm_count, most));
    }, plan);
    if (e != 0) return (cudaError_t)e;
    switch (plan.form) {
        case kForm64: return RingLaunch<T, O, Cut64, Args>::launch(a, k, plan.cluster, sm_count, stream);
        case kForm128: return RingLaunch<T, O, Cut128, Args>::launch(a, k, plan.cluster, sm_count, stream);
        case kForm256: return RingLaunch<T, O, Cut256, Args>::launch(a, k, plan.cluster, sm_count, stream);
        case kForm512: return RingLaunch<T, O, Cut512, Args>::launch(a, k, plan.cluster, sm_count, stream);
        case kForm640: return RingLaunch<T, O, Cut640, Args>::launch(a, k, plan.cluster, sm_count, stream);
        case kFormRows: launch_rows<T, O>(a, k, grid_of((a.rows + kWarps - 1) / kWarps, (int64_t)sm_count * 2), stream); break;
        case kFormLong: launch_long<T, O>(a, k, grid_of(a.rows, (int64_t)sm_count * 4), stream); break;
    }
    return cudaGetLastError();
}

// Distillation: rows that a warp holds in one kernel, others in three.
template <typename T, typename O>
cudaError_t distill(const DistillArgs &a, int sm_count, cudaStream_t stream, int *launches) {
    const unsigned rows = (unsigned)((a.rows + kEntryWarps - 1) / kEntryWarps);
    const bool whole = a.vocab / kUnit<T> <= 32 * kRowUnits;
    if (!whole && a.rows > 0) distill_teacher_kernel<T><<<rows, 32 * kEntryWarps, 0, stream>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) e = loss<T, O>(a, sm_count, stream);
    if (e != cudaSuccess) return e;
    *launches += whole ? 1 : a.rows > 0 ? 3 : 2;
    if (!whole) {
        const unsigned grid = grid_of(rows, (int64_t)sm_count * 4);
        return launch_chained(distill_entries_kernel<O>, dim3(grid), dim3(32 * kEntryWarps), 0, stream, a, (float)(a.scale_exact * kLog2e));
    }
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_token_logprobs(const LogprobArgs &a, int sm_count, cudaStream_t stream) {
    return a.dtype == ADAMA_F32 ? logprobs<float>(a, sm_count, stream) : logprobs<__nv_bfloat16>(a, sm_count, stream);
}

cudaError_t launch_policy_loss(const PolicyArgs &a, int sm_count, cudaStream_t stream) {
    if (a.logits_dtype == ADAMA_F32)
        return a.dlogits_dtype == ADAMA_F32 ? loss<float, float>(a, sm_count, stream) : loss<float, __nv_bfloat16>(a, sm_count, stream);
    return a.dlogits_dtype == ADAMA_F32 ? loss<__nv_bfloat16, float>(a, sm_count, stream)
                                        : loss<__nv_bfloat16, __nv_bfloat16>(a, sm_count, stream);
}

size_t distill_scratch_bytes(int64_t rows, int top) { return (size_t)rows * (top * sizeof(float4) + 2 * sizeof(float2)); }

cudaError_t launch_distill_loss(DistillArgs a, void *scratch, int sm_count, cudaStream_t stream, int *launches) {
    a.entries = static_cast<float4 *>(scratch);
    a.masses = reinterpret_cast<float2 *>(a.entries + a.rows * a.top);
    a.row_stats = a.masses + a.rows;
    if (a.logits_dtype == ADAMA_F32)
        return a.dlogits_dtype == ADAMA_F32 ? distill<float, float>(a, sm_count, stream, launches)
                                            : distill<float, __nv_bfloat16>(a, sm_count, stream, launches);
    return a.dlogits_dtype == ADAMA_F32 ? distill<__nv_bfloat16, float>(a, sm_count, stream, launches)
                                        : distill<__nv_bfloat16, __nv_bfloat16>(a, sm_count, stream, launches);
}

}  // namespace adama
