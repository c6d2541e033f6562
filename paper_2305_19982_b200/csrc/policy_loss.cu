// Token log-probabilities and the clipped policy loss with its gradient, from rows of logits.
// With z = s*x (s = logit_scale) a row's lse = log sum_j exp(z_j), p_j = exp(z_j - lse),
// logp = z_target - lse, entropy = lse - sum_j p_j z_j.  For a row with weight w:
//     r = exp(logp - old),  pg = -min(r*A, clamp(r, 1-cl, 1+ch)*A),  d = ref - logp,
//     kl = exp(d) - d - 1,  loss += w*(pg + beta*kl)
//     dlogits_j = w*s*c*([j = target] - p_j),  c = -(r*A while r*A <= the clamped product) + beta*(1 - exp(d))
// A row is read once (loss: and its gradient written once); what bounds every form is HBM.
#include <type_traits>

#include "adama_device.cuh"
#include "bulk_copy.cuh"
#include "softmax_rows.cuh"
#include "tensor_table.cuh"

namespace adama {
namespace {

constexpr int kThreads = 512;  // that work on rows, in every kernel here
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ void record_bad_target(unsigned *status, int64_t row) {
    if (atomicCAS(status, (unsigned)kDevOk, (unsigned)kDevBadTarget) == (unsigned)kDevOk) {
        status[1] = (unsigned)row;
        status[2] = (unsigned)(row >> 32);
    }
}

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

__device__ __forceinline__ float logp_of(float x_target, const Stats &s, float log2sum, float k) {
    return CUDART_LN2_F * (k * (x_target - s.top) - log2sum);
}

constexpr int kMaxCluster = 8;  // CTAs that may share a row

// The slice of a row's units that CTA `rank` of 2^log_size takes (units < 2^29, so 32 bits hold it).
__device__ __forceinline__ void slice_of(int units, int rank, int log_size, int &from, int &count) {
    from = (int)(((unsigned)units * (unsigned)rank) >> log_size);
    count = (int)(((unsigned)units * (unsigned)(rank + 1)) >> log_size) - from;
}

__device__ __forceinline__ void store_peer(const Stats *slot, uint32_t rank, const Stats &s) {
    store12(shared_addr(slot), rank, s.top, s.sum, s.wsum);
}

// ---- token log-probabilities -----------------------------------------------------------------

// W warps to a row (or to the slice of a row that a cluster of CTAs shares), ROWS rows to a CTA, kLoads
// units of each thread in flight.
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
            cluster_sync();
            if (rank != 0) return;
            const Stats none = {-CUDART_INF_F, 0.f, 0.f};
            const int lane = t % 32;
            s = warp_join<ENT>(lane < 1 << log_cluster ? peers[lane] : none, k);
        }
        const float log2sum = log2f(s.sum);
        lse = fmaf(s.top, (float)a.scale, CUDART_LN2_F * log2sum);
        logp = logp_of(x_target, s, log2sum, k);
        if (ENT) entropy = CUDART_LN2_F * (log2sum - s.wsum / s.sum);
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

// One row's loss terms and its gradient: dlogits_j = unit*[j = target] + per_e*2^(k*(x_j - top)).
struct RowOut {
    float logp, pg, kl, cut, unit, per_e;
};
__device__ __forceinline__ RowOut row_out(const PolicyArgs &a, const RowIn &in, const Stats &s, float x_target, float k) {
    RowOut o;
    o.logp = logp_of(x_target, s, log2f(s.sum), k);
    const float r = expf(o.logp - in.old), plain = r * in.adv;
    const float clipped = fminf(fmaxf(r, a.ratio_min), a.ratio_max) * in.adv;
    const bool cut = plain > clipped;
    o.pg = -(cut ? clipped : plain);
    o.cut = cut ? 1.f : 0.f;
    float slope = cut ? 0.f : -plain;
    o.kl = 0.f;
    if (a.ref_logp) {
        const float d = in.ref - o.logp, e = expf(d);
        o.kl = e - d - 1.f;
        slope += a.kl_coef * (1.f - e);
    }
    if (r != r) o.pg = slope = r;  // a NaN log-probability stays visible
    o.unit = in.weight * slope * a.scale;
    o.per_e = __fdividef(-o.unit, s.sum);  // 2 ulp; sum >= 1 or NaN
    return o;
}

// Sums of one thread over its rows; in double, so that their order does not show in fp32.
struct Sums {
    double v[4] = {0.0, 0.0, 0.0, 0.0};

    __device__ __forceinline__ void add(const PolicyArgs &a, const RowIn &in, const RowOut &o) {
        const double w = in.weight;
        v[0] += w * (o.pg + (a.ref_logp ? a.kl_coef * o.kl : 0.f));
        v[1] += w * o.pg;
        v[2] += w * o.kl;
        v[3] += w * o.cut;
    }
};

// The leaders' sums -> the CTA's in the workspace -> stats, by the last CTA, in the CTAs' order.  All
// THREADS call it; thread LEADER*i holds the sums of leader i.
template <int THREADS, int LEADER>
__device__ __forceinline__ void finish_stats(const PolicyArgs &a, const Sums &s, double (*slots)[4], volatile int *last,
                                             int t) {
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
        if (gridDim.x == 1) a.stats[t] = (float)sum;
    }
    if (gridDim.x == 1) return;
    if (t < 32) {
        if (t < 4) {
            ws->part[4 * blockIdx.x + t] = sum;
            __threadfence();
        }
        __syncwarp();
        if (t == 0) *last = atomicAdd(&ws->ticket, 1u) == gridDim.x - 1;
    }
    sync();
    if (!*last) return;
    __threadfence();
    sum = 0.0;  // threads of one remainder mod 4 add up the same of the four sums
    for (unsigned i = t; i < 4 * gridDim.x; i += THREADS) sum += __ldcg(&ws->part[i]);
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

template <typename O>
__device__ __forceinline__ O narrow(float y);
template <>
__device__ __forceinline__ float narrow<float>(float y) { return y; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float y) { return __float2bfloat16_rn(y); }

__device__ __forceinline__ void store_wide(float *p, const float (&y)[4]) {
    st_stream(reinterpret_cast<float4 *>(p), make_float4(y[0], y[1], y[2], y[3]));
}
__device__ __forceinline__ void store_wide(float *p, const float (&y)[8]) {
    st_stream(reinterpret_cast<float4 *>(p), make_float4(y[0], y[1], y[2], y[3]));
    st_stream(reinterpret_cast<float4 *>(p) + 1, make_float4(y[4], y[5], y[6], y[7]));
}
__device__ __forceinline__ void store_wide(__nv_bfloat16 *p, const float (&y)[4]) {
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack2_bf16(y[0], y[1]), pack2_bf16(y[2], y[3]));
}
__device__ __forceinline__ void store_wide(__nv_bfloat16 *p, const float (&y)[8]) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack2_bf16(y[0], y[1]), pack2_bf16(y[2], y[3]),
                                               pack2_bf16(y[4], y[5]), pack2_bf16(y[6], y[7]));
}

// How a row's gradient is written.  The units are written without the target's extra term; the
// thread that wrote the target's element writes it again, with the term.
template <typename T, typename O>
struct RowWriter {
    static constexpr int N = kUnit<T>;
    O *y;
    bool wide;
    float top, unit, per_e, k;

    __device__ __forceinline__ RowWriter(O *row, const RowShape &shape, float top_, const RowOut &o, float k_)
        : y(row), top(top_), unit(o.unit), per_e(o.per_e), k(k_) {
        constexpr int align = N * sizeof(O) < 16 ? N * sizeof(O) : 16;
        wide = reinterpret_cast<uintptr_t>(row + shape.head) % align == 0;
    }
    template <bool WIDE>
    __device__ __forceinline__ static void store(O *p, const float (&v)[N]) {
        if (WIDE) {
            store_wide(p, v);
        } else {
#pragma unroll
            for (int q = 0; q < N; ++q) p[q] = narrow<O>(v[q]);
        }
    }
    // a unit of logits whose gradient goes to p
    template <bool WIDE>
    __device__ __forceinline__ void put(const uint4 &u, O *p) const {
        float v[N];
        const Pair minus = pair(-top, -top), k2 = pair(k, k), per = pair(per_e, per_e);
#pragma unroll
        for (int q = 0; q < N / 2; ++q) {
            float d0, d1;
            split(mul2(add2(unit_pair<T>(u, q), minus), k2), d0, d1);
            split(mul2(pair(exp2_fast(d0), exp2_fast(d1)), per), v[2 * q], v[2 * q + 1]);
        }
        store<WIDE>(p, v);
    }
    template <bool WIDE>
    __device__ __forceinline__ static void put_zeros(O *p) {
        float v[N];
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = 0.f;
        store<WIDE>(p, v);
    }
    __device__ __forceinline__ void put_one(float x, int j) const { y[j] = narrow<O>(per_e * exp2_fast(k * (x - top))); }
    __device__ __forceinline__ void put_target(float x, int64_t j) const {
        y[j] = narrow<O>(per_e * exp2_fast(k * (x - top)) + unit);
    }
};

// Thread of a group of `threads` that writes element j of a row: units go round the threads from the
// first unit of the slice on (stages hold a multiple of `threads` units), extra i belongs to thread i.
template <typename T>
__device__ __forceinline__ int owner_of(const RowShape &shape, int64_t j, int from, int threads) {
    const int at = (int)j - shape.head;
    if (at < 0) return (int)j;
    if (at >= shape.units * kUnit<T>) return shape.head + at - shape.units * kUnit<T>;
    return (at / kUnit<T> - from) % threads;
}

// ---- rows that fit a few warps' registers ------------------------------------------------------

constexpr int kRowUnits = 8;  // units of a thread

template <typename T, typename O, int W>
__global__ void __launch_bounds__(kThreads, 2)
policy_loss_rows_kernel(const PolicyArgs a, float k) {
    constexpr int kGroupThreads = 32 * W, kGroups = kWarps / W;
    __shared__ Stats shared[kWarps];
    __shared__ double sums[kWarps][4];
    __shared__ int last;
    const int g = threadIdx.x / kGroupThreads, t = threadIdx.x % kGroupThreads;
    Sums acc;
    for (int64_t row = (int64_t)blockIdx.x * kGroups + g; row < a.rows; row += (int64_t)gridDim.x * kGroups) {
        const RowIn in = row_in(a, row);
        const bool live = in.live();
        const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
        const RowShape shape = row_shape(x, (int)a.vocab);
        const uint4 *body = reinterpret_cast<const uint4 *>(x + shape.head);
        const bool has_extra = t < shape.head + shape.tail;
        const int extra = has_extra ? extra_index<T>(shape, t) : 0;
        uint4 u[kRowUnits];
        float x_extra = 0.f, x_target = CUDART_NAN_F, top = 0.f;
        RowOut o = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (live) {
            const bool inside = in.target < a.vocab;
            if (inside) x_target = widen(x[in.target]);
#pragma unroll
            for (int i = 0; i < kRowUnits; ++i)
                if (t + i * kGroupThreads < shape.units) u[i] = ld_unit(body + t + i * kGroupThreads);
            if (has_extra) x_extra = widen(x[extra]);
            Running<false> run;
#pragma unroll
            for (int i = 0; i < kRowUnits; ++i) {
                if (t + i * kGroupThreads < shape.units) {
                    const uint4 one[1] = {u[i]};
                    run.template add_units<T>(one, k);
                }
            }
            if (has_extra) run.add_one(x_extra, k);
            // the gradient may replace the logits: all have been read when the join is through
            const Stats s = group_join<W, false>(run.stats(), k, shared + g * W, g);
            top = s.top;
            o = row_out(a, in, s, x_target, k);
            if (t == 0) {
                acc.add(a, in, o);
                if (!inside) record_bad_target(a.status, row);
            }
        }
        if (t == 0 && a.logp) a.logp[row] = o.logp;
        if (a.dlogits) {
            const RowWriter<T, O> out(static_cast<O *>(a.dlogits) + row * a.ld_dlogits, shape, top, o, k);
            O *p = out.y + shape.head + t * kUnit<T>;
            const auto units = [&](auto wide) {
#pragma unroll
                for (int i = 0; i < kRowUnits; ++i) {
                    if (t + i * kGroupThreads < shape.units) {
                        if (live) out.template put<decltype(wide)::value>(u[i], p + i * kGroupThreads * kUnit<T>);
                        else out.template put_zeros<decltype(wide)::value>(p + i * kGroupThreads * kUnit<T>);
                    }
                }
            };
            if (out.wide) units(std::true_type());
            else units(std::false_type());
            if (has_extra) out.put_one(x_extra, extra);
            if (live && in.target < a.vocab && t == owner_of<T>(shape, in.target, 0, kGroupThreads))
                out.put_target(x_target, in.target);
        }
        if (W > 1) group_sync<W>(g);  // the slots are used again
    }
    finish_stats<kThreads, 32 * W>(a, acc, sums, &last, threadIdx.x);
}

// ---- longer rows: a ring in shared memory ------------------------------------------------------
// A row, or its slice where a cluster of CTAs shares one, is brought to shared memory by bulk
// copies, in stages of kStageBytes; the statistics are taken from the stages as they arrive, then the
// gradient is computed from the same stages, each of which is refilled as soon as it has been used:
// the next row streams in while this one's gradient streams out, and every logit crosses the HBM bus
// once.  One producer warp, kRingWork threads that compute.

constexpr int kStageBytes = 12288;
constexpr int kStages = 9;
constexpr int kRingsPerSm = 2;
constexpr int kRingWork = 256;
constexpr int kRingWarps = kRingWork / 32;
constexpr int kRingThreads = kRingWork + 32;
constexpr int kStageUnits = kStageBytes / 16;

struct RingShared {
    alignas(128) unsigned char stage[kStages][kStageBytes];
    alignas(16) float4 peer[2][kMaxCluster];  // {top, sum, x_target} of the cluster's CTAs, for even and odd rows
    unsigned long long full[kStages], empty[kStages], joined[2];
    Stats slots[2][kRingWarps];  // for even and odd rows: a warp may be a row ahead of another
    double sums[kRingWarps][4];
    int last, give_up;
};

// Place in the ring: a stage, and the parity of the barrier phase that its current use completes.
struct Cursor {
    uint32_t slot = 0, parity = 0;

    __device__ __forceinline__ void advance() {
        if (++slot == kStages) {
            slot = 0;
            parity ^= 1;
        }
    }
};

template <typename T, typename O>
__global__ void __launch_bounds__(kRingThreads, kRingsPerSm)
policy_loss_ring_kernel(const PolicyArgs a, float k, int log_cluster) {
    extern __shared__ unsigned char raw[];
    RingShared &sh = *reinterpret_cast<RingShared *>((reinterpret_cast<uintptr_t>(raw) + 127) & ~(uintptr_t)127);
    const int t = threadIdx.x, lane = t % 32, warp = t / 32;
    const int cluster = 1 << log_cluster;
    const int rank = cluster > 1 ? (int)cluster_rank() : 0;
    const int64_t first = blockIdx.x >> log_cluster, step = gridDim.x >> log_cluster;
    if (t == 0) {
        for (int i = 0; i < kStages; ++i) {
            barrier_init(shared_addr(&sh.full[i]), 1);
            barrier_init(shared_addr(&sh.empty[i]), kRingWarps);
        }
        for (int i = 0; i < 2; ++i) barrier_init(shared_addr(&sh.joined[i]), 1);
        sh.give_up = 0;
        barrier_init_fence();
    }
    __syncthreads();
    if (cluster > 1) cluster_sync();  // the peers' barriers are ready before the first message

    if (warp == kRingWarps) {
        // ---- producer
        if (lane == 0) {
            Cursor c;
            uint32_t issued = 0;  // stages, up to kStages
            for (int64_t row = first; row < a.rows && !*(volatile int *)&sh.give_up; row += step) {
                if (a.weights[row] == 0.f || a.targets[row] < 0) continue;
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
            }
        }
    } else {
        Sums acc;
        Cursor c;
        uint32_t joins = 0;  // rows joined
        RowIn next = {-1, 0.f, 0.f, 0.f, 0.f};
        if (first < a.rows) next = row_in(a, first);
        for (int64_t row = first; row < a.rows; row += step) {
            const RowIn in = next;
            if (row + step < a.rows) next = row_in(a, row + step);
            const bool live = in.live();
            const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
            const RowShape shape = row_shape(x, (int)a.vocab);
            int from, count;
            slice_of(shape.units, rank, log_cluster, from, count);
            const bool has_extra = rank == 0 && t < shape.head + shape.tail;
            const int extra = has_extra ? extra_index<T>(shape, t) : 0;
            const Cursor c0 = c;
            float x_extra = 0.f, xt = 0.f, top = 0.f;
            RowOut o = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (live) {
                const bool inside = in.target < a.vocab;
                const float x_target = t == 0 && inside ? widen(x[in.target]) : CUDART_NAN_F;
                if (has_extra) x_extra = widen(x[extra]);
                Running<false> run;
                for (int at = 0; at < count; at += kStageUnits, c.advance()) {
                    barrier_wait(shared_addr(&sh.full[c.slot]), c.parity, &sh.give_up);
                    const uint4 *units = reinterpret_cast<const uint4 *>(sh.stage[c.slot]);
                    if (count - at >= kStageUnits) {
                        uint4 u[kStageUnits / kRingWork];
#pragma unroll
                        for (int i = 0; i < kStageUnits / kRingWork; ++i) u[i] = units[t + i * kRingWork];
                        run.template add_units<T>(u, k);
                    } else {
                        for (int i = t; i < count - at; i += kRingWork) {
                            const uint4 u[1] = {units[i]};
                            run.template add_units<T>(u, k);
                        }
                    }
                }
                if (has_extra) run.add_one(x_extra, k);
                // the CTA's statistics, then the cluster's; thread 0's x_target travels with them
                Stats s = warp_join<false>(run.stats(), k);
                const int b = joins & 1;
                if (lane == 0) sh.slots[b][warp] = {s.top, s.sum, x_target};
                asm volatile("bar.sync 1, %0;" ::"n"(kRingWork) : "memory");
                const Stats none = {-CUDART_INF_F, 0.f, 0.f};
                const Stats mine = lane < kRingWarps ? sh.slots[b][lane] : none;
                s = warp_join<false>(mine, k);
                xt = __shfl_sync(0xffffffffu, mine.wsum, 0);
                if (cluster > 1) {
                    const uint32_t bar = shared_addr(&sh.joined[b]);
                    if (t == 0) barrier_expect(bar, 16u * cluster);
                    if (t < cluster) send16(shared_addr(&sh.peer[b][rank]), bar, t, s.top, s.sum, xt, 0.f);
                    barrier_wait(bar, (joins >> 1) & 1, &sh.give_up);
                    Stats p = none;
                    if (lane < cluster) {
                        const float4 q = sh.peer[b][lane];
                        p = {q.x, q.y, q.z};
                    }
                    s = warp_join<false>(p, k);
                }
                ++joins;
                top = s.top;
                o = row_out(a, in, s, xt, k);
                if (t == 0 && rank == 0) {
                    acc.add(a, in, o);
                    if (!inside) record_bad_target(a.status, row);
                }
            }
            if (t == 0 && rank == 0 && a.logp) a.logp[row] = o.logp;
            const RowWriter<T, O> out(static_cast<O *>(a.dlogits) + row * a.ld_dlogits, shape, top, o, k);
            O *p = out.y + shape.head + (int64_t)(from + t) * kUnit<T>;
            if (live) {
                c = c0;
                const auto release = [&]() {
                    __syncwarp();
                    if (lane == 0) barrier_arrive(shared_addr(&sh.empty[c.slot]));
                };
                const auto stages = [&](auto wide) {
                    for (int at = 0; at < count; at += kStageUnits, c.advance(), p += kStageUnits * kUnit<T>) {
                        const uint4 *units = reinterpret_cast<const uint4 *>(sh.stage[c.slot]) + t;
                        if (count - at >= kStageUnits) {
                            uint4 u[kStageUnits / kRingWork];
#pragma unroll
                            for (int i = 0; i < kStageUnits / kRingWork; ++i) u[i] = units[i * kRingWork];
#pragma unroll
                            for (int i = 0; i < kStageUnits / kRingWork; ++i)
                                out.template put<decltype(wide)::value>(u[i], p + i * kRingWork * kUnit<T>);
                        } else {
                            for (int i = 0; i < count - at - t; i += kRingWork)
                                out.template put<decltype(wide)::value>(units[i], p + i * kUnit<T>);
                        }
                        release();
                    }
                };
                if (!a.dlogits)
                    for (int at = 0; at < count; at += kStageUnits, c.advance()) release();
                else if (out.wide) stages(std::true_type());
                else stages(std::false_type());
            } else if (a.dlogits) {
                for (int i = 0; i < count - t; i += kRingWork) {
                    if (out.wide) out.template put_zeros<true>(p + (int64_t)i * kUnit<T>);
                    else out.template put_zeros<false>(p + (int64_t)i * kUnit<T>);
                }
            }
            if (a.dlogits) {
                if (has_extra) out.put_one(x_extra, extra);
                if (live && in.target < a.vocab && t == owner_of<T>(shape, in.target, from, kRingWork)) {
                    const int at = ((int)in.target - shape.head) / kUnit<T> - from;
                    const bool extra_one = in.target < shape.head || in.target >= shape.head + shape.units * kUnit<T>;
                    if (extra_one ? rank == 0 : at >= 0 && at < count) out.put_target(xt, in.target);
                }
            }
        }
        if (t == 0 && sh.give_up && atomicCAS(a.status, (unsigned)kDevOk, (unsigned)kDevTimeout) == (unsigned)kDevOk)
            a.status[1] = kWaitPolicyRing;
        finish_stats<kRingWork, kRingWork>(a, acc, sh.sums, &sh.last, t);
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
            o = row_out(a, in, s, x_target, k);
            if (t == 0) {
                acc.add(a, in, o);
                if (!inside) record_bad_target(a.status, row);
            }
        }
        if (t == 0 && a.logp) a.logp[row] = o.logp;
        if (a.dlogits) {
            const RowWriter<T, O> out(static_cast<O *>(a.dlogits) + row * a.ld_dlogits, shape, top, o, k);
            O *p = out.y + shape.head;
            const auto units = [&](auto wide) {
                for (int i = t; i < shape.units; i += kThreads) {
                    if (live) out.template put<decltype(wide)::value>(ld_unit(body + i), p + (int64_t)i * kUnit<T>);
                    else out.template put_zeros<decltype(wide)::value>(p + (int64_t)i * kUnit<T>);
                }
            };
            if (out.wide) units(std::true_type());
            else units(std::false_type());
            if (has_extra) out.put_one(x_extra, extra);
            if (live && in.target < a.vocab && t == owner_of<T>(shape, in.target, 0, kThreads))
                out.put_target(x_target, in.target);
        }
        group_sync<kWarps>(0);  // the slots are used again
    }
    finish_stats<kThreads, kThreads>(a, acc, sums, &last, t);
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
    if (units <= 128 * kRowUnits || a.rows >= 8 * (int64_t)sm_count) return logprobs_groups<T, 4, 1>(a, k, stream);
    int cluster = 1;  // more CTAs to a row while there are fewer rows than SMs and work for their threads
    while (cluster < kMaxCluster && a.rows * cluster * 2 <= sm_count && units >= cluster * 2 * kThreads) cluster *= 2;
    return cluster > 1 ? logprobs_cluster<T>(a, k, cluster, stream) : logprobs_groups<T, kWarps, 1>(a, k, stream);
}

template <typename T, typename O, int W>
cudaError_t policy_rows(const PolicyArgs &a, float k, int sm_count, cudaStream_t stream) {
    const int64_t ctas = (a.rows + kWarps / W - 1) / (kWarps / W);
    policy_loss_rows_kernel<T, O, W><<<grid_of(ctas, (int64_t)sm_count * 2), kThreads, 0, stream>>>(a, k);
    return cudaGetLastError();
}

template <typename T, typename O>
cudaError_t policy_ring(const PolicyArgs &a, float k, int cluster, int sm_count, cudaStream_t stream) {
    constexpr size_t bytes = sizeof(RingShared) + 128;
    static std::atomic<unsigned long long> ready{0};
    cudaError_t e = allow_shared(policy_loss_ring_kernel<T, O>, (int)bytes, ready);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    const int64_t most = sm_count * kRingsPerSm / cluster;
    cfg.gridDim = dim3((unsigned)((a.rows < 1 ? 1 : a.rows < most ? a.rows : most) * cluster));
    cfg.blockDim = dim3(kRingThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim = {(unsigned)cluster, 1, 1};
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, policy_loss_ring_kernel<T, O>, a, k, log2_of(cluster));
}

template <typename T, typename O>
cudaError_t policy(const PolicyArgs &a, int sm_count, cudaStream_t stream) {
    const float k = (float)(a.scale_exact * kLog2e);
    const int64_t units = a.vocab / kUnit<T>;
    if (units <= 32 * kRowUnits) return policy_rows<T, O, 1>(a, k, sm_count, stream);
    if (units <= 128 * kRowUnits) return policy_rows<T, O, 4>(a, k, sm_count, stream);
    // as few CTAs to a row as hold it, more while there are fewer rows than SMs
    constexpr int64_t kRing = (int64_t)kStages * kStageUnits;
    int cluster = 1;
    while (cluster < kMaxCluster && ((units + cluster - 1) / cluster > kRing || a.rows * cluster * 2 <= sm_count)) cluster *= 2;
    if ((units + cluster - 1) / cluster <= kRing)
        return policy_ring<T, O>(a, k, cluster, sm_count, stream);
    policy_loss_long_kernel<T, O><<<grid_of(a.rows, (int64_t)sm_count * 4), kThreads, 0, stream>>>(a, k);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_token_logprobs(const LogprobArgs &a, int sm_count, cudaStream_t stream) {
    return a.dtype == ADAMA_F32 ? logprobs<float>(a, sm_count, stream) : logprobs<__nv_bfloat16>(a, sm_count, stream);
}

cudaError_t launch_policy_loss(const PolicyArgs &a, int sm_count, cudaStream_t stream) {
    if (a.logits_dtype == ADAMA_F32)
        return a.dlogits_dtype == ADAMA_F32 ? policy<float, float>(a, sm_count, stream)
                                            : policy<float, __nv_bfloat16>(a, sm_count, stream);
    return a.dlogits_dtype == ADAMA_F32 ? policy<__nv_bfloat16, float>(a, sm_count, stream)
                                        : policy<__nv_bfloat16, __nv_bfloat16>(a, sm_count, stream);
}

}  // namespace adama
