// Token log-probabilities and the clipped policy loss with its gradient, from rows of logits.
// With z = s*x (s = logit_scale) a row's lse = log sum_j exp(z_j), p_j = exp(z_j - lse),
// logp = z_target - lse, entropy = lse - sum_j p_j z_j.  For a row with weight w:
//     r = exp(logp - old),  pg = -min(r*A, clamp(r, 1-cl, 1+ch)*A),  d = ref - logp,
//     kl = exp(d) - d - 1,  loss += w*(pg + beta*kl)
//     dlogits_j = w*s*c*([j = target] - p_j),  c = -(r*A while r*A <= the clamped product) + beta*(1 - exp(d))
// A row is read once (loss: and its gradient written once).  Beside HBM the exponentials count, one per
// element for the statistics and one for the gradient, at 16 per clock and SM.  Log-probabilities of 4096 rows
// of 50304 bf16 with entropy: 69 us = 5.98 TB/s; loss and gradient of 8192 rows of 50257, a quarter of them
// masked: 256 us = 5.6 TB/s, of 6103 rows of 32768, which fill the ring's stages, 117 us = 6.0 TB/s; the
// log-probability of one row of 50257 fp32: 3.9 us.

#include "adama_device.cuh"
#include "bulk_copy.cuh"
#include "policy_plan.h"
#include "softmax_rows.cuh"
#include "tensor_table.cuh"

namespace adama {
namespace {

constexpr int kThreads = 512;  // that work on rows, in every kernel here
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ void record_bad_target(unsigned *status, int64_t row) {
    if (atomicCAS(status + kStatusTarget, 0u, 1u) == 0u) {
        status[kStatusTarget + 1] = (unsigned)row;
        status[kStatusTarget + 2] = (unsigned)(row >> 32);
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

// In natural units: the rounding of k does not show but through the sum.
__device__ __forceinline__ float logp_of(float x_target, const Stats &s, float log_sum, float scale) {
    return fmaf(scale, x_target - s.top, -log_sum);
}

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

// Sums of one thread over its rows; in double, so that their order does not show in fp32.
struct Sums {
    double v[4] = {0.0, 0.0, 0.0, 0.0};

    __device__ __forceinline__ void add(const PolicyArgs &a, const RowIn &in, const RowOut &o) {
        const double w = in.weight;
        v[0] += w * (o.pg + (a.ref_logp && a.kl_coef != 0.f ? a.kl_coef * o.kl : 0.f));
        v[1] += w * o.pg;
        v[2] += w * o.kl;
        v[3] += w * o.cut;
    }
};

// The leaders' sums -> the CTA's in the workspace -> stats, by the last CTA, in the CTAs' order.  All
// THREADS call it; thread LEADER*i holds the sums of leader i.  CTA `index` of `count` that have sums.
template <int THREADS, int LEADER>
__device__ __forceinline__ void finish_stats(const PolicyArgs &a, const Sums &s, double (*slots)[4], volatile int *last,
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

template <typename O>
__device__ __forceinline__ O narrow(float y);
template <>
__device__ __forceinline__ float narrow<float>(float y) { return y; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float y) { return __float2bfloat16_rn(y); }

// N values as 32-bit words of their type
__device__ __forceinline__ void to_words(const float (&v)[4], unsigned (&w)[4], float) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[i]);
}
__device__ __forceinline__ void to_words(const float (&v)[8], unsigned (&w)[8], float) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
}
__device__ __forceinline__ void to_words(const float (&v)[4], unsigned (&w)[2], __nv_bfloat16) {
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = pack2_bf16(v[2 * i], v[2 * i + 1]);
}
__device__ __forceinline__ void to_words(const float (&v)[8], unsigned (&w)[4], __nv_bfloat16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack2_bf16(v[2 * i], v[2 * i + 1]);
}
__device__ __forceinline__ void store_words(void *p, const unsigned (&w)[2]) { *static_cast<uint2 *>(p) = make_uint2(w[0], w[1]); }
__device__ __forceinline__ void store_words(void *p, const unsigned (&w)[4]) {
    *static_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_words(void *p, const unsigned (&w)[8]) {
    static_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    static_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

// Zeros to p[0 .. n) by `threads` threads.
template <typename O>
__device__ __forceinline__ void fill_zeros(O *p, int64_t n, int t, int threads) {
    constexpr int kPer = 16 / sizeof(O);
    const int mis = (int)(reinterpret_cast<uintptr_t>(p) % 16 / sizeof(O));
    const int64_t head = mis ? (kPer - mis < n ? kPer - mis : n) : 0, body = (n - head) / kPer;
    for (int64_t i = t; i < body; i += threads) reinterpret_cast<uint4 *>(p + head)[i] = make_uint4(0, 0, 0, 0);
    const int64_t tail0 = head + body * kPer;
    if (t < head) p[t] = narrow<O>(0.f);
    if (t < n - tail0) p[tail0 + t] = narrow<O>(0.f);
}

// How a row's gradient is written.  The units are written without the target's extra term; the
// thread that wrote the target's element writes it again, with the term.
//
// A unit's gradient is one aligned store where logits and gradient have the same alignment.  Where they
// have not, a thread takes the window of N logits from `shift` on, which ends in the next unit: the
// raw words of both are shifted into place before anything is computed, and only the first `shift`
// elements of a slice and the last N - shift are stored one by one.  (Then logits and gradient are
// different buffers: in place they share their pitch.)
template <typename T, typename O>
struct RowWriter {
    static constexpr int N = kUnit<T>;
    static constexpr int kWords = N * sizeof(O) / 4;             // a unit's gradient
    static constexpr int kStoreWords = kWords < 4 ? kWords : 4;  // one store
    int shift;  // elements between a unit's first one and the next aligned address; 0: aligned stores
    float top, unit, per_e, k;

    __device__ __forceinline__ RowWriter(const O *row, const RowShape &shape, float top_, float unit_, float per_e_, float k_)
        : top(top_), unit(unit_), per_e(per_e_), k(k_) {
        constexpr int kPer = kStoreWords * 4 / sizeof(O);
        const int mis = (int)(reinterpret_cast<uintptr_t>(row + shape.head) % (kStoreWords * 4) / sizeof(O));
        shift = mis ? kPer - mis : 0;
    }
    // the gradient of N logits
    __device__ __forceinline__ void values(const uint4 &u, float (&v)[N]) const {
        const Pair k2 = pair(k, k), per = pair(per_e, per_e);
#pragma unroll
        for (int q = 0; q < N / 2; ++q) {
            float d0, d1;
            split(mul2(unit_less<T>(u, q, top), k2), d0, d1);
            split(mul2(pair(exp2_fast(d0), exp2_fast(d1)), per), v[2 * q], v[2 * q + 1]);
        }
    }
    __device__ __forceinline__ void put(const uint4 &u, O *p) const {
        float v[N];
        values(u, v);
        unsigned w[kWords];
        to_words(v, w, O());
        store_words(p, w);
    }
    // shift > 0: u goes to p; `first`: the slice begins with it, `last`: it ends with it, else `next` follows
    __device__ __forceinline__ void put_shifted(const uint4 &u, const uint4 &next, O *p, bool first, bool last) const {
        unsigned z[8] = {u.x, u.y, u.z, u.w, next.x, next.y, next.z, next.w};
        const int words = shift * (int)sizeof(T) / 4;
        if (words & 2) {
#pragma unroll
            for (int i = 0; i < 6; ++i) z[i] = z[i + 2];
        }
        if (words & 1) {
#pragma unroll
            for (int i = 0; i < 5; ++i) z[i] = z[i + 1];
        }
        if (sizeof(T) == 2 && (shift & 1)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = __funnelshift_r(z[i], z[i + 1], 16);
        }
        if (!last) put(make_uint4(z[0], z[1], z[2], z[3]), p + shift);
        if (first || last) {
            float v[N];
            values(u, v);
#pragma unroll
            for (int q = 0; q < N; ++q)
                if (q < shift ? first : last) p[q] = narrow<O>(v[q]);
        }
    }
    __device__ __forceinline__ O value(float x, bool is_target) const {
        const float p = per_e * exp2_fast(k * (x - top));
        return narrow<O>(is_target ? p + unit : p);
    }
    // Thread of a group of `threads` that wrote element j, of a slice of `count` units from unit `from`
    // on that go round the threads; -1: it is not among the slice's units.
    __device__ __forceinline__ int writer_of(const RowShape &shape, int64_t j, int from, int count, int threads) const {
        const int64_t at = j - shape.head - (int64_t)from * N;
        if (at < 0 || at >= (int64_t)count * N) return -1;
        const int u = (int)(at / N);
        return (at % N < shift && u > 0 ? u - 1 : u) % threads;
    }
};

// ---- rows that fit a warp's registers -----------------------------------------------------------

// One row at a time to a warp, 32 warps to an SM hide its latencies: 100000 x 2000 bf16 143 us (76 % of a
// copy's rate), 333333 x 600 248 us (44 %).  What holds these back is no floor: all 32 lanes compute the row's
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
            acc.add(a, in, o);
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

// ---- longer rows: a ring in shared memory ------------------------------------------------------
// A row, or its slice where a cluster of CTAs shares one, is brought to shared memory by bulk copies,
// in stages; the statistics are taken from the stages as they arrive, then the gradient is computed
// from the same stages, each of which is refilled as soon as it has been used: every logit crosses the
// HBM bus once.  The warps that compute take row i+1's statistics BEFORE they write row i's gradient:
// between a row's statistics and its gradient lie the joins over warps and CTAs and the loss itself,
// which one warp of its own does meanwhile, and nobody waits for them.  The ring therefore holds two
// rows (slices).  One more warp issues the copies.

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

template <typename T, typename O, typename Cut>
__global__ void __launch_bounds__(Cut::kThreads, Cut::kPerSm)
policy_loss_ring_kernel(const PolicyArgs a, float k, int log_cluster) {
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
                report_expired_wait(&sh.give_up, a.status, kWaitPolicyRing);
            }
        }
    } else if (warp == Cut::kScalarWarp) {
        Sums acc;
        uint32_t n = 0;  // live rows
        RowIn next = {-1, 0.f, 0.f, 0.f, 0.f};
        if (first < a.rows) next = row_in(a, first);
        for (int64_t row = first; row < a.rows; row += step) {
            const RowIn in = next;
            if (row + step < a.rows) next = row_in(a, row + step);
            if (!in.live()) {
                if (lane == 0 && rank == 0 && a.logp) a.logp[row] = 0.f;
                continue;
            }
            const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
            const RowShape shape = row_shape(x, (int)a.vocab);
            int from, count;
            slice_of(shape.units, rank, log_cluster, from, count);
            const int b = n & 1;
            const uint32_t parity = n >> 1 & 1;
            const bool inside = in.target < a.vocab, has_extra = rank == 0 && lane < shape.head + shape.tail;
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
                if (rank == 0) {
                    acc.add(a, in, o);
                    if (a.logp) a.logp[row] = o.logp;
                    if (!inside) record_bad_target(a.status, row);
                }
            }
            if (has_extra && a.dlogits) y[extra] = out.value(x_extra, extra == in.target);
            ++n;
        }
        if (lane == 0) report_expired_wait(&sh.give_up, a.status, kWaitPolicyRing);
        __syncwarp();
        if (rank == 0) finish_stats<32, 32>(a, acc, sh.sums, &sh.last, lane, (unsigned)first, (unsigned)step);
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
            const auto release = [&]() {
                __syncwarp();
                if (lane == 0) barrier_arrive(shared_addr(&sh.empty[at_stage.slot]));
            };
            O *p = y + shape.head + (int64_t)(from + t) * kUnit<T>;
            if (!a.dlogits || !ok) {
                for (int at = 0; at < count; at += kStageUnits, at_stage.advance()) release();
                return;
            }
            if (out.shift == 0) {
                int at = 0;
                for (; count - at >= 2 * kStageUnits; at += 2 * kStageUnits, p += 2 * kStageUnits * kUnit<T>) {
                    uint4 u[2 * kEach];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint4 *units = reinterpret_cast<const uint4 *>(sh.stage[at_stage.slot]) + t;
#pragma unroll
                        for (int i = 0; i < kEach; ++i) u[j * kEach + i] = units[i * kRingWork];
                        release();
                        at_stage.advance();
                    }
#pragma unroll
                    for (int i = 0; i < 2 * kEach; ++i) out.put(u[i], p + i * kRingWork * kUnit<T>);
                }
                for (; at < count; at += kStageUnits, at_stage.advance(), p += kStageUnits * kUnit<T>) {
                    const uint4 *units = reinterpret_cast<const uint4 *>(sh.stage[at_stage.slot]) + t;
                    if (count - at >= kStageUnits) {
                        uint4 u[kEach];
#pragma unroll
                        for (int i = 0; i < kEach; ++i) u[i] = units[i * kRingWork];
#pragma unroll
                        for (int i = 0; i < kEach; ++i) out.put(u[i], p + i * kRingWork * kUnit<T>);
                    } else {
#pragma unroll 1
                        for (int i = 0; i < count - at - t; i += kRingWork) out.put(units[i], p + i * kUnit<T>);
                    }
                    release();
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
        float next_weight = 0.f;
        int64_t next_target = -1;
        if (first < a.rows) {
            next_weight = a.weights[first];
            next_target = a.targets[first];
        }
        for (int64_t row = first; row < a.rows; row += step) {
            const bool live = next_weight != 0.f && next_target >= 0;
            if (row + step < a.rows) {
                next_weight = a.weights[row + step];
                next_target = a.targets[row + step];
            }
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
                acc.add(a, in, o);
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
cudaError_t policy_rows(const PolicyArgs &a, float k, int sm_count, cudaStream_t stream) {
    policy_loss_rows_kernel<T, O><<<grid_of((a.rows + kWarps - 1) / kWarps, (int64_t)sm_count * 2), kThreads, 0, stream>>>(a, k);
    return cudaGetLastError();
}

template <typename T, typename O, typename Cut>
struct RingLaunch {
    static constexpr int kBytes = (int)sizeof(RingShared<Cut>) + 128;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;

    RingLaunch(int cluster, int64_t clusters, cudaStream_t stream) {
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim = {(unsigned)cluster, 1, 1};
        cfg.gridDim = dim3((unsigned)(clusters * cluster));
        cfg.blockDim = dim3(Cut::kThreads);
        cfg.dynamicSmemBytes = kBytes;
        cfg.stream = stream;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
    }
    RingLaunch(const RingLaunch &) = delete;  // cfg points at attr

    static cudaError_t prepare() {
        static std::atomic<unsigned long long> ready{0};
        return allow_shared(policy_loss_ring_kernel<T, O, Cut>, kBytes, ready);
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
            e = cudaOccupancyMaxActiveClusters(&m, policy_loss_ring_kernel<T, O, Cut>, &l.cfg);
            if (e != cudaSuccess) return e;
            if (m < 1) m = 1;
            if (slot) slot->store(m);
        }
        *out = m;
        return cudaSuccess;
    }
    static cudaError_t launch(const PolicyArgs &a, float k, int cluster, int sm_count, cudaStream_t stream) {
        int most = 0;
        cudaError_t e = prepare();
        if (e == cudaSuccess) e = resident(cluster, sm_count, &most);
        if (e != cudaSuccess) return e;
        RingLaunch l(cluster, a.rows < 1 ? 1 : a.rows < most ? a.rows : most, stream);
        return cudaLaunchKernelEx(&l.cfg, policy_loss_ring_kernel<T, O, Cut>, a, k, log2_of(cluster));
    }
};

template <typename T, typename O>
cudaError_t policy(const PolicyArgs &a, int sm_count, cudaStream_t stream) {
    const float k = (float)(a.scale_exact * kLog2e);
    PolicyPlan plan;
    const int e = plan_policy(a.vocab / kUnit<T>, a.rows, sm_count, [&](PolicyForm form, int cluster, int *most) {
        return (int)(form == kForm640 ? RingLaunch<T, O, Cut640>::resident(cluster, sm_count, most)
                                      : RingLaunch<T, O, Cut512>::resident(cluster, sm_count, most));
    }, plan);
    if (e != 0) return (cudaError_t)e;
    switch (plan.form) {
        case kFormRows: return policy_rows<T, O>(a, k, sm_count, stream);
        case kForm64: return RingLaunch<T, O, Cut64>::launch(a, k, plan.cluster, sm_count, stream);
        case kForm128: return RingLaunch<T, O, Cut128>::launch(a, k, plan.cluster, sm_count, stream);
        case kForm256: return RingLaunch<T, O, Cut256>::launch(a, k, plan.cluster, sm_count, stream);
        case kForm512: return RingLaunch<T, O, Cut512>::launch(a, k, plan.cluster, sm_count, stream);
        case kForm640: return RingLaunch<T, O, Cut640>::launch(a, k, plan.cluster, sm_count, stream);
        case kFormLong: break;
    }
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
