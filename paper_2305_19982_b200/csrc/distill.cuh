// Distillation from a teacher's top logits: the part of a row that its few entries make, for the kernels on rows
// of logits.  With z = s*x, q_j = exp(z_j - lse) the student's probabilities, and per entry i the teacher's
//     log p_i = s*t_i - lse_T   (lse_T given, or the log-sum over the row's entries: they then sum to 1),  P = sum p_i
//     kl = sum p_i (log p_i - log q_{j_i}),   dlogits_j = w*s*(P*q_j - sum over entries of j of p_i)
// All but the entries' own elements have the form that the ring writes for any loss, per_e * 2^(k*(x - top)); the
// entries' elements are written once more, with their term, when the row's other writers are through.
#pragma once

#include "adama_device.cuh"
#include "logit_ring.cuh"
#include "row_writer.cuh"

namespace adama {

constexpr int kTopEach = ADAMA_DISTILL_TOP / 32;  // entries of a lane

// Whether a warp has entries at 32*e: most rows have fewer than 128, and the warp that deals with them works alone.
__device__ __forceinline__ bool in_use(const DistillArgs &a, int e) { return e == 0 || 32 * e < a.top; }

// A lane's entries, 32*e + lane, as they come from memory: nothing here waits for the loads.
struct RawEntries {
    int64_t id[kTopEach];
    unsigned t[kTopEach];  // fp32 or bf16
};
__device__ __forceinline__ void load_entries(const DistillArgs &a, int64_t row, int lane, RawEntries &r) {
    const int64_t *ids = a.ids + row * a.ld_ids + lane;
    const int64_t at = row * a.ld_teacher + lane;
    const bool wide = a.teacher_dtype == ADAMA_F32;
#pragma unroll
    for (int e = 0; e < kTopEach; ++e)
        if (in_use(a, e) && 32 * e + lane < a.top) {
            r.id[e] = ids[32 * e];
            if (wide) r.t[e] = static_cast<const unsigned *>(a.teacher)[at + 32 * e];
            else r.t[e] = static_cast<const unsigned short *>(a.teacher)[at + 32 * e];
        }
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
__device__ __forceinline__ float warp_max(float x) {
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}

// The teacher's side of a row.
struct Entries {
    int id[kTopEach];      // -1: none
    float p[kTopEach];     // probability, 0 for none
    float logp[kTopEach];  // where p > 0
    float own[kTopEach];   // sum of p over the entries of the same index
    float mass;            // P; NaN where an index lies outside the vocabulary
    bool bad;              // there is one
};
// (own is p: join_twice sees to indices that occur more than once)
__device__ __forceinline__ Entries entries_of(const DistillArgs &a, const RawEntries &raw, float lse, int lane) {
    Entries r;
    bool bad = false;
    float t[kTopEach], top = -CUDART_INF_F;
#pragma unroll
    for (int e = 0; e < kTopEach; ++e) {
        r.id[e] = -1;
        t[e] = -CUDART_INF_F;
        r.p[e] = r.logp[e] = 0.f;
        if (in_use(a, e) && 32 * e + lane < a.top && raw.id[e] >= 0) {
            if (raw.id[e] < a.vocab) {
                r.id[e] = (int)raw.id[e];
                t[e] = __uint_as_float(a.teacher_dtype == ADAMA_F32 ? raw.t[e] : raw.t[e] << 16);
                top = fmaxf(top, t[e] != t[e] ? CUDART_INF_F : t[e]);  // a NaN shows below
            } else {
                bad = true;
            }
        }
    }
    r.bad = __any_sync(0xffffffffu, bad);
    float offset = -lse, ref = 0.f;  // log p = s*(t - ref) + offset
    if (!a.teacher_lse) {
        ref = warp_max(top);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < kTopEach; ++e)
            if (in_use(a, e) && t[e] != -CUDART_INF_F) sum += expf(a.scale * (t[e] - ref));
        offset = -logf(warp_sum(sum));
    }
    float mass = 0.f;
#pragma unroll
    for (int e = 0; e < kTopEach; ++e) {
        if (in_use(a, e) && t[e] != -CUDART_INF_F) {
            r.logp[e] = fmaf(a.scale, t[e] - ref, offset);
            r.p[e] = expf(r.logp[e]);
        }
        mass += r.p[e];
        r.own[e] = r.p[e];
    }
    // without a given log-sum the entries are the whole of it: a sum of 1, or of NaN, or no entry at all
    if (a.teacher_lse) r.mass = warp_sum(mass);
    else r.mass = ref == -CUDART_INF_F ? 0.f : offset == offset && ref != CUDART_INF_F ? 1.f : CUDART_NAN_F;
    if (r.bad) r.mass = CUDART_NAN_F;
    return r;
}

// The same index more than once is rare, but its element has one gradient.  Whether there is any: every entry
// is compared with all others.
__device__ __forceinline__ bool any_twice(const DistillArgs &a, const Entries &r) {
    bool twice = false;
#pragma unroll
    for (int e = 0; e < kTopEach; ++e)
        if (in_use(a, e)) {
            const unsigned same = __match_any_sync(0xffffffffu, r.id[e]);
            twice |= r.id[e] >= 0 && (same & (same - 1)) != 0;
        }
#pragma unroll
    for (int f = 0; f < kTopEach - 1; ++f)
        if (in_use(a, f + 1)) {
            const int id = r.id[f] < 0 ? -2 : r.id[f];
#pragma unroll 8
            for (int l = 0; l < 32; ++l) {
                const int other = __shfl_sync(0xffffffffu, id, l);
#pragma unroll
                for (int e = f + 1; e < kTopEach; ++e) twice |= r.id[e] == other;
            }
        }
    return __any_sync(0xffffffffu, twice);
}
__device__ __noinline__ void join_twice(const int (&id)[kTopEach], const float (&p)[kTopEach], float (&own)[kTopEach]) {
#pragma unroll
    for (int e = 0; e < kTopEach; ++e) own[e] = 0.f;
#pragma unroll 1
    for (int l = 0; l < 32; ++l)
#pragma unroll
        for (int f = 0; f < kTopEach; ++f) {
            const int other = __shfl_sync(0xffffffffu, id[f], l);
            const float q = __shfl_sync(0xffffffffu, p[f], l);
#pragma unroll
            for (int e = 0; e < kTopEach; ++e)
                if (id[e] == other) own[e] += q;
        }
}

// What all but the entries' elements of a row's gradient are made of.
__device__ __forceinline__ float per_e_of(const DistillArgs &a, float mass, float weight, float sum) {
    return mass == 0.f ? 0.f : weight * a.scale * mass / sum;  // no entry: nothing to learn, whatever the logits
}

// A lane's share of a row's loss terms; g: the gradient of its entries' elements.
struct DistillOut {
    float kl, cross, held;  // held: the student's mass on the entries
    float g[kTopEach];
};
__device__ __forceinline__ DistillOut distill_out(const DistillArgs &a, const Entries &en, const float (&x)[kTopEach],
                                                  const bool (&mine)[kTopEach], float weight, float top, float sum, float k) {
    DistillOut o;
    const float log_sum = logf(sum), unit = weight * a.scale, inv = 1.f / sum;
    o.kl = o.cross = o.held = 0.f;
#pragma unroll
    for (int e = 0; e < kTopEach; ++e)
        if (in_use(a, e) && mine[e]) {
            const float d = x[e] - top, logq = fmaf(a.scale, d, -log_sum);
            const float q = exp2_fast(k * d) * inv;
            o.g[e] = en.bad ? CUDART_NAN_F : unit * fmaf(en.mass, q, -en.own[e]);
            o.held += q;
            if (en.p[e] != 0.f) {  // no probability, no loss, also where the student has none either
                o.kl = fmaf(en.p[e], en.logp[e] - logq, o.kl);
                o.cross = fmaf(-en.p[e], logq, o.cross);
            }
        }
    if (en.bad) o.kl = o.cross = o.held = CUDART_NAN_F;
    return o;
}

// Every lane adds its share; the mass is the row's, and added once.
__device__ __forceinline__ void add_terms(Sums &sums, float weight, const Entries &en, const DistillOut &o, bool once) {
    sums.add(weight, o.kl, o.cross, o.held, once ? en.mass : 0.f);
}
__device__ __forceinline__ void sum_lanes(Sums &sums) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sums.v[i] += __shfl_xor_sync(0xffffffffu, sums.v[i], o);
}

// ---- the warp between a row's statistics and its gradient ----------------------------------------

// Elements of a row that wait to be written over.
template <typename O>
struct Patches {
    O *row;
    int id[kTopEach];  // -1: none, or another CTA's
    float g[kTopEach];

    __device__ __forceinline__ void write(const DistillArgs &a) const {
#pragma unroll
        for (int e = 0; e < kTopEach; ++e)
            if (in_use(a, e) && id[e] >= 0) row[id[e]] = narrow<O>(g[e]);
    }
};

// Marks an element of a stage that holds x; false where it has been marked before.  Nobody but this warp looks
// at a row's stages between its statistics and its verdict, and what is written for a marked element is
// written over, so the mark (a NaN) stays.
__device__ __forceinline__ bool mark(float *at, float x) {
    const unsigned bits = __float_as_uint(x);
    return atomicCAS(reinterpret_cast<unsigned *>(at), bits, 0x7fffffffu) == bits;
}
__device__ __forceinline__ bool mark(__nv_bfloat16 *at, float x) {
    const unsigned short bits = (unsigned short)(__float_as_uint(x) >> 16);
    return atomicCAS(reinterpret_cast<unsigned short *>(at), bits, (unsigned short)0x7fff) == bits;
}

// In the ring's warp of its own: joins, loss terms, verdicts.  It shares its scheduler and its path to memory with
// busy warps, so what counts is the number of its instructions, above all of exchanges between lanes, and that it waits
// for no load: weights come two rows ahead, entries and a row's extras one, the entries' logits from the ring.
// The working warps have written row n-2 when they have all given their statistics of row n: then the entries'
// elements of row n-2 are written over, those of the last two rows when the working warps have come to their end.
template <typename T, typename O, typename Cut>
__device__ __forceinline__ void distill_verdicts(const DistillArgs &a, float k, RingShared<Cut> &sh, int lane, int rank, int log_cluster,
                                                 int64_t first, int64_t step, Sums &acc) {
    const int cluster = 1 << log_cluster;
    uint32_t n = 0;     // live rows
    uint32_t slot = 0;  // the stage that a row's slice begins in
    Patches<O> waiting[2];
    float after_weight = 0.f, next_weight = 0.f, next_lse = 0.f;
    T next_extra = narrow<T>(0.f);
    RawEntries next = {};
    const auto look_ahead = [&](int64_t row) {
        next_weight = after_weight;
        after_weight = row + step < a.rows ? a.weights[row + step] : 0.f;
        if (next_weight != 0.f) {
            load_entries(a, row, lane, next);
            if (a.teacher_lse) next_lse = a.teacher_lse[row];
            const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
            const RowShape shape = row_shape(x, (int)a.vocab);
            if (rank == 0 && lane < shape.head + shape.tail) next_extra = x[extra_index<T>(shape, lane)];
        }
    };
    after_weight = first < a.rows ? a.weights[first] : 0.f;
    look_ahead(first);
    for (int64_t row = first; row < a.rows; row += step) {
        const float weight = next_weight, lse = next_lse;
        if (weight == 0.f) {
            look_ahead(row + step);
            if (lane == 0 && rank == 0 && a.loss) a.loss[row] = 0.f;
            continue;
        }
        const RowShape shape = row_shape(static_cast<const T *>(a.logits) + row * a.ld_logits, (int)a.vocab);
        int from, count;
        slice_of(shape.units, rank, log_cluster, from, count);
        const int b = n & 1;
        const uint32_t parity = n >> 1 & 1;
        const Entries known = entries_of(a, next, lse, lane);
        Entries en = known;
        const bool has_extra = rank == 0 && lane < shape.head + shape.tail;
        const int extra = has_extra ? extra_index<T>(shape, lane) : 0;
        const float x_extra = has_extra ? widen(next_extra) : -CUDART_INF_F;
        look_ahead(row + step);
        Running<false> run;
        run.add_one(x_extra, k);
        barrier_wait(shared_addr(&sh.joined[b]), parity, &sh.give_up);
        // the entries' logits: this CTA's slice is in the ring, extras are in the lanes
        float x[kTopEach];
        T *held[kTopEach];
        bool mine[kTopEach], twice = false;
#pragma unroll
        for (int e = 0; e < kTopEach; ++e) {
            x[e] = 0.f;
            held[e] = nullptr;
            mine[e] = false;
            if (!in_use(a, e)) continue;
            const int j = en.id[e], body = j - shape.head;
            const unsigned at = (unsigned)(body - from * kUnit<T>);  // beyond the slice also where it wraps
            const bool inside = j >= 0 && body >= 0 && at < (unsigned)(count * kUnit<T>);
            if (inside) {
                const unsigned unit = at / kUnit<T>;
                unsigned stage = slot + unit / Cut::kStageUnits;
                if (stage >= Cut::kStages) stage -= Cut::kStages;
                held[e] = reinterpret_cast<T *>(sh.stage[stage] + 16 * (unit % Cut::kStageUnits)) + at % kUnit<T>;
                x[e] = widen(*held[e]);
            }
            const bool at_ends = rank == 0 && j >= 0 && (body < 0 || body >= shape.units * kUnit<T>);
            mine[e] = inside || at_ends;
            if (__any_sync(0xffffffffu, at_ends)) {
                const float of_lane = __shfl_sync(0xffffffffu, x_extra, body < 0 ? j & 31 : (shape.head + body - shape.units * kUnit<T>) & 31);
                if (at_ends) x[e] = of_lane;
                twice |= any_twice(a, known);  // (extras carry no marks)
            }
        }
        __syncwarp();  // all have read before the first one marks
#pragma unroll
        for (int e = 0; e < kTopEach; ++e)
            if (in_use(a, e) && held[e] && !mark(held[e], x[e])) twice = true;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the marks come before the stages' next copies
        if (__any_sync(0xffffffffu, twice)) join_twice(known.id, known.p, en.own);
        const Stats none = {-CUDART_INF_F, 0.f, 0.f};
        Stats s = none;
        if (lane < Cut::kWarps) s = {sh.slots[b][lane].x, sh.slots[b][lane].y, 0.f};
        s = warp_join<false>(join2(s, run.stats(), k), k);
        float cross = 0.f;  // of the row, where the CTAs' shares have to be put together
        if (cluster > 1) {
            float distance = 0.f, share = 0.f;
            const float ref = s.top == -CUDART_INF_F ? 0.f : s.top;
            if (a.loss) {
#pragma unroll
                for (int e = 0; e < kTopEach; ++e)
                    if (in_use(a, e) && mine[e] && en.p[e] != 0.f) {
                        share += en.p[e];
                        distance = fmaf(en.p[e], x[e] - ref, distance);
                    }
                share = warp_sum(share);
                distance = warp_sum(distance);
            }
            const uint32_t bar = shared_addr(&sh.peered[b]);
            if (lane == 0) barrier_expect(bar, 16u * cluster);
            if (lane < cluster) send16(shared_addr(&sh.peer[b][rank]), bar, lane, s.top, s.sum, distance, share);
            barrier_wait(bar, parity, &sh.give_up);
            float4 q = make_float4(-CUDART_INF_F, 0.f, 0.f, 0.f);
            if (lane < cluster) q = sh.peer[b][lane];
            s = warp_join<false>({q.x, q.y, 0.f}, k);
            if (a.loss && rank == 0 && q.w != 0.f)
                cross = q.w * logf(s.sum) - a.scale * fmaf(q.w, (q.x == -CUDART_INF_F ? 0.f : q.x) - s.top, q.z);
        }
        const float per_e = per_e_of(a, en.mass, weight, s.sum);
        __syncwarp();  // all lanes have taken their logits from the ring, and read the statistics
        if (lane == 0) {
            sh.verdict[b] = {s.top, 0.f, per_e, 0.f, -1, -1};
            barrier_arrive(shared_addr(&sh.ready[b]));
        }
        const DistillOut o = distill_out(a, en, x, mine, weight, s.top, s.sum, k);  // while the others write
        add_terms(acc, weight, en, o, rank == 0 && lane == 0);
        if (a.loss && rank == 0) {
            float kl = o.kl;
            if (cluster > 1) {
                kl = cross;
#pragma unroll
                for (int e = 0; e < kTopEach; ++e)
                    if (en.p[e] != 0.f) kl = fmaf(en.p[e], en.logp[e], kl);
                if (en.bad) kl = CUDART_NAN_F;
            }
            kl = warp_sum(kl);
            if (lane == 0) a.loss[row] = kl;
        }
        if (en.bad && lane == 0 && rank == 0) record_bad_target(a.status, row);
        if (a.dlogits) {
            O *y = static_cast<O *>(a.dlogits) + row * a.ld_dlogits;
            if (has_extra) y[extra] = narrow<O>(per_e == 0.f ? 0.f : per_e * exp2_fast(k * (x_extra - s.top)));
            __syncwarp();  // (an extra may be an entry's)
            if (n >= 2) waiting[0].write(a);
            waiting[0] = waiting[1];
            waiting[1].row = y;
#pragma unroll
            for (int e = 0; e < kTopEach; ++e) {
                waiting[1].id[e] = mine[e] ? en.id[e] : -1;
                waiting[1].g[e] = o.g[e];
            }
        }
        slot += (unsigned)(count + Cut::kStageUnits - 1) / Cut::kStageUnits;
        if (slot >= Cut::kStages) slot -= Cut::kStages;
        ++n;
    }
    sum_lanes(acc);
    if (!a.dlogits || n == 0) return;
    if (!barrier_wait(shared_addr(&sh.done), 0, &sh.give_up)) return;
    if (n >= 2) waiting[0].write(a);
    waiting[1].write(a);
}

}  // namespace adama
