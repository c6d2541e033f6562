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

// A lane's entries: 32*e + lane, as the row has them.  id -1: none, -2: outside the vocabulary.
struct RawEntries {
    int id[kTopEach];
    float t[kTopEach];
};
// Whether a warp has entries at 32*e: most rows have fewer than 128, and the warp that deals with them works alone.
__device__ __forceinline__ bool in_use(const DistillArgs &a, int e) { return e == 0 || 32 * e < a.top; }

__device__ __forceinline__ RawEntries load_entries(const DistillArgs &a, int64_t row, int lane) {
    RawEntries r;
    const int64_t *ids = a.ids + row * a.ld_ids + lane;
    const int64_t at = row * a.ld_teacher + lane;
#pragma unroll
    for (int e = 0; e < kTopEach; ++e) {
        r.id[e] = -1;
        r.t[e] = -CUDART_INF_F;
        if (in_use(a, e) && 32 * e + lane < a.top) {
            const int64_t id = ids[32 * e];
            r.id[e] = id < 0 ? -1 : id < a.vocab ? (int)id : -2;
            r.t[e] = a.teacher_dtype == ADAMA_F32 ? static_cast<const float *>(a.teacher)[at + 32 * e]
                                                  : widen(static_cast<const __nv_bfloat16 *>(a.teacher)[at + 32 * e]);
        }
    }
    return r;
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
    bool bad;
};
__device__ __forceinline__ Entries entries_of(const DistillArgs &a, const RawEntries &raw, float lse) {
    Entries r;
    bool bad = false;
    float top = -CUDART_INF_F;
#pragma unroll
    for (int e = 0; e < kTopEach; ++e) {
        r.id[e] = raw.id[e] < 0 ? -1 : raw.id[e];
        r.p[e] = r.logp[e] = 0.f;
        if (in_use(a, e)) {
            bad |= raw.id[e] == -2;
            if (r.id[e] >= 0) top = fmaxf(top, raw.t[e] != raw.t[e] ? CUDART_INF_F : raw.t[e]);  // a NaN shows below
        }
    }
    r.bad = __any_sync(0xffffffffu, bad);
    float offset = -lse, ref = 0.f;  // log p = s*(t - ref) + offset
    if (!a.teacher_lse) {
        ref = warp_max(top);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < kTopEach; ++e)
            if (in_use(a, e) && r.id[e] >= 0 && ref != -CUDART_INF_F) sum += expf(a.scale * (raw.t[e] - ref));
        offset = -logf(warp_sum(sum));
    }
    float mass = 0.f;
#pragma unroll
    for (int e = 0; e < kTopEach; ++e) {
        if (in_use(a, e) && r.id[e] >= 0 && raw.t[e] != -CUDART_INF_F) {
            r.logp[e] = fmaf(a.scale, raw.t[e] - ref, offset);
            r.p[e] = expf(r.logp[e]);
        }
        mass += r.p[e];
        r.own[e] = r.p[e];
    }
    r.mass = warp_sum(mass);
    if (r.bad) r.mass = CUDART_NAN_F;
    // The same index twice: rare, but its element has one gradient.  First whether there is any.
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
    if (__any_sync(0xffffffffu, twice)) {
#pragma unroll
        for (int e = 0; e < kTopEach; ++e) r.own[e] = 0.f;
#pragma unroll 1
        for (int l = 0; l < 32; ++l)
#pragma unroll
            for (int f = 0; f < kTopEach; ++f) {
                const int id = __shfl_sync(0xffffffffu, r.id[f], l);
                const float p = __shfl_sync(0xffffffffu, r.p[f], l);
#pragma unroll
                for (int e = 0; e < kTopEach; ++e)
                    if (r.id[e] == id) r.own[e] += p;
            }
    }
    return r;
}

// What all but the entries' elements of a row's gradient are made of.
__device__ __forceinline__ float per_e_of(const DistillArgs &a, float mass, float weight, float sum) {
    return mass == 0.f ? 0.f : weight * a.scale * mass / sum;  // no entry: nothing to learn, whatever the logits
}

// A row's loss terms; g: the gradient of the entries' elements.
struct DistillOut {
    float kl, cross, held;  // held: the student's mass on the entries
    float g[kTopEach];
};
__device__ __forceinline__ DistillOut distill_out(const DistillArgs &a, const Entries &en, const float (&x)[kTopEach], float weight,
                                                  float top, float sum, float k) {
    DistillOut o;
    const float log_sum = logf(sum), unit = weight * a.scale, inv = 1.f / sum;
    float kl = 0.f, cross = 0.f, held = 0.f;
#pragma unroll
    for (int e = 0; e < kTopEach; ++e)
        if (in_use(a, e)) {
            const float d = x[e] - top, logq = fmaf(a.scale, d, -log_sum);
            const float q = exp2_fast(k * d) * inv;
            o.g[e] = en.bad ? CUDART_NAN_F : unit * fmaf(en.mass, q, -en.own[e]);
            if (en.id[e] >= 0) held += q;
            if (en.p[e] != 0.f) {  // no probability, no loss, also where the student has none either
                kl = fmaf(en.p[e], en.logp[e] - logq, kl);
                cross = fmaf(-en.p[e], logq, cross);
            }
        }
    o.kl = warp_sum(kl);
    o.cross = warp_sum(cross);
    o.held = warp_sum(held);
    if (en.bad) o.kl = o.cross = o.held = CUDART_NAN_F;
    return o;
}

__device__ __forceinline__ void add_terms(Sums &sums, const DistillArgs &a, float weight, const Entries &en, const DistillOut &o) {
    sums.add(weight, o.kl, o.cross, o.held, en.mass);
}

// ---- the warp between a row's statistics and its gradient ----------------------------------------

// Elements of a row that wait to be written over.
struct Patches {
    int64_t row;
    int id[kTopEach];  // -1: none, or another CTA's
    float g[kTopEach];
};
template <typename O>
__device__ __forceinline__ void write_patches(const DistillArgs &a, const Patches &p) {
    O *y = static_cast<O *>(a.dlogits) + p.row * a.ld_dlogits;
#pragma unroll
    for (int e = 0; e < kTopEach; ++e)
        if (in_use(a, e) && p.id[e] >= 0) y[p.id[e]] = narrow<O>(p.g[e]);
}

// In the ring's warp of its own: joins, loss terms, verdicts.  The working warps have written row n-2 when they
// have all given their statistics of row n: then the entries' elements of row n-2 are written over, those of
// the last two rows when the working warps have come to their end.
template <typename T, typename O, typename Cut>
__device__ __forceinline__ void distill_verdicts(const DistillArgs &a, float k, RingShared<Cut> &sh, int lane, int rank, int log_cluster,
                                                 int64_t first, int64_t step, Sums &acc) {
    const int cluster = 1 << log_cluster;
    uint32_t n = 0;  // live rows
    Patches waiting[2];
    // a row's weight is loaded two rows ahead, its entries one: loads that nobody waits for
    float after_weight = 0.f, next_weight = 0.f, next_lse = 0.f;
    RawEntries next = {};
    const auto look_ahead = [&](int64_t row) {
        next_weight = after_weight;
        after_weight = row + step < a.rows ? a.weights[row + step] : 0.f;
        if (next_weight != 0.f) {
            next = load_entries(a, row, lane);
            if (a.teacher_lse) next_lse = a.teacher_lse[row];
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
        const RawEntries raw = next;
        const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
        const RowShape shape = row_shape(x, (int)a.vocab);
        int from, count;
        slice_of(shape.units, rank, log_cluster, from, count);
        const int b = n & 1;
        const uint32_t parity = n >> 1 & 1;
        // the gradient may replace the logits: what is read here travels with this CTA's message or verdict, before
        // which nobody writes
        const int begin = shape.head + from * kUnit<T>, end = shape.head + (from + count) * kUnit<T>;
        const int body_end = shape.head + shape.units * kUnit<T>;
        float x_at[kTopEach];
        bool mine[kTopEach];
#pragma unroll
        for (int e = 0; e < kTopEach; ++e) {
            const int j = raw.id[e];
            mine[e] = j >= 0 && ((j >= begin && j < end) || (rank == 0 && (j < shape.head || j >= body_end)));
            x_at[e] = 0.f;
            if (in_use(a, e) && j >= 0 && (rank == 0 || mine[e])) x_at[e] = widen(x[j]);
        }
        const bool has_extra = rank == 0 && lane < shape.head + shape.tail;
        const int extra = has_extra ? extra_index<T>(shape, lane) : 0;
        const float x_extra = has_extra ? widen(x[extra]) : -CUDART_INF_F;
        look_ahead(row + step);
        const Entries en = entries_of(a, raw, lse);
        Running<false> run;
        run.add_one(x_extra, k);
        float seen = x_at[0];  // of all that this warp has read
#pragma unroll
        for (int e = 1; e < kTopEach; ++e) seen = fmaxf(seen, x_at[e]);
        seen = warp_max(seen);
        barrier_wait(shared_addr(&sh.joined[b]), parity, &sh.give_up);
        const Stats none = {-CUDART_INF_F, 0.f, 0.f};
        Stats s = none;
        if (lane < Cut::kWarps) s = {sh.slots[b][lane].x, sh.slots[b][lane].y, 0.f};
        s = warp_join<false>(join2(s, run.stats(), k), k);
        if (cluster > 1) {
            const uint32_t bar = shared_addr(&sh.peered[b]);
            if (lane == 0) barrier_expect(bar, 16u * cluster);
            if (lane < cluster) send16(shared_addr(&sh.peer[b][rank]), bar, lane, s.top, s.sum, seen, 0.f);
            barrier_wait(bar, parity, &sh.give_up);
            float4 q = make_float4(-CUDART_INF_F, 0.f, 0.f, 0.f);
            if (lane < cluster) q = sh.peer[b][lane];
            s = warp_join<false>({q.x, q.y, 0.f}, k);
        }
        const float per_e = per_e_of(a, en.mass, weight, s.sum);
        __syncwarp();  // all lanes have read their logits, which the verdict's readers may overwrite
        if (lane == 0) {
            sh.verdict[b] = {s.top, 0.f, per_e, seen, -1, -1};
            barrier_arrive(shared_addr(&sh.ready[b]));
        }
        const DistillOut o = distill_out(a, en, x_at, weight, s.top, s.sum, k);  // while the others write
        if (lane == 0 && rank == 0) {
            add_terms(acc, a, weight, en, o);
            if (a.loss) a.loss[row] = o.kl;
            if (en.bad) record_bad_target(a.status, row);
        }
        if (a.dlogits) {
            if (has_extra) {
                O *y = static_cast<O *>(a.dlogits) + row * a.ld_dlogits;
                y[extra] = narrow<O>(per_e == 0.f ? 0.f : per_e * exp2_fast(k * (x_extra - s.top)));
            }
            __syncwarp();  // (an extra may be an entry's)
            if (n >= 2) write_patches<O>(a, waiting[0]);
            waiting[0] = waiting[1];
            waiting[1].row = row;
#pragma unroll
            for (int e = 0; e < kTopEach; ++e) {
                waiting[1].id[e] = mine[e] ? raw.id[e] : -1;
                waiting[1].g[e] = o.g[e];
            }
        }
        ++n;
    }
    if (!a.dlogits || n == 0) return;
    if (!barrier_wait(shared_addr(&sh.done), 0, &sh.give_up)) return;
    if (n >= 2) write_patches<O>(a, waiting[0]);
    write_patches<O>(a, waiting[1]);
}

}  // namespace adama
