// Distillation from a teacher's top logits: the part of a row that its few entries make, for the kernels on rows
// of logits.  With z = s*x, q_j = exp(z_j - lse) the student's probabilities, and per entry i the teacher's
//     log p_i = s*t_i - lse_T   (lse_T given, or the log-sum over the row's entries: they then sum to 1),  P = sum p_i
//     kl = sum p_i (log p_i - log q_{j_i}),   dlogits_j = w*s*(P*q_j - sum over entries of j of p_i)
// All but the entries' own elements have the form that the kernels write for any loss, per_e * 2^(k*(x - top)).
// Rows that a warp holds are dealt with whole.  For longer ones a short kernel takes the teacher's side and the
// entries' logits ahead of the main one, which leaves each row's top and sum; a third one makes the loss terms and
// writes the entries' elements over, at 16 bytes an entry to L2 and back.  (4096 x 50257 bf16, 64 entries: 151 us.  When it took 157, the
// main kernel doing all of it gained nothing: 160 us with one warp for the entries between a row's statistics and its gradient, 156
// with all of them, but 24 rows of 32000 then took 12.3 instead of 10.3.)
#pragma once

#include "adama_device.cuh"
#include "logit_ring.cuh"

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
    // (the last entry again where there are no more: a load with a condition of its own waits for the one before it)
    const int64_t *ids = a.ids + row * a.ld_ids;
    const int64_t first = row * a.ld_teacher;
#pragma unroll
    for (int e = 0; e < kTopEach; ++e)
        if (in_use(a, e)) r.id[e] = ids[min(32 * e + lane, a.top - 1)];
    if (a.teacher_dtype == ADAMA_F32) {
#pragma unroll
        for (int e = 0; e < kTopEach; ++e)
            if (in_use(a, e)) r.t[e] = static_cast<const unsigned *>(a.teacher)[first + min(32 * e + lane, a.top - 1)];
    } else {
#pragma unroll
        for (int e = 0; e < kTopEach; ++e)
            if (in_use(a, e)) r.t[e] = static_cast<const unsigned short *>(a.teacher)[first + min(32 * e + lane, a.top - 1)];
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
    float own[kTopEach];   // sum of p over the entries of the same index
    float mass;            // P; NaN where an index lies outside the vocabulary
    float inner;           // this lane's share of sum p log p
    bool bad;              // there is such an index
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
    r.inner = 0.f;
#pragma unroll
    for (int e = 0; e < kTopEach; ++e) {
        r.p[e] = 0.f;
        if (in_use(a, e) && t[e] != -CUDART_INF_F) {
            const float logp = fmaf(a.scale, t[e] - ref, offset);
            r.p[e] = expf(logp);
            if (r.p[e] != 0.f) r.inner = fmaf(r.p[e], logp, r.inner);
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

// One entry's share of a row's loss terms, and the gradient of its element.
struct EntryTerms {
    float cross, held, g;
};
__device__ __forceinline__ EntryTerms entry_terms(float x, float p, float own, float mass, float scale, float unit, float top, float log_sum,
                                                  float inv, float k) {
    EntryTerms t;
    const float d = x - top, q = exp2_fast(k * d) * inv;
    // no mass: nothing to learn here either, and no NaN of the student's row (fmaxf leaves it out) in any sum
    t.held = mass == 0.f ? fmaxf(q, 0.f) : mass == mass ? q : mass;
    t.g = mass == 0.f ? 0.f : unit * fmaf(mass, q, -own);
    t.cross = p != 0.f ? p * (log_sum - scale * d) : 0.f;  // no probability, no loss, also where the student has none either
    if (mass != mass) t.cross = mass;
    return t;
}

// Every lane has added its share: the warp's sums, in all lanes.
__device__ __forceinline__ void sum_lanes(Sums &sums) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sums.v[i] += __shfl_xor_sync(0xffffffffu, sums.v[i], o);
}

}  // namespace adama
