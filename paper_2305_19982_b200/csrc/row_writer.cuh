// The gradient of a row of logits, written beside the logits' 16-byte units whatever its own alignment.
#pragma once

#include "softmax_rows.cuh"
#include "tensor_table.cuh"

namespace adama {

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

}  // namespace adama
