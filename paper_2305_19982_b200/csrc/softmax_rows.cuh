// Softmax statistics of rows of logits, in registers: 16-byte units of fp32 or bf16 values, widened
// exactly, two values per instruction where sm_100a has the packed fp32 form.
#pragma once

#include <cuda_bf16.h>
#include <math.h>
#include <math_constants.h>

#include "stream_access.cuh"

namespace adama {

// Statistics of a set of logits, with k = s*log2(e): the largest one, the sum of 2^(k*(x - top)) and
// that of the same times k*(x - top).  The difference is formed first: a common offset of the logits,
// or the lowest value of their type as a mask, then costs neither precision nor range.  An empty
// set, or one of -inf alone, has top = -inf and sums of zero.
struct Stats {
    float top, sum, wsum;
};

__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// ---- two fp32 values in one register pair ------------------------------------------------------
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair(float lo, float hi) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split(Pair p, float &lo, float &hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p));
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// a unit from global memory; not a read-only load: a gradient may be written over the logits
__device__ __forceinline__ uint4 ld_unit(const uint4 *p) {
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
                 : "l"(p));
    return r;
}

__device__ __forceinline__ uint4 ld_unit_ro(const uint4 *p) {
    uint4 r;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
                 : "l"(p));
    return r;
}

// ---- 16-byte units -------------------------------------------------------------------------------
template <typename T>
constexpr int kUnit = 16 / sizeof(T);  // values in a unit

template <typename T>
__device__ __forceinline__ Pair unit_pair(const uint4 &u, int i);  // values 2i and 2i+1
template <>
__device__ __forceinline__ Pair unit_pair<float>(const uint4 &u, int i) {
    return i == 0 ? pair(__uint_as_float(u.x), __uint_as_float(u.y)) : pair(__uint_as_float(u.z), __uint_as_float(u.w));
}
template <>
__device__ __forceinline__ Pair unit_pair<__nv_bfloat16>(const uint4 &u, int i) {
    const unsigned w = i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w;
    return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));  // bf16 -> fp32 is a shift
}

// values 2i and 2i+1, less r: for bf16 one instruction each widens and subtracts
template <typename T>
__device__ __forceinline__ Pair unit_less(const uint4 &u, int i, float r);
template <>
__device__ __forceinline__ Pair unit_less<float>(const uint4 &u, int i, float r) {
    return add2(unit_pair<float>(u, i), pair(-r, -r));
}
template <>
__device__ __forceinline__ Pair unit_less<__nv_bfloat16>(const uint4 &u, int i, float r) {
    const unsigned w = i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w;
    float lo, hi;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tadd.rn.f32.bf16 %0, a, %3;\n\tadd.rn.f32.bf16 %1, b, %3;\n\t}"
        : "=f"(lo), "=f"(hi)
        : "r"(w), "f"(-r));
    return pair(lo, hi);
}

// a unit of -inf
template <typename T>
__device__ __forceinline__ uint4 nothing() {
    const unsigned w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    return make_uint4(w, w, w, w);
}

__device__ __forceinline__ float unit_max(const uint4 &u, float) {
    return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
}
__device__ __forceinline__ __nv_bfloat162 as_bf162(unsigned w) { return *reinterpret_cast<const __nv_bfloat162 *>(&w); }
__device__ __forceinline__ float unit_max(const uint4 &u, __nv_bfloat16) {
    const __nv_bfloat162 m = __hmax2(__hmax2(as_bf162(u.x), as_bf162(u.y)), __hmax2(as_bf162(u.z), as_bf162(u.w)));
    return fmaxf(__bfloat162float(m.x), __bfloat162float(m.y));
}

// One thread's running statistics.  ENT: wsum is kept as well.
template <bool ENT>
struct Running {
    float top = -INFINITY;
    Pair sum = 0, wsum = 0;

    __device__ __forceinline__ void raise(float t, float k) {
        if (t > top) {
            const float d = top == -CUDART_INF_F ? 0.f : k * (top - t), e = exp2_fast(d);
            if (ENT) wsum = e > 0.f ? mul2(fma2(sum, pair(d, d), wsum), pair(e, e)) : 0;
            sum = mul2(sum, pair(e, e));
            top = t;
        }
    }
    __device__ __forceinline__ float ref() const { return top == -CUDART_INF_F ? 0.f : top; }
    __device__ __forceinline__ void add_pair(Pair x_less_ref, Pair k2) {
        float d0, d1;
        split(mul2(x_less_ref, k2), d0, d1);
        const Pair e = pair(exp2_fast(d0), exp2_fast(d1));
        sum = add2(sum, e);
        if (ENT) wsum = fma2(e, pair(fmaxf(d0, -1e30f), fmaxf(d1, -1e30f)), wsum);  // -inf has e = 0
    }
    template <typename T, int N>
    __device__ __forceinline__ void add_units(const uint4 (&u)[N], float k) {
        float t = unit_max(u[0], T());
#pragma unroll
        for (int i = 1; i < N; ++i) t = fmaxf(t, unit_max(u[i], T()));
        raise(t, k);
        const float r = ref();
        const Pair k2 = pair(k, k);
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int q = 0; q < kUnit<T> / 2; ++q) add_pair(unit_less<T>(u[i], q, r), k2);
    }
    __device__ __forceinline__ void add_one(float x, float k) {
        raise(x, k);
        add_pair(pair(x - ref(), -CUDART_INF_F), pair(k, k));
    }
    __device__ __forceinline__ Stats stats() const {
        float a, b, c = 0.f, d = 0.f;
        split(sum, a, b);
        if (ENT) split(wsum, c, d);
        return {top, a + b, c + d};
    }
};

// s brought to a larger (or equal) top
__device__ __forceinline__ Stats raised(Stats s, float top, float k) {
    const float d = s.top == top ? 0.f : k * (s.top - top), e = exp2_fast(d);
    // an empty set has weight 0 and distance -inf: its product is left out
    return {top, s.sum * e, e > 0.f ? e * (s.wsum + s.sum * d) : 0.f};
}

// Statistics of the union over the 32 lanes of a warp, in every lane.
template <bool ENT>
__device__ __forceinline__ Stats warp_join(Stats s, float k) {
    float top;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(top) : "f"(s.top));
    s = raised(s, top, k);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s.sum += __shfl_xor_sync(0xffffffffu, s.sum, o);
        if (ENT) s.wsum += __shfl_xor_sync(0xffffffffu, s.wsum, o);
    }
    return s;
}

// Elements of a row before the first 16-byte boundary; the units behind them; the rest are extras too.
struct RowShape {
    int head, units, tail;
};
template <typename T>
__device__ __forceinline__ RowShape row_shape(const T *x, int vocab) {
    const int mis = (int)((reinterpret_cast<uintptr_t>(x) % 16) / sizeof(T));
    RowShape r;
    r.head = mis ? kUnit<T> - mis : 0;
    if (r.head > vocab) r.head = vocab;
    r.units = (vocab - r.head) / kUnit<T>;
    r.tail = vocab - r.head - r.units * kUnit<T>;
    return r;
}
// index of extra element i (i < head + tail)
template <typename T>
__device__ __forceinline__ int extra_index(const RowShape &r, int i) {
    return i < r.head ? i : r.head + r.units * kUnit<T> + (i - r.head);
}

}  // namespace adama
