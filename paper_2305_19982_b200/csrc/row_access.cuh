// Rows of any alignment in pieces of eight consecutive elements, one piece to a lane: 16-byte accesses
// wherever memory allows them, whatever the row's pitch.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "stream_access.cuh"

namespace adama {

constexpr int kPiece = 8;  // elements of a piece: 16 bytes of bf16, 32 of fp32

__device__ __forceinline__ uint4 ld16(const void *p) {
    uint4 r;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

template <typename O>
__device__ __forceinline__ O narrowed(float y);
template <>
__device__ __forceinline__ float narrowed<float>(float y) { return y; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrowed<__nv_bfloat16>(float y) { return __float2bfloat16_rn(y); }

// A matrix's memory from its first element to past its last one: 16-byte loads that begin before a piece or
// end behind it stay inside.
struct Extent {
    uintptr_t begin, end;
};
template <typename T>
__device__ __forceinline__ Extent extent_of(const T *p, int64_t rows, int64_t cols, int64_t ld) {
    return {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p + (rows - 1) * ld + cols)};
}

// Words of 16-byte loads, moved down by `shift` words (0 to 3).
template <int N>
__device__ __forceinline__ void move_words(unsigned (&z)[N], int shift) {
    if (shift & 2) {
#pragma unroll
        for (int i = 0; i < N - 2; ++i) z[i] = z[i + 2];
    }
    if (shift & 1) {
#pragma unroll
        for (int i = 0; i < N - 1; ++i) z[i] = z[i + 1];
    }
}
template <int N>
__device__ __forceinline__ void load_words(unsigned (&z)[N], const unsigned char *p) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const uint4 u = ld16(p + 16 * i);
        z[4 * i] = u.x;
        z[4 * i + 1] = u.y;
        z[4 * i + 2] = u.z;
        z[4 * i + 3] = u.w;
    }
}
__device__ __forceinline__ void widen_words(const unsigned *z, float (&v)[kPiece], __nv_bfloat16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // bf16 -> fp32 is a 16-bit left shift
        v[2 * i] = __uint_as_float(z[i] << 16);
        v[2 * i + 1] = __uint_as_float(z[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen_words(const unsigned *z, float (&v)[kPiece], float) {
#pragma unroll
    for (int i = 0; i < kPiece; ++i) v[i] = __uint_as_float(z[i]);
}

// A piece on its way: loads are issued for all of a thread's pieces before the first one is looked at.  EVEN: all
// rows begin on 16-byte boundaries and are whole pieces long.  Otherwise the 16-byte units that a piece
// touches are loaded, one more than it is long, as far as they lie in the matrix.
template <typename T, bool EVEN>
struct Piece {
    static constexpr int kWords = kPiece * sizeof(T) / 4;
    unsigned z[kWords + (EVEN ? 0 : 4)];

    __device__ __forceinline__ void load(const T *p, int count, const Extent &all) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p), base = EVEN ? at : at & ~(uintptr_t)15;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(z) / 16); ++i) {
            const uintptr_t unit = base + 16 * i;
            const bool wanted = EVEN ? count != 0 : unit < at + count * sizeof(T) && unit >= all.begin && unit + 16 <= all.end;
            uint4 u = make_uint4(0, 0, 0, 0);
            if (wanted) u = ld16(reinterpret_cast<const void *>(unit));
            z[4 * i] = u.x;
            z[4 * i + 1] = u.y;
            z[4 * i + 2] = u.z;
            z[4 * i + 3] = u.w;
        }
    }
    // its elements as fp32, zeros from `count` on
    __device__ __forceinline__ void get(const T *p, int count, const Extent &all, float (&v)[kPiece]) const {
        if constexpr (EVEN) {
            widen_words(z, v, T());
        } else {
            const uintptr_t at = reinterpret_cast<uintptr_t>(p), base = at & ~(uintptr_t)15;
            unsigned y[kWords + 4];
#pragma unroll
            for (int i = 0; i < kWords + 4; ++i) y[i] = z[i];
            move_words(y, (int)(at - base) / 4);
            if (sizeof(T) == 2 && (at & 2)) {
#pragma unroll
                for (int i = 0; i < kWords; ++i) y[i] = __funnelshift_r(y[i], y[i + 1], 16);
            }
            widen_words(y, v, T());
            if (count != kPiece) {
#pragma unroll
                for (int i = 0; i < kPiece; ++i)
                    if (i >= count) v[i] = 0.f;
            }
            const uintptr_t end = (at + count * sizeof(T) + 15) & ~(uintptr_t)15;
            if (count != 0 && (base < all.begin || end > all.end)) {  // at the matrix's ends a unit lies outside in part
#pragma unroll
                for (int i = 0; i < kPiece; ++i) v[i] = i < count ? widen(p[i]) : 0.f;
            }
        }
    }
};

template <bool EVEN, typename T>
__device__ __forceinline__ void load_piece(const T *p, int count, const Extent &all, float (&v)[kPiece]) {
    Piece<T, EVEN> q;
    q.load(p, count, all);
    q.get(p, count, all, v);
}

// Whether rows of a matrix are even in that sense.
inline bool even_rows(const void *p, int64_t cols, int64_t ld, int size) {
    return aligned(p, 16) && cols % kPiece == 0 && ld * size % 16 == 0;
}

__device__ __forceinline__ void pack_words(const float (&v)[kPiece], unsigned (&w)[4], __nv_bfloat16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const unsigned *>(&p);
    }
}
__device__ __forceinline__ void pack_words(const float (&v)[kPiece], unsigned (&w)[8], float) {
#pragma unroll
    for (int i = 0; i < kPiece; ++i) w[i] = __float_as_uint(v[i]);
}

// Stores a run of pieces: `lanes` (a power of two) neighbouring lanes hold consecutive pieces, this one
// `count` elements that go to p (8, fewer at the row's end, 0 behind it).  All 32 lanes of a warp call it.
// Where p is not on a 16-byte boundary a lane stores the eight elements from the next boundary on, of which
// its neighbour has the last ones; only a run's ends are stored one by one.
template <bool EVEN, typename O>
__device__ __forceinline__ void store_run(O *p, const float (&v)[kPiece], int count, int lanes) {
    constexpr int kWords = kPiece * sizeof(O) / 4;
    unsigned w[kWords];
    pack_words(v, w, O());
    if constexpr (EVEN) {
        if (count != 0) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i)
                reinterpret_cast<uint4 *>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        }
        return;
    }
    const int past = (int)(reinterpret_cast<uintptr_t>(p) & 15);
    const int shift = past ? (16 - past) / (int)sizeof(O) : 0;  // elements before the boundary
    if (!__any_sync(0xffffffffu, shift != 0 && count > 0)) {
        if (count == kPiece) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i)
                reinterpret_cast<uint4 *>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (i < count) p[i] = narrowed<O>(v[i]);
        }
        return;
    }
    const int lane = threadIdx.x % 32, at = lane & (lanes - 1);
    const int next_count = __shfl_down_sync(0xffffffffu, count, 1);
    const bool whole = count == kPiece && (shift == 0 || (at != lanes - 1 && next_count >= shift));
    const bool before = __shfl_up_sync(0xffffffffu, whole, 1) && at != 0;  // the lane below has stored the first ones
    unsigned z[kWords + 4];
#pragma unroll
    for (int i = 0; i < kWords; ++i) z[i] = w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) z[kWords + i] = __shfl_down_sync(0xffffffffu, w[i], 1);
    if (whole) {
        move_words(z, shift * (int)sizeof(O) / 4);
        if (sizeof(O) == 2 && (shift & 1)) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) z[i] = __funnelshift_r(z[i], z[i + 1], 16);
        }
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i)
            reinterpret_cast<uint4 *>(p + shift)[i] = make_uint4(z[4 * i], z[4 * i + 1], z[4 * i + 2], z[4 * i + 3]);
    }
#pragma unroll
    for (int i = 0; i < kPiece; ++i)
        if (i < count && (i < shift ? !before : !whole)) p[i] = narrowed<O>(v[i]);
}

}  // namespace adama
