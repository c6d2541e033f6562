// Rows of any alignment, eight elements ("a piece") to a thread and turn.  EVEN: rows begin on 16-byte boundaries and
// are whole pieces long; a thread takes eight consecutive elements with 16-byte accesses.  Otherwise threads
// take every width-th element: a warp's accesses then cover consecutive elements whatever the pitch, and
// cost no shifting of words (8192 rows of 1601 bf16, layer norm: 39 us with 16-byte loads shifted into place and stores
// traded between lanes, @ODD@ so).
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "stream_access.cuh"

namespace adama {

constexpr int kPiece = 8;  // elements of a piece: 16 bytes of bf16, 32 of fp32

template <typename O>
__device__ __forceinline__ O narrowed(float y);
template <>
__device__ __forceinline__ float narrowed<float>(float y) { return y; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrowed<__nv_bfloat16>(float y) { return __float2bfloat16_rn(y); }

// Columns of a thread: element i of its piece u, of threads `t` of `width` that share a row.
template <bool EVEN>
struct Columns {
    int t, width, dim;

    __device__ __forceinline__ int at(int u, int i) const { return EVEN ? (t + u * width) * kPiece + i : t + (u * kPiece + i) * width; }
    __device__ __forceinline__ bool has(int u, int i) const { return at(u, i) < dim; }  // (EVEN: the same for all i)
};

__device__ __forceinline__ void widen_words(const uint4 (&u)[1], float (&v)[kPiece]) {  // bf16 -> fp32 is a 16-bit left shift
    const unsigned z[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(z[i] << 16);
        v[2 * i + 1] = __uint_as_float(z[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen_words(const uint4 (&u)[2], float (&v)[kPiece]) {
    v[0] = __uint_as_float(u[0].x); v[1] = __uint_as_float(u[0].y); v[2] = __uint_as_float(u[0].z); v[3] = __uint_as_float(u[0].w);
    v[4] = __uint_as_float(u[1].x); v[5] = __uint_as_float(u[1].y); v[6] = __uint_as_float(u[1].z); v[7] = __uint_as_float(u[1].w);
}

// A piece as it comes from memory, so that many can be on their way before the first one is looked at.
template <typename T, bool EVEN>
struct Piece {
    static constexpr int kUnits = kPiece * sizeof(T) / 16;
    uint4 even[EVEN ? kUnits : 1];
    T odd[EVEN ? 1 : kPiece];

    // row: the row's first element; zeros for columns that it does not have, and for none at all (`live` false)
    __device__ __forceinline__ void load(const T *row, const Columns<EVEN> &c, int u, bool live) {
        if constexpr (EVEN) {
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                even[i] = make_uint4(0, 0, 0, 0);
                if (live && c.has(u, 0)) even[i] = reinterpret_cast<const uint4 *>(row + c.at(u, 0))[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                odd[i] = narrowed<T>(0.f);
                if (live && c.has(u, i)) odd[i] = row[c.at(u, i)];
            }
        }
    }
    __device__ __forceinline__ void get(float (&v)[kPiece]) const {
        if constexpr (EVEN) {
            widen_words(even, v);
        } else {
#pragma unroll
            for (int i = 0; i < kPiece; ++i) v[i] = widen(odd[i]);
        }
    }
};
template <typename T, bool EVEN>
__device__ __forceinline__ void load_piece(const T *row, const Columns<EVEN> &c, int u, bool live, float (&v)[kPiece]) {
    Piece<T, EVEN> q;
    q.load(row, c, u, live);
    q.get(v);
}

__device__ __forceinline__ void pack_words(const float (&v)[kPiece], uint4 (&w)[1]) {
    unsigned z[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        z[i] = *reinterpret_cast<const unsigned *>(&p);
    }
    w[0] = make_uint4(z[0], z[1], z[2], z[3]);
}
__device__ __forceinline__ void pack_words(const float (&v)[kPiece], uint4 (&w)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
        w[h] = make_uint4(__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]), __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3]));
}
template <typename O, bool EVEN>
__device__ __forceinline__ void store_piece(O *row, const Columns<EVEN> &c, int u, bool live, const float (&v)[kPiece]) {
    if (!live) return;
    if constexpr (EVEN) {
        uint4 w[kPiece * sizeof(O) / 16];
        pack_words(v, w);
        if (c.has(u, 0)) {
#pragma unroll
            for (int i = 0; i < (int)(kPiece * sizeof(O) / 16); ++i) reinterpret_cast<uint4 *>(row + c.at(u, 0))[i] = w[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPiece; ++i)
            if (c.has(u, i)) row[c.at(u, i)] = narrowed<O>(v[i]);
    }
}

// Whether rows of a matrix are even in that sense.
inline bool even_rows(const void *p, int64_t cols, int64_t ld, int size) {
    return aligned(p, 16) && cols % kPiece == 0 && ld * size % 16 == 0;
}

// ---- rows ahead -----------------------------------------------------------------------------------
// A thread's own pieces of the next rows on their way to shared memory (asynchronous copies that the thread itself waits
// for: no other one reads them), or, of uneven rows, of the next row to registers.
__device__ __forceinline__ void copy16(uint32_t to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {  // for all but the last N groups
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

}  // namespace adama
