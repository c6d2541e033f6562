// Rows of any alignment, eight elements ("a piece") to a thread and turn.  EVEN: a thread takes eight consecutive elements,
// or twice four where some of the matrices are fp32, so that a warp's accesses cover consecutive 8 or 16 bytes of each
// lane (fp32 in eights leaves half of every 32-byte sector to a second access); rows are whole eights or fours long
// and begin on boundaries of as many elements.  Otherwise threads
// take every width-th element: a warp's accesses then cover consecutive elements whatever the pitch, and
// cost no shifting of words (8192 rows of 1601 bf16, layer norm: 39 us with 16-byte loads shifted into place and stores
// traded between lanes, 24 so).
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "softmax_rows.cuh"

namespace adama {

constexpr int kPiece = 8;  // elements of a piece: 16 bytes of bf16, 32 of fp32

// Eight elements as fp32, two to a register pair.
struct Vec {
    Pair p[kPiece / 2];
};
__device__ __forceinline__ Vec zeros() { return {{0, 0, 0, 0}}; }
__device__ __forceinline__ float pair_sum(Pair p) {
    float a, b;
    split(p, a, b);
    return a + b;
}

// Elements that lie together in a piece of even rows whose matrices have elements of these sizes.
__host__ __device__ constexpr int together(size_t a, size_t b) { return a == 2 && b == 2 ? 8 : 4; }

// Columns of a thread: element i of its piece u, of threads `t` of a row's `width`; N elements lie together.  W: that
// width, known to the compiler (0: it is not), so that uneven rows' accesses need no address of their own each.
template <bool EVEN, int N, int W = 0>
struct Columns {
    static constexpr int kTogether = N, kParts = kPiece / N;
    int t, threads, dim;

    __device__ __forceinline__ int width() const { return W ? W : threads; }
    __device__ __forceinline__ int at(int u, int i) const {
        return EVEN ? (t + (u * kParts + i / N) * width()) * N + i % N : t + (u * kPiece + i) * width();
    }
    __device__ __forceinline__ bool has(int u, int i) const {  // (EVEN: the same for elements that lie together)
        return EVEN ? (t + (u * kParts + i / N) * width()) * N < dim : t < dim - (u * kPiece + i) * width();
    }
};

__device__ __forceinline__ Vec widened(const uint4 (&u)[1]) {  // bf16 -> fp32 is a 16-bit left shift
    const unsigned z[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
    Vec v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v.p[i] = pair(__uint_as_float(z[i] << 16), __uint_as_float(z[i] & 0xffff0000u));
    return v;
}
__device__ __forceinline__ Vec widened(const uint4 (&u)[2]) {
    Vec v;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        v.p[2 * h] = pair(__uint_as_float(u[h].x), __uint_as_float(u[h].y));
        v.p[2 * h + 1] = pair(__uint_as_float(u[h].z), __uint_as_float(u[h].w));
    }
    return v;
}

// A piece as it comes from memory, so that many can be on their way before the first one is looked at.
template <typename T, bool EVEN>
struct Piece {
    static constexpr int kUnits = kPiece * sizeof(T) / 16;
    uint4 even[EVEN ? kUnits : 1];
    T odd[EVEN ? 1 : kPiece];

    // row: the row's first element; zeros for columns that it does not have, and for none at all (`live` false)
    template <int N, int W>
    __device__ __forceinline__ void load(const T *row, const Columns<EVEN, N, W> &c, int u, bool live) {
        if constexpr (EVEN) {
#pragma unroll
            for (int i = 0; i < kUnits; ++i) even[i] = make_uint4(0, 0, 0, 0);
            if constexpr (N * sizeof(T) == 8) {
                uint2 q[2] = {make_uint2(0, 0), make_uint2(0, 0)};
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (live && c.has(u, N * i)) q[i] = *reinterpret_cast<const uint2 *>(row + c.at(u, N * i));
                even[0] = make_uint4(q[0].x, q[0].y, q[1].x, q[1].y);
            } else {
#pragma unroll
                for (int i = 0; i < kUnits; ++i)
                    if (live && c.has(u, kPiece / kUnits * i)) even[i] = *reinterpret_cast<const uint4 *>(row + c.at(u, kPiece / kUnits * i));
            }
        } else {
            const T *from = row + c.t;
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                odd[i] = narrow<T>(0.f);
                if (live && c.has(u, i)) odd[i] = from[(u * kPiece + i) * c.width()];
            }
        }
    }
    __device__ __forceinline__ Vec get() const {
        if constexpr (EVEN) {
            return widened(even);
        } else {
            Vec v;
#pragma unroll
            for (int i = 0; i < kPiece / 2; ++i) v.p[i] = pair(widen(odd[2 * i]), widen(odd[2 * i + 1]));
            return v;
        }
    }
};
template <typename T, bool EVEN, int N, int W>
__device__ __forceinline__ Vec load_piece(const T *row, const Columns<EVEN, N, W> &c, int u, bool live) {
    Piece<T, EVEN> q;
    q.load(row, c, u, live);
    return q.get();
}

__device__ __forceinline__ void pack_words(const Vec &v, uint4 (&w)[1]) {
    unsigned z[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        split(v.p[i], a, b);
        const __nv_bfloat162 q = __floats2bfloat162_rn(a, b);
        z[i] = *reinterpret_cast<const unsigned *>(&q);
    }
    w[0] = make_uint4(z[0], z[1], z[2], z[3]);
}
__device__ __forceinline__ void pack_words(const Vec &v, uint4 (&w)[2]) {
    float a[kPiece];
#pragma unroll
    for (int i = 0; i < 4; ++i) split(v.p[i], a[2 * i], a[2 * i + 1]);
#pragma unroll
    for (int h = 0; h < 2; ++h)
        w[h] = make_uint4(__float_as_uint(a[4 * h]), __float_as_uint(a[4 * h + 1]), __float_as_uint(a[4 * h + 2]), __float_as_uint(a[4 * h + 3]));
}
template <typename O, bool EVEN, int N, int W>
__device__ __forceinline__ void store_piece(O *row, const Columns<EVEN, N, W> &c, int u, bool live, const Vec &v) {
    if constexpr (EVEN) {
        constexpr int kUnits = kPiece * sizeof(O) / 16;
        uint4 w[kUnits];
        pack_words(v, w);
        if constexpr (N * sizeof(O) == 8) {
            if (live && c.has(u, 0)) *reinterpret_cast<uint2 *>(row + c.at(u, 0)) = make_uint2(w[0].x, w[0].y);
            if (live && c.has(u, N)) *reinterpret_cast<uint2 *>(row + c.at(u, N)) = make_uint2(w[0].z, w[0].w);
        } else {
#pragma unroll
            for (int i = 0; i < kUnits; ++i)
                if (live && c.has(u, kPiece / kUnits * i)) *reinterpret_cast<uint4 *>(row + c.at(u, kPiece / kUnits * i)) = w[i];
        }
    } else {
        O *to = row + c.t;
#pragma unroll
        for (int i = 0; i < kPiece / 2; ++i) {
            float a, b;
            split(v.p[i], a, b);
            if (live && c.has(u, 2 * i)) to[(u * kPiece + 2 * i) * c.width()] = narrow<O>(a);
            if (live && c.has(u, 2 * i + 1)) to[(u * kPiece + 2 * i + 1) * c.width()] = narrow<O>(b);
        }
    }
}

// Whether rows of a matrix are even in that sense, n elements lying together.
inline bool even_rows(const void *p, int64_t cols, int64_t ld, int size, int n) {
    return aligned(p, n * size) && cols % n == 0 && ld % n == 0;
}

// ---- pieces ahead ----------------------------------------------------------------------------------
// Asynchronous copies to shared memory that the thread itself waits for: no other one reads them.
__device__ __forceinline__ void copy16(uint32_t to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t to, const void *from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, const void *from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {  // for all but the last N groups
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Thread `t` of `threads` that share a slot of kBytes * threads: its piece of a row.  Two-byte elements of uneven rows
// cannot come that way, and are loaded when they are wanted.
template <typename T, bool EVEN>
struct Slot {
    static constexpr bool kCopied = EVEN || sizeof(T) == 4;
    static constexpr int kBytes = kCopied ? kPiece * (int)sizeof(T) : 0;
    static constexpr int kUnits = kPiece * sizeof(T) / 16;

    template <int N, int W>
    static __device__ __forceinline__ void send_for(unsigned char *slot, const T *row, const Columns<EVEN, N, W> &c, int u, int t, int threads) {
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(slot);
        if constexpr (EVEN && N * sizeof(T) == 8) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (c.has(u, N * i)) copy8(to + (threads * i + t) * 8, row + c.at(u, N * i));
        } else if constexpr (EVEN) {
#pragma unroll
            for (int i = 0; i < kUnits; ++i)
                if (c.has(u, kPiece / kUnits * i)) copy16(to + (threads * i + t) * 16, row + c.at(u, kPiece / kUnits * i));
        } else if constexpr (kCopied) {
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (c.has(u, i)) copy4(to + (threads * i + t) * 4, row + c.at(u, i));
        }
    }
    // Zeros where nothing will be sent to, so that get need not ask which columns there are.
    template <int N, int W>
    static __device__ __forceinline__ void clear(unsigned char *slot, const Columns<EVEN, N, W> &c, int u, int t, int threads) {
        static_assert(EVEN, "uneven rows are not cleared");
        constexpr int kEach = N * sizeof(T) == 8 ? 2 : kUnits, kLen = kBytes / kEach;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (!c.has(u, kPiece / kEach * i)) {
#pragma unroll
                for (int q = 0; q < kLen / 4; ++q) reinterpret_cast<unsigned *>(slot)[(threads * i + t) * (kLen / 4) + q] = 0;
            }
    }
    template <int N, int W>
    static __device__ __forceinline__ Vec get(const unsigned char *slot, const T *row, const Columns<EVEN, N, W> &c, int u, int t, int threads) {
        if constexpr (EVEN) {
            uint4 w[kUnits];
            if constexpr (N * sizeof(T) == 8) {
                const uint2 p = reinterpret_cast<const uint2 *>(slot)[t], q = reinterpret_cast<const uint2 *>(slot)[threads + t];
                w[0] = make_uint4(p.x, p.y, q.x, q.y);
            } else {
#pragma unroll
                for (int i = 0; i < kUnits; ++i) w[i] = reinterpret_cast<const uint4 *>(slot)[threads * i + t];
            }
            return widened(w);
        } else if constexpr (kCopied) {
            Vec v;
            const float *f = reinterpret_cast<const float *>(slot) + t;
#pragma unroll
            for (int i = 0; i < kPiece / 2; ++i) v.p[i] = pair(f[2 * i * threads], f[(2 * i + 1) * threads]);
            return v;
        } else {
            return load_piece(row, c, u, true);
        }
    }
};

}  // namespace adama
