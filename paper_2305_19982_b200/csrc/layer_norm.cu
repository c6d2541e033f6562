// Layer norm and its backward pass.  Over the D elements of a row:
//     mean = sum x / D,  var = sum (x - mean)^2 / D,  rstd = 1/sqrt(var + eps),  xhat = (x - mean)*rstd
//     y = xhat*weight + bias
// and, with g = dy*weight, the sums over a row s1 = sum g, s2 = sum g*xhat:
//     dx = rstd*(g - s1/D - xhat*s2/D),   dweight = sum over rows of dy*xhat,   dbias = the same of dy
// A row is read once and held in registers; the variance is taken of x - mean, so that a common offset costs
// no precision.  In the backward pass a thread keeps its columns for all rows of its block, with their two sums
// in registers; the blocks' sums go to the workspace, and a second, short kernel adds them in the blocks' order
// and writes the parameters' gradients or folds them into their moments (m += a*g, v += b*g^2: the sum over
// rows is complete before it is squared).  Nothing depends on scheduling.  Bound by HBM.
#include "adama_device.cuh"
#include "chained.cuh"
#include "row_access.cuh"
#include "softmax_rows.cuh"
#include "tensor_table.cuh"

namespace adama {
namespace {

// ---- threads that share a row -------------------------------------------------------------------
// Up to 32 lanes of a warp (a power of two), or some warps of a block.

__device__ __forceinline__ float lanes_sum(float x, int lanes) {
    for (int o = lanes / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
__device__ __forceinline__ float pair_sum(Pair p) {
    float a, b;
    split(p, a, b);
    return a + b;
}

// Warps of a block that share rows: `warps` to a row, several such groups side by side.
struct Group {
    int warps, index, count, t;

    __device__ __forceinline__ explicit Group(int w)
        : warps(w), index((int)threadIdx.x / 32 / w), count((int)blockDim.x / 32 / w), t((int)threadIdx.x - index * 32 * w) {}
    __device__ __forceinline__ void sync() const {
        if (warps == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + index), "r"(32 * warps) : "memory");
    }
    // The sum of x over the group, in every thread.  `slots`: one for each warp of the block, used again no sooner than
    // behind another sync of the group.
    __device__ __forceinline__ float sum(float x, float *slots) const {
        x = lanes_sum(x, 32);
        if (warps == 1) return x;
        if (threadIdx.x % 32 == 0) slots[threadIdx.x / 32] = x;
        sync();
        x = 0.f;
        for (int i = 0; i < warps; ++i) x += slots[index * warps + i];
        return x;
    }
};

constexpr int kGroupWarps = 16;  // of a block, at most
constexpr int kAhead = 3;        // rows of a thread on their way, of even ones

// A row's elements as fp32, and its distances from the mean.
template <bool EVEN>
__device__ __forceinline__ float sum_of(const float (&v)[kPiece]) {
    Pair s = 0;
#pragma unroll
    for (int i = 0; i < kPiece; i += 2) s = add2(s, pair(v[i], v[i + 1]));
    return pair_sum(s);
}
template <bool EVEN>
__device__ __forceinline__ float centre(float (&v)[kPiece], const Columns<EVEN> &c, int u, float mean) {
#pragma unroll
    for (int i = 0; i < kPiece; ++i)
        if (!c.has(u, i)) v[i] = mean;  // columns that the row does not have lie at no distance
    Pair s = 0;
#pragma unroll
    for (int i = 0; i < kPiece; i += 2) {
        const Pair d = add2(pair(v[i], v[i + 1]), pair(-mean, -mean));
        s = fma2(d, d, s);
        split(d, v[i], v[i + 1]);
    }
    return pair_sum(s);
}
__device__ __forceinline__ void scale_shift(float (&v)[kPiece], float rstd, const float (&w)[kPiece], const float (&b)[kPiece]) {
#pragma unroll
    for (int i = 0; i < kPiece; i += 2)
        split(fma2(mul2(pair(v[i], v[i + 1]), pair(rstd, rstd)), pair(w[i], w[i + 1]), pair(b[i], b[i + 1])), v[i], v[i + 1]);
}

// ---- forward -------------------------------------------------------------------------------------

// Rows of up to 256 elements: `lanes` lanes to a row, one piece to a lane.
constexpr int kShortThreads = 128;

template <typename T, typename O, bool EVEN>
__global__ void __launch_bounds__(kShortThreads)
layer_norm_short_kernel(const NormArgs a, int lanes) {
    const Columns<EVEN> c = {(int)threadIdx.x % lanes, lanes, a.dim};
    const int64_t row = (int64_t)blockIdx.x * (kShortThreads / lanes) + threadIdx.x / lanes;
    const bool live = row < a.rows;
    float v[kPiece], w[kPiece], b[kPiece];
    Piece<T, EVEN> raw;
    Piece<float, EVEN> raw_w, raw_b;
    raw.load(static_cast<const T *>(a.x) + (live ? row : 0) * a.ld_x, c, 0, live);
    raw_w.load(a.weight, c, 0, live);
    raw_b.load(a.bias, c, 0, live && a.bias);
    raw.get(v);
    const float mean = lanes_sum(sum_of<EVEN>(v), lanes) / (float)a.dim;  // (a product with 1/D would move the mean of equal values)
    const float rstd = 1.f / sqrtf(lanes_sum(centre(v, c, 0, mean), lanes) / (float)a.dim + a.eps);
    if (c.t == 0 && live) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    raw_w.get(w);
    raw_b.get(b);
    scale_shift(v, rstd, w, b);
    store_piece(static_cast<O *>(a.y) + (live ? row : 0) * a.ld_y, c, 0, live, v);
}

// Longer rows: a group of warps walks rows, U pieces to a thread, weight and bias in registers, the next rows on their
// way.  (One row to a block that ends with it: @FWD@.)
template <typename T, typename O, int U, bool EVEN>
__global__ void __launch_bounds__(32 * kGroupWarps)
layer_norm_kernel(const NormArgs a, int warps) {
    extern __shared__ uint4 ahead[];  // [rows ahead][U][units of a piece][threads]
    __shared__ float slots[2][kGroupWarps];
    constexpr int kUnits = Piece<T, true>::kUnits;
    const Group group(warps);
    const Columns<EVEN> c = {group.t, 32 * warps, a.dim};
    const T *x0 = static_cast<const T *>(a.x);
    const int64_t step = (int64_t)gridDim.x * group.count;
    int64_t row = (int64_t)blockIdx.x * group.count + group.index;
    const auto slot = [&](int stage, int u, int i) { return ahead + ((stage * U + u) * kUnits + i) * blockDim.x + threadIdx.x; };
    const auto send_for = [&](int64_t r, int stage) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r < a.rows && c.has(u, 0)) {
#pragma unroll
                for (int i = 0; i < kUnits; ++i)
                    copy16((uint32_t)__cvta_generic_to_shared(slot(stage, u, i)), reinterpret_cast<const uint4 *>(x0 + r * a.ld_x + c.at(u, 0)) + i);
            }
        copies_end_group();
    };
    Piece<T, EVEN> next[U];
    if constexpr (EVEN) {
        for (int i = 0; i < kAhead; ++i) send_for(row + i * step, i);
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) next[u].load(x0 + (row < a.rows ? row : 0) * a.ld_x, c, u, row < a.rows);
    }
    float w[U][kPiece], b[U][kPiece];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        load_piece(a.weight, c, u, true, w[u]);
        load_piece(a.bias, c, u, a.bias != nullptr, b[u]);
    }
    for (int stage = 0; row < a.rows; row += step, stage = stage + 1 == kAhead ? 0 : stage + 1) {
        float v[U][kPiece], s = 0.f;
        if constexpr (EVEN) {
            copies_wait<kAhead - 1>();
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c.has(u, 0)) {
#pragma unroll
                    for (int i = 0; i < kUnits; ++i) next[u].even[i] = *slot(stage, u, i);
                } else {
#pragma unroll
                    for (int i = 0; i < kUnits; ++i) next[u].even[i] = make_uint4(0, 0, 0, 0);
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            next[u].get(v[u]);
            s += sum_of<EVEN>(v[u]);
        }
        if constexpr (!EVEN) {
            const int64_t r = row + step;
#pragma unroll
            for (int u = 0; u < U; ++u) next[u].load(x0 + (r < a.rows ? r : 0) * a.ld_x, c, u, r < a.rows);
        }
        const float mean = group.sum(s, slots[0]) / (float)a.dim;
        if constexpr (EVEN) send_for(row + kAhead * step, stage);  // what was there has been summed up
        s = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) s += centre(v[u], c, u, mean);
        const float rstd = 1.f / sqrtf(group.sum(s, slots[1]) / (float)a.dim + a.eps);
        if (c.t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        O *y = static_cast<O *>(a.y) + row * a.ld_y;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            scale_shift(v[u], rstd, w[u], b[u]);
            store_piece(y, c, u, true, v[u]);
        }
    }
}

// Rows that no group holds in registers: read three times, from L2 if they stay there.
constexpr int kLongThreads = 512;

template <typename T, typename O>
__global__ void __launch_bounds__(kLongThreads)
layer_norm_long_kernel(const NormArgs a) {
    __shared__ float slots[2][kGroupWarps];
    const Group group(kGroupWarps);
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
    float s = 0.f;
    for (int c = threadIdx.x; c < a.dim; c += kLongThreads) s += widen(x[c]);
    const float mean = group.sum(s, slots[0]) / (float)a.dim;
    s = 0.f;
    for (int c = threadIdx.x; c < a.dim; c += kLongThreads) {
        const float d = widen(x[c]) - mean;
        s = fmaf(d, d, s);
    }
    const float rstd = 1.f / sqrtf(group.sum(s, slots[1]) / (float)a.dim + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    O *y = static_cast<O *>(a.y) + row * a.ld_y;
    for (int c = threadIdx.x; c < a.dim; c += kLongThreads)
        y[c] = narrowed<O>(fmaf((widen(x[c]) - mean) * rstd, a.weight[c], a.bias ? a.bias[c] : 0.f));
}

// ---- backward ------------------------------------------------------------------------------------

// A block's sums in the workspace: dweight, then dbias, each padded to whole pieces.
__host__ __device__ inline int64_t padded(int dim) { return ((int64_t)dim + kPiece - 1) / kPiece * kPiece; }

// Sums over rows, of a thread's columns.
struct PieceSums {
    Pair dw[kPiece / 2], db[kPiece / 2];
};
__device__ __forceinline__ Pair xhat_of(float x0, float x1, float mean, float rstd) {
    return mul2(add2(pair(x0, x1), pair(-mean, -mean)), pair(rstd, rstd));
}
// A piece's part in its columns' sums and in its row's two.  Columns that the row does not have are 0 in dy and add nothing.
__device__ __forceinline__ void take_piece(const float (&x)[kPiece], const float (&dy)[kPiece], const float (&w)[kPiece], float mean, float rstd,
                                           PieceSums &sums, Pair &s1, Pair &s2) {
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i) {
        const Pair d = pair(dy[2 * i], dy[2 * i + 1]), xhat = xhat_of(x[2 * i], x[2 * i + 1], mean, rstd);
        sums.db[i] = add2(sums.db[i], d);
        sums.dw[i] = fma2(d, xhat, sums.dw[i]);
        const Pair g = mul2(d, pair(w[2 * i], w[2 * i + 1]));
        s1 = add2(s1, g);
        s2 = fma2(g, xhat, s2);
    }
}
// dx of a piece; s1, s2: the row's sums divided by its length.  (Computed anew rather than kept: registers are dearer.)
__device__ __forceinline__ void piece_dx(const float (&x)[kPiece], const float (&dy)[kPiece], const float (&w)[kPiece], float mean, float rstd,
                                         float s1, float s2, float (&dx)[kPiece]) {
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i) {
        const Pair xhat = xhat_of(x[2 * i], x[2 * i + 1], mean, rstd);
        const Pair g = fma2(pair(dy[2 * i], dy[2 * i + 1]), pair(w[2 * i], w[2 * i + 1]), pair(-s1, -s1));
        split(mul2(fma2(xhat, pair(-s2, -s2), g), pair(rstd, rstd)), dx[2 * i], dx[2 * i + 1]);
    }
}
// A piece's sums to a vector of all columns, or in addition to what is there.
template <bool EVEN>
__device__ __forceinline__ void put_sums(float *to, const Columns<EVEN> &c, int u, const Pair (&v)[kPiece / 2], bool add) {
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i) {
        float p, q;
        split(v[i], p, q);
        if (c.has(u, 2 * i)) to[c.at(u, 2 * i)] = add ? to[c.at(u, 2 * i)] + p : p;
        if (c.has(u, 2 * i + 1)) to[c.at(u, 2 * i + 1)] = add ? to[c.at(u, 2 * i + 1)] + q : q;
    }
}

// Rows of up to 256 elements: `lanes` lanes to a row, one piece to a lane.
constexpr int kLanesThreads = 256;

template <typename T, typename G, bool EVEN>
__global__ void __launch_bounds__(kLanesThreads)
layer_norm_backward_short_kernel(const NormBackArgs a, int lanes) {
    __shared__ float total[2 * 32 * kPiece];
    let_next_start();
    const Columns<EVEN> c = {(int)threadIdx.x % lanes, lanes, a.dim};
    const int groups = kLanesThreads / lanes;
    const T *x0 = static_cast<const T *>(a.x);
    const G *dy0 = static_cast<const G *>(a.dy);
    float w[kPiece];
    load_piece(a.weight, c, 0, true, w);
    PieceSums sums = {};
    const int64_t step = (int64_t)gridDim.x * groups;
    Piece<T, EVEN> next_x;
    Piece<G, EVEN> next_dy;
    float next_mean = 0.f, next_rstd = 0.f;
    const auto send_for = [&](int64_t row) {
        const bool live = row < a.rows;
        next_x.load(x0 + (live ? row * a.ld_x : 0), c, 0, live);
        next_dy.load(dy0 + (live ? row * a.ld_dy : 0), c, 0, live);
        next_mean = live ? a.mean[row] : 0.f;
        next_rstd = live ? a.rstd[row] : 0.f;
    };
    send_for((int64_t)blockIdx.x * groups + threadIdx.x / lanes);
    // all lanes of a warp go round together, the last rows of some being none
    for (int64_t base = (int64_t)blockIdx.x * groups; base < a.rows; base += step) {
        const int64_t row = base + threadIdx.x / lanes;
        float x[kPiece], dy[kPiece];
        next_x.get(x);
        next_dy.get(dy);
        const float mean = next_mean, rstd = next_rstd;
        send_for(row + step);
        Pair p1 = 0, p2 = 0;
        take_piece(x, dy, w, mean, rstd, sums, p1, p2);
        if (!a.dx) continue;
        const float s1 = lanes_sum(pair_sum(p1), lanes) * a.inv_dim, s2 = lanes_sum(pair_sum(p2), lanes) * a.inv_dim;
        float dx[kPiece];
        piece_dx(x, dy, w, mean, rstd, s1, s2, dx);
        const bool live = row < a.rows;
        store_piece(static_cast<T *>(a.dx) + (live ? row * a.ld_dx : 0), c, 0, live, dx);
    }
    if (!a.parts) return;
    // the rows of a warp by exchange, the warps one after the other in shared memory
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i)
        for (int o = lanes; o < 32; o <<= 1) {
            sums.dw[i] = add2(sums.dw[i], __shfl_xor_sync(0xffffffffu, sums.dw[i], o));
            sums.db[i] = add2(sums.db[i], __shfl_xor_sync(0xffffffffu, sums.db[i], o));
        }
    for (int warp = 0; warp < kLanesThreads / 32; ++warp) {
        if ((int)threadIdx.x / 32 == warp && (int)threadIdx.x % 32 < lanes) {
            put_sums(total, c, 0, sums.dw, warp > 0);
            put_sums(total + 32 * kPiece, c, 0, sums.db, warp > 0);
        }
        __syncthreads();
    }
    const int64_t pad = padded(a.dim);
    float *part = a.parts + (int64_t)blockIdx.x * 2 * pad;
    for (int i = threadIdx.x; i < a.dim; i += kLanesThreads) {
        part[i] = total[i];
        part[pad + i] = total[32 * kPiece + i];
    }
}

// Longer rows: a group of warps walks rows, U pieces to a thread, the next rows on their way (to registers, of uneven rows,
// with one piece to a thread).  The groups of a block join their sums in shared memory, so that one set of them leaves an SM.
template <typename T, typename G, int U, bool EVEN>
__global__ void __launch_bounds__(32 * kGroupWarps)
layer_norm_backward_kernel(const NormBackArgs a, int warps) {
    constexpr int kUnitsX = Piece<T, true>::kUnits, kUnits = kUnitsX + Piece<G, true>::kUnits;
    constexpr bool kNext = !EVEN && U == 1;
    extern __shared__ uint4 ahead[];  // [rows ahead][U][units of both pieces][threads]; at the end two sums of each column
    __shared__ float slots[2][kGroupWarps][2];
    let_next_start();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const Group group(warps);
    const Columns<EVEN> c = {group.t, 32 * warps, a.dim};
    const T *x0 = static_cast<const T *>(a.x);
    const G *dy0 = static_cast<const G *>(a.dy);
    const int64_t step = (int64_t)gridDim.x * group.count;
    int64_t row = (int64_t)blockIdx.x * group.count + group.index;
    const auto slot = [&](int stage, int u, int i) { return ahead + ((stage * U + u) * kUnits + i) * blockDim.x + threadIdx.x; };
    const auto send_for = [&](int64_t r, int stage) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r < a.rows && c.has(u, 0)) {
#pragma unroll
                for (int i = 0; i < kUnits; ++i)
                    copy16((uint32_t)__cvta_generic_to_shared(slot(stage, u, i)),
                           i < kUnitsX ? reinterpret_cast<const uint4 *>(x0 + r * a.ld_x + c.at(u, 0)) + i
                                       : reinterpret_cast<const uint4 *>(dy0 + r * a.ld_dy + c.at(u, 0)) + (i - kUnitsX));
            }
        copies_end_group();
    };
    Piece<T, EVEN> raw_x[U], next_x[U];
    Piece<G, EVEN> raw_dy[U], next_dy[U];
    float next_mean = 0.f, next_rstd = 0.f;
    const auto load = [&](int64_t r, Piece<T, EVEN> (&px)[U], Piece<G, EVEN> (&pdy)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            px[u].load(x0 + (r < a.rows ? r * a.ld_x : 0), c, u, r < a.rows);
            pdy[u].load(dy0 + (r < a.rows ? r * a.ld_dy : 0), c, u, r < a.rows);
        }
    };
    if constexpr (EVEN) {
        for (int i = 0; i < kAhead; ++i) send_for(row + i * step, i);
    } else if constexpr (kNext) {
        load(row, next_x, next_dy);
    }
    if (row < a.rows) {
        next_mean = a.mean[row];
        next_rstd = a.rstd[row];
    }
    float w[U][kPiece];
    PieceSums sums[U] = {};
#pragma unroll
    for (int u = 0; u < U; ++u) load_piece(a.weight, c, u, true, w[u]);
    for (int stage = 0, turn = 0; row < a.rows; row += step, stage = stage + 1 == kAhead ? 0 : stage + 1, turn ^= 1) {
        const float mean = next_mean, rstd = next_rstd;
        if (row + step < a.rows) {
            next_mean = a.mean[row + step];
            next_rstd = a.rstd[row + step];
        }
        if constexpr (EVEN) {
            copies_wait<kAhead - 1>();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool has = c.has(u, 0);
#pragma unroll
                for (int i = 0; i < kUnits; ++i) {
                    const uint4 q = has ? *slot(stage, u, i) : make_uint4(0, 0, 0, 0);
                    if (i < kUnitsX) raw_x[u].even[i < kUnitsX ? i : 0] = q;
                    else raw_dy[u].even[i < kUnitsX ? 0 : i - kUnitsX] = q;
                }
            }
        } else if constexpr (kNext) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                raw_x[u] = next_x[u];
                raw_dy[u] = next_dy[u];
            }
            load(row + step, next_x, next_dy);
        } else {
            load(row, raw_x, raw_dy);
        }
        Pair p1 = 0, p2 = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[kPiece], dy[kPiece];
            raw_x[u].get(x);
            raw_dy[u].get(dy);
            take_piece(x, dy, w[u], mean, rstd, sums[u], p1, p2);
        }
        if (a.dx) {
            // two sums over a warp: each half of it takes one
            const float s1 = pair_sum(p1), s2 = pair_sum(p2);
            float s = (lane & 16 ? s2 : s1) + __shfl_xor_sync(0xffffffffu, lane & 16 ? s1 : s2, 16);
            s = lanes_sum(s, 16);
            if (lane % 16 == 0) slots[turn][warp][lane / 16] = s;
            group.sync();
            float m1 = 0.f, m2 = 0.f;
            for (int i = 0; i < warps; ++i) {
                const float2 q = *reinterpret_cast<const float2 *>(slots[turn][group.index * warps + i]);
                m1 += q.x;
                m2 += q.y;
            }
            m1 *= a.inv_dim;
            m2 *= a.inv_dim;
            T *dx = static_cast<T *>(a.dx) + row * a.ld_dx;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x[kPiece], dy[kPiece], out[kPiece];
                raw_x[u].get(x);
                raw_dy[u].get(dy);
                piece_dx(x, dy, w[u], mean, rstd, m1, m2, out);
                store_piece(dx, c, u, true, out);
            }
        }
        if constexpr (EVEN) send_for(row + kAhead * step, stage);  // behind the last use of what was there
    }
    if (!a.parts) return;
    const int64_t pad = padded(a.dim);
    float *part = a.parts + (int64_t)blockIdx.x * 2 * pad, *joined = reinterpret_cast<float *>(ahead);
    __syncthreads();  // all copies have been waited for by those who sent for them
    for (int q = 0; q < group.count; ++q) {
        if (q == group.index) {
            const bool last = q + 1 == group.count;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (q > 0 && last) {  // the last group brings the sums out
#pragma unroll
                    for (int i = 0; i < kPiece / 2; ++i) {
                        const int at0 = c.at(u, 2 * i), at1 = c.at(u, 2 * i + 1);
                        const bool has0 = c.has(u, 2 * i), has1 = c.has(u, 2 * i + 1);
                        sums[u].dw[i] = add2(sums[u].dw[i], pair(has0 ? joined[at0] : 0.f, has1 ? joined[at1] : 0.f));
                        sums[u].db[i] = add2(sums[u].db[i], pair(has0 ? joined[pad + at0] : 0.f, has1 ? joined[pad + at1] : 0.f));
                    }
                }
                put_sums(last ? part : joined, c, u, sums[u].dw, q > 0 && !last);
                put_sums((last ? part : joined) + pad, c, u, sums[u].db, q > 0 && !last);
            }
        }
        if (q + 1 < group.count) __syncthreads();
    }
}

// Rows too long for that: the two sums of each row first, then columns by the tile.
template <typename T, typename G>
__global__ void __launch_bounds__(kLongThreads)
layer_norm_row_sums_kernel(const NormBackArgs a, float2 *sums) {
    __shared__ float slots[2][kGroupWarps];
    const Group group(kGroupWarps);
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
    const G *dy = static_cast<const G *>(a.dy) + row * a.ld_dy;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.f, s2 = 0.f;
    for (int c = threadIdx.x; c < a.dim; c += kLongThreads) {
        const float g = widen(dy[c]) * a.weight[c];
        s1 += g;
        s2 = fmaf(g, (widen(x[c]) - mean) * rstd, s2);
    }
    s1 = group.sum(s1, slots[0]);
    s2 = group.sum(s2, slots[1]);
    if (threadIdx.x == 0) sums[row] = make_float2(s1 * a.inv_dim, s2 * a.inv_dim);
}

constexpr int kTileColumns = 2;  // of a thread, kLanesThreads apart

template <typename T, typename G>
__global__ void __launch_bounds__(kLanesThreads)
layer_norm_tiles_kernel(const NormBackArgs a, const float2 *sums) {
    const int c0 = blockIdx.x * kTileColumns * kLanesThreads + threadIdx.x;
    const T *x0 = static_cast<const T *>(a.x);
    const G *dy0 = static_cast<const G *>(a.dy);
    T *dx0 = static_cast<T *>(a.dx);
    float w[kTileColumns], dw[kTileColumns], db[kTileColumns];
#pragma unroll
    for (int i = 0; i < kTileColumns; ++i) {
        w[i] = c0 + i * kLanesThreads < a.dim ? a.weight[c0 + i * kLanesThreads] : 0.f;
        dw[i] = db[i] = 0.f;
    }
#pragma unroll 4
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        const float2 s = a.dx ? sums[row] : make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kTileColumns; ++i) {
            const int c = c0 + i * kLanesThreads;
            if (c >= a.dim) continue;
            const float g = widen(dy0[row * a.ld_dy + c]), xhat = (widen(x0[row * a.ld_x + c]) - mean) * rstd;
            db[i] += g;
            dw[i] = fmaf(g, xhat, dw[i]);
            if (a.dx) dx0[row * a.ld_dx + c] = narrowed<T>(rstd * (g * w[i] - fmaf(xhat, s.y, s.x)));
        }
    }
    if (!a.parts) return;
    float *part = a.parts + (int64_t)blockIdx.y * 2 * padded(a.dim);
#pragma unroll
    for (int i = 0; i < kTileColumns; ++i) {
        const int c = c0 + i * kLanesThreads;
        if (c >= a.dim) continue;
        part[c] = dw[i];
        part[padded(a.dim) + c] = db[i];
    }
}

// The blocks' sums, 32 columns to a block; warps take every 16th, then the warps' sums in their order.
constexpr int kJoinWarps = 16;

__global__ void __launch_bounds__(32 * kJoinWarps)
layer_norm_join_kernel(const NormBackArgs a, int parts) {
    __shared__ float slots[kJoinWarps][32];
    wait_for_previous();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const bool of_bias = blockIdx.y == 1;
    const int c = blockIdx.x * 32 + lane;
    const int64_t pad = padded(a.dim);
    const float *from = a.parts + (of_bias ? pad : 0) + c;
    float s = 0.f;
    if (c < a.dim) {
#pragma unroll 8
        for (int i = warp; i < parts; i += kJoinWarps) s += __ldcg(from + (int64_t)i * 2 * pad);
    }
    slots[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || c >= a.dim) return;
    s = 0.f;
    for (int i = 0; i < kJoinWarps; ++i) s += slots[i][lane];
    float *g = of_bias ? a.dbias : a.dweight, *m = of_bias ? a.m_bias : a.m_weight, *v = of_bias ? a.v_bias : a.v_weight;
    if (g) g[c] = s;
    if (m) fold1(s, m[c], v[c], a.fold.a, a.fold.b);
}

// ---- launches --------------------------------------------------------------------------------------

int lanes_for(int pieces) {
    int lanes = 1;
    while (lanes < pieces) lanes *= 2;
    return lanes;
}
constexpr int kLongPieces = 64 * kGroupWarps;  // longer rows are read more than once

// How a call over rows of up to kLongPieces pieces runs: pieces to a thread, warps to a row, rows side by side.
struct RowPlan {
    int pieces, each, warps, groups;
};

template <typename T, typename O, int U, bool EVEN>
cudaError_t forward_groups(const NormArgs &a, const RowPlan &p, int sm_count, cudaStream_t stream) {
    constexpr int kResident = 768;  // threads of an SM that 80 registers allow
    const int threads = 32 * p.warps * p.groups;
    const size_t shared = EVEN ? (size_t)kAhead * U * Piece<T, true>::kUnits * threads * 16 : 0;
    const unsigned grid = grid_for((size_t)a.rows, (size_t)p.groups, sm_count, threads < kResident ? kResident / threads : 1);
    if (shared > 40 * 1024) {  // with the static part, more than a kernel has unasked
        static std::atomic<unsigned long long> ready{0};
        const cudaError_t e = allow_shared(layer_norm_kernel<T, O, U, EVEN>, 160 * 1024, ready);
        if (e != cudaSuccess) return e;
    }
    layer_norm_kernel<T, O, U, EVEN><<<grid, threads, shared, stream>>>(a, p.warps);
    return cudaGetLastError();
}

template <typename T, typename O, bool EVEN>
cudaError_t forward(const NormArgs &a, int sm_count, cudaStream_t stream) {
    RowPlan p;
    p.pieces = (int)(padded(a.dim) / kPiece);
    if (p.pieces <= 32) {
        const int lanes = lanes_for(p.pieces), rows = kShortThreads / lanes;
        layer_norm_short_kernel<T, O, EVEN><<<(unsigned)((a.rows + rows - 1) / rows), kShortThreads, 0, stream>>>(a, lanes);
        return cudaGetLastError();
    }
    if (p.pieces > kLongPieces) {
        layer_norm_long_kernel<T, O><<<(unsigned)a.rows, kLongThreads, 0, stream>>>(a);
        return cudaGetLastError();
    }
    // few rows: more threads to each
    p.each = p.pieces > 32 * kGroupWarps || a.rows >= 2 * (int64_t)sm_count ? 2 : 1;
    p.warps = (p.pieces + 32 * p.each - 1) / (32 * p.each);
    p.groups = p.warps < 4 && a.rows >= 2 * (int64_t)sm_count ? 4 / p.warps : 1;
    return p.each == 2 ? forward_groups<T, O, 2, EVEN>(a, p, sm_count, stream) : forward_groups<T, O, 1, EVEN>(a, p, sm_count, stream);
}
template <typename T, typename O>
cudaError_t forward(const NormArgs &a, int sm_count, cudaStream_t stream) {
    const bool even = even_rows(a.x, a.dim, a.ld_x, sizeof(T)) && even_rows(a.y, a.dim, a.ld_y, sizeof(O)) && aligned(a.weight, 16) &&
                      aligned(a.bias, 16);
    return even ? forward<T, O, true>(a, sm_count, stream) : forward<T, O, false>(a, sm_count, stream);
}

// Blocks of the backward pass, whose sums the workspace holds; behind them two sums of each row where rows are long.
struct BackPlan : RowPlan {
    bool is_long;
    int64_t parts;
};
BackPlan plan_back(int64_t rows, int dim, int sm_count, bool even) {
    BackPlan p;
    p.pieces = (int)(padded(dim) / kPiece);
    p.each = p.pieces > 32 * kGroupWarps || (even && rows >= 2 * (int64_t)sm_count) ? 2 : 1;
    p.warps = (p.pieces + 32 * p.each - 1) / (32 * p.each);
    p.groups = 1;
    p.is_long = p.pieces > kLongPieces;
    int64_t most = sm_count;
    if (p.pieces <= 32) {
        p.groups = kLanesThreads / lanes_for(p.pieces);
        most = 4 * (int64_t)sm_count;
    } else if (p.is_long) {
        const int64_t tiles = (dim + kTileColumns * kLanesThreads - 1) / (kTileColumns * kLanesThreads);
        most = (4 * (int64_t)sm_count + tiles - 1) / tiles;
    } else {
        // as many rows to a block as it has warps for, fewer where that would leave SMs without any
        p.groups = kGroupWarps / p.warps;
        while (p.groups > 1 && rows < (int64_t)sm_count * p.groups) p.groups -= 1;
    }
    p.parts = (rows + p.groups - 1) / p.groups;
    if (p.parts > most) p.parts = most;
    if (p.parts < 1) p.parts = 1;
    return p;
}

template <typename T, typename G, int U, bool EVEN>
cudaError_t back_groups(const NormBackArgs &a, const BackPlan &p, cudaStream_t stream) {
    const int threads = 32 * p.warps * p.groups;
    size_t shared = EVEN ? (size_t)kAhead * U * (Piece<T, true>::kUnits + Piece<G, true>::kUnits) * threads * 16 : 0;
    const size_t joined = p.groups > 1 && a.parts ? (size_t)2 * padded(a.dim) * sizeof(float) : 0;
    if (shared < joined) shared = joined;
    if (shared > 40 * 1024) {  // with the static part, more than a kernel has unasked
        static std::atomic<unsigned long long> ready{0};
        const cudaError_t e = allow_shared(layer_norm_backward_kernel<T, G, U, EVEN>, 200 * 1024, ready);
        if (e != cudaSuccess) return e;
    }
    layer_norm_backward_kernel<T, G, U, EVEN><<<(unsigned)p.parts, threads, shared, stream>>>(a, p.warps);
    return cudaGetLastError();
}
template <typename T, typename G, bool EVEN>
cudaError_t launch_back(const NormBackArgs &a, const BackPlan &p, cudaStream_t stream) {
    if (p.pieces <= 32) {
        layer_norm_backward_short_kernel<T, G, EVEN><<<(unsigned)p.parts, kLanesThreads, 0, stream>>>(a, lanes_for(p.pieces));
        return cudaGetLastError();
    }
    return p.each == 2 ? back_groups<T, G, 2, EVEN>(a, p, stream) : back_groups<T, G, 1, EVEN>(a, p, stream);
}

template <typename T, typename G>
cudaError_t backward(const NormBackArgs &a, int sm_count, cudaStream_t stream, int *launches) {
    const bool even = even_rows(a.x, a.dim, a.ld_x, sizeof(T)) && even_rows(a.dy, a.dim, a.ld_dy, sizeof(G)) &&
                      (!a.dx || even_rows(a.dx, a.dim, a.ld_dx, sizeof(T))) && aligned(a.weight, 16);
    const BackPlan p = plan_back(a.rows, a.dim, sm_count, even);
    cudaError_t e = cudaSuccess;
    if (a.rows > 0) {
        if (p.is_long) {
            float2 *sums = reinterpret_cast<float2 *>(static_cast<float *>(a.workspace) + p.parts * 2 * padded(a.dim));
            if (a.dx) layer_norm_row_sums_kernel<T, G><<<(unsigned)a.rows, kLongThreads, 0, stream>>>(a, sums);
            const dim3 tiles((unsigned)((a.dim + kTileColumns * kLanesThreads - 1) / (kTileColumns * kLanesThreads)), (unsigned)p.parts);
            layer_norm_tiles_kernel<T, G><<<tiles, kLanesThreads, 0, stream>>>(a, sums);
            e = cudaGetLastError();
        } else {
            e = even ? launch_back<T, G, true>(a, p, stream) : launch_back<T, G, false>(a, p, stream);
        }
        if (e != cudaSuccess) return e;
        *launches += p.is_long && a.dx ? 2 : 1;
    }
    if (a.parts) {
        const dim3 columns((unsigned)((a.dim + 31) / 32), 2), block(32 * kJoinWarps);
        if (a.rows > 0) {
            e = launch_chained(layer_norm_join_kernel, columns, block, 0, stream, a, (int)p.parts);
        } else {  // nothing in front that it could be chained to
            layer_norm_join_kernel<<<columns, block, 0, stream>>>(a, 0);
            e = cudaGetLastError();
        }
        *launches += 1;
    }
    return e;
}

}  // namespace

size_t norm_workspace_bytes(int64_t rows, int dim, int sm_count) {
    // (whichever way the rows lie: an even call has no more blocks than an uneven one)
    const BackPlan p = plan_back(rows, dim, sm_count, false);
    return (size_t)p.parts * 2 * padded(dim) * sizeof(float) + (p.is_long ? (size_t)rows * sizeof(float2) : 0);
}

cudaError_t launch_layer_norm(const NormArgs &a, int sm_count, cudaStream_t stream) {
    if (a.x_dtype == ADAMA_F32)
        return a.y_dtype == ADAMA_F32 ? forward<float, float>(a, sm_count, stream) : forward<float, __nv_bfloat16>(a, sm_count, stream);
    return a.y_dtype == ADAMA_F32 ? forward<__nv_bfloat16, float>(a, sm_count, stream) : forward<__nv_bfloat16, __nv_bfloat16>(a, sm_count, stream);
}

cudaError_t launch_layer_norm_backward(const NormBackArgs &a, int sm_count, cudaStream_t stream, int *launches) {
    if (a.x_dtype == ADAMA_F32)
        return a.dy_dtype == ADAMA_F32 ? backward<float, float>(a, sm_count, stream, launches)
                                       : backward<float, __nv_bfloat16>(a, sm_count, stream, launches);
    return a.dy_dtype == ADAMA_F32 ? backward<__nv_bfloat16, float>(a, sm_count, stream, launches)
                                   : backward<__nv_bfloat16, __nv_bfloat16>(a, sm_count, stream, launches);
}

}  // namespace adama
