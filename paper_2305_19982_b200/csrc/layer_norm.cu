// Layer norm and its backward pass.  Over the D elements of a row:
//     mean = sum x / D,  var = sum (x - mean)^2 / D,  rstd = 1/sqrt(var + eps),  xhat = (x - mean)*rstd
//     y = xhat*weight + bias
// and, with g = dy*weight, the sums over a row s1 = sum g, s2 = sum g*xhat:
//     dx = rstd*(g - s1/D - xhat*s2/D),   dweight = sum over rows of dy*xhat,   dbias = the same of dy
// A row is read once and held in registers; the variance is taken of x - mean, so that a common offset costs
// no precision.  In the backward pass a thread keeps its columns for all rows of its block, with their two sums
// in registers; the blocks' sums go to the workspace, and a second, short kernel adds them in the blocks' order
// and writes the parameters' gradients or folds them into their moments (m += a*g, v += b*g^2: the sum over
// rows is complete before it is squared).  Nothing depends on scheduling.
//
// Bound by HBM where there is enough to do: 16384 x 4096 bf16 takes 48 us forward = 5.6 TB/s, 75 us backward = 5.4 TB/s.  4096 x 1600
// is one wave, in which launch, first rows, sums across warps and the last rows come in sequence: 13 us forward (fp32 to
// bf16, floor 6), 17 us backward with the moments (floor 6).  Its 200 pieces take 256 places (four to a lane of two warps forward,
// two of four backward), and forward 1184 groups go round four times for 3.5 turns of rows.  One row: 2.8 us.  Rows that are not even (row_access.cuh) are bound
// by instructions, an element to an access: 8192 x 1601 bf16 24 us forward, 39 backward (floors 8 and 12).  Bringing them to
// shared memory by the 16 bytes made them slower (17696 x 760 39 -> 57): it is not latency that they wait for.
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
#pragma unroll 4
        for (int i = 0; i < warps; ++i) x += slots[index * warps + i];
        return x;
    }
};

// s/n for a whole number n, without a division's length: a product, and what it lacks.  (The product alone would
// move the mean of equal values.)
__device__ __forceinline__ float share(float s, float n, float inv_n) {
    const float q = s * inv_n, lack = fmaf(-q, n, s);
    return lack == lack ? fmaf(lack, inv_n, q) : q;  // (an infinite sum stays one)
}

constexpr int kGroupWarps = 16;  // of a block, at most

__device__ __forceinline__ Vec sum_of(const Vec &a, const Vec &b) {
    return {{add2(a.p[0], b.p[0]), add2(a.p[1], b.p[1]), add2(a.p[2], b.p[2]), add2(a.p[3], b.p[3])}};
}
__device__ __forceinline__ Pair sum_of(const Vec &v) { return add2(add2(v.p[0], v.p[1]), add2(v.p[2], v.p[3])); }
// v becomes its distance from the mean; returns that squared, summed.  Columns that the row does not have lie at none.
template <bool EVEN, int N, int W>
__device__ __forceinline__ Pair centre(Vec &v, const Columns<EVEN, N, W> &c, int u, float mean) {
    if constexpr (!EVEN) {
#pragma unroll
        for (int i = 0; i < kPiece / 2; ++i) {
            float a, b;
            split(v.p[i], a, b);
            v.p[i] = pair(c.has(u, 2 * i) ? a : mean, c.has(u, 2 * i + 1) ? b : mean);
        }
    }
    Pair s[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i) {
        v.p[i] = add2(v.p[i], pair(-mean, -mean));
        s[i / 2] = fma2(v.p[i], v.p[i], s[i / 2]);
    }
    return add2(EVEN && !c.has(u, 0) ? 0 : s[0], EVEN && !c.has(u, kPiece / 2) ? 0 : s[1]);
}
__device__ __forceinline__ void scale_shift(Vec &v, float rstd, const Vec &w, const Vec &b) {
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i) v.p[i] = fma2(mul2(v.p[i], pair(rstd, rstd)), w.p[i], b.p[i]);
}

// ---- forward -------------------------------------------------------------------------------------

// Rows of up to 256 elements: `lanes` lanes to a row, one piece to a lane.
constexpr int kShortThreads = 128;

template <typename T, typename O, bool EVEN>
__global__ void __launch_bounds__(kShortThreads)
layer_norm_short_kernel(const NormArgs a, int lanes) {
    const Columns<EVEN, together(sizeof(T), sizeof(O))> c = {(int)threadIdx.x % lanes, lanes, a.dim};
    const int64_t row = (int64_t)blockIdx.x * (kShortThreads / lanes) + threadIdx.x / lanes;
    const bool live = row < a.rows;
    Piece<T, EVEN> raw;
    Piece<float, EVEN> raw_w, raw_b;
    raw.load(static_cast<const T *>(a.x) + (live ? row : 0) * a.ld_x, c, 0, live);
    raw_w.load(a.weight, c, 0, live);
    raw_b.load(a.bias, c, 0, live && a.bias);
    Vec v = raw.get();
    const float n = (float)a.dim, mean = share(lanes_sum(pair_sum(sum_of(v)), lanes), n, a.inv_dim);
    const float rstd = __frsqrt_rn(share(lanes_sum(pair_sum(centre(v, c, 0, mean)), lanes), n, a.inv_dim) + a.eps);
    if (c.t == 0 && live) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    scale_shift(v, rstd, raw_w.get(), raw_b.get());
    store_piece(static_cast<O *>(a.y) + (live ? row : 0) * a.ld_y, c, 0, live, v);
}

// Longer rows: a group of warps walks rows, U pieces to a thread; weight and bias lie in shared memory, as do the next
// rows of a thread, which are on their way while it works on one.  A row costs a warp some 200 instructions beside those of
// its elements, and exchanges between lanes and warps wait for each other: so few warps share a row, with many pieces
// to a thread, where there are rows enough (4096 x 1600 fp32 to bf16: four warps to a row 20 us, two 13).
constexpr int kAhead = 2;  // rows of a thread on their way, of even ones

template <typename T, typename O, int U, bool EVEN, int WARPS>
__global__ void __launch_bounds__(32 * kGroupWarps)
layer_norm_kernel(const NormArgs a, int warps) {
    extern __shared__ uint4 shared[];  // even: [pieces][2][threads of a row] of weight, of bias, then [rows ahead][U][units][threads]
    __shared__ float slots[2][kGroupWarps];
    constexpr int N = together(sizeof(T), sizeof(O));
    using Ahead = Slot<T, EVEN>;
    const Group group(WARPS ? WARPS : warps);
    const Columns<EVEN, N, 32 * WARPS> c = {group.t, 32 * warps, a.dim};
    const T *x0 = static_cast<const T *>(a.x);
    const int64_t step = (int64_t)gridDim.x * group.count;
    int64_t row = (int64_t)blockIdx.x * group.count + group.index;
    uint4 *const params = shared;
    unsigned char *const ahead = reinterpret_cast<unsigned char *>(shared + 4 * U * c.width());
    float *const odd_params = reinterpret_cast<float *>(shared);  // uneven: weight, bias
    const auto slot = [&](int stage, int u) { return ahead + (stage * U + u) * (int)blockDim.x * Ahead::kBytes; };
    const auto send_for = [&](int64_t r, int stage) {
        if (r < a.rows) {
#pragma unroll
            for (int u = 0; u < U; ++u) Ahead::send_for(slot(stage, u), x0 + r * a.ld_x, c, u, threadIdx.x, blockDim.x);
        }
        copies_end_group();
    };
    if constexpr (EVEN) {
        for (int i = 0; i < kAhead; ++i) {
#pragma unroll
            for (int u = 0; u < U; ++u) Ahead::clear(slot(i, u), c, u, threadIdx.x, blockDim.x);
            send_for(row + i * step, i);
        }
        const uint4 zero = make_uint4(0, 0, 0, 0);
        for (int i = threadIdx.x; i < 2 * U * c.width(); i += blockDim.x) {
            // fours of columns, in the order in which a piece's halves lie
            const int piece = i / 2, at = N == 4 ? i : ((piece / c.width()) * 2 + i % 2) * c.width() + piece % c.width();
            const bool has = i * 4 < a.dim;
            params[at] = has ? reinterpret_cast<const uint4 *>(a.weight)[i] : zero;
            params[2 * U * c.width() + at] = has && a.bias ? reinterpret_cast<const uint4 *>(a.bias)[i] : zero;
        }
    } else {
        for (int i = threadIdx.x; i < a.dim; i += blockDim.x) {
            odd_params[i] = a.weight[i];
            odd_params[a.dim + i] = a.bias ? a.bias[i] : 0.f;
        }
    }
    __syncthreads();
    const float n = (float)a.dim;
    for (int stage = 0; row < a.rows; row += step, stage = stage + 1 == kAhead ? 0 : stage + 1) {
        Vec v[U];
        Pair s = 0;
        if constexpr (EVEN) {
            copies_wait<kAhead - 1>();
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = Ahead::get(slot(stage, u), x0, c, u, threadIdx.x, blockDim.x);
        } else {
            Piece<T, EVEN> raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u].load(x0 + row * a.ld_x, c, u, true);
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = raw[u].get();
        }
#pragma unroll
        for (int u = 0; u < U; ++u) s = add2(s, sum_of(v[u]));
        const float mean = share(group.sum(pair_sum(s), slots[0]), n, a.inv_dim);
        if constexpr (EVEN) send_for(row + kAhead * step, stage);  // what was there has been summed up
        s = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) s = add2(s, centre(v[u], c, u, mean));
        const float rstd = __frsqrt_rn(share(group.sum(pair_sum(s), slots[1]), n, a.inv_dim) + a.eps);
        if (c.t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        O *y = static_cast<O *>(a.y) + row * a.ld_y;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Vec w, b;
            if constexpr (EVEN) {
                uint4 q[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) q[i] = params[(u * 2 + i) * c.width() + c.t];
                w = widened(q);
#pragma unroll
                for (int i = 0; i < 2; ++i) q[i] = params[(2 * U + u * 2 + i) * c.width() + c.t];
                b = widened(q);
            } else {
                w = load_piece(odd_params, c, u, true);
                b = load_piece(odd_params + a.dim, c, u, true);
            }
            scale_shift(v[u], rstd, w, b);
            store_piece(y, c, u, true, v[u]);
        }
    }
}

// Rows that no group holds in registers: read three times, from L2 if they stay there, an element to an access.
// 2048 x 12288 bf16 48 us (floor 15), fp32 57 (31); 2048 x 14336 bf16 54 (18).
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
    const float n = (float)a.dim, mean = share(group.sum(s, slots[0]), n, a.inv_dim);
    s = 0.f;
    for (int c = threadIdx.x; c < a.dim; c += kLongThreads) {
        const float d = widen(x[c]) - mean;
        s = fmaf(d, d, s);
    }
    const float rstd = __frsqrt_rn(share(group.sum(s, slots[1]), n, a.inv_dim) + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    O *y = static_cast<O *>(a.y) + row * a.ld_y;
    for (int c = threadIdx.x; c < a.dim; c += kLongThreads)
        y[c] = narrow<O>(fmaf((widen(x[c]) - mean) * rstd, a.weight[c], a.bias ? a.bias[c] : 0.f));
}

// ---- backward ------------------------------------------------------------------------------------

// A block's sums in the workspace: dweight, then dbias, each padded to whole pieces.
__host__ __device__ inline int64_t padded(int dim) { return ((int64_t)dim + kPiece - 1) / kPiece * kPiece; }

// Sums over rows, of a thread's columns.
struct PieceSums {
    Vec dw, db;
};
__device__ __forceinline__ Pair xhat_of(Pair x, float mean, float rstd) { return mul2(add2(x, pair(-mean, -mean)), pair(rstd, rstd)); }
// A piece's part in its columns' sums and in its row's two.  Columns that the row does not have are 0 in dy and add nothing.
__device__ __forceinline__ void take_piece(const Vec &x, const Vec &dy, const Vec &w, float mean, float rstd, PieceSums &sums, Pair &s1, Pair &s2) {
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i) {
        const Pair xhat = xhat_of(x.p[i], mean, rstd);
        sums.db.p[i] = add2(sums.db.p[i], dy.p[i]);
        sums.dw.p[i] = fma2(dy.p[i], xhat, sums.dw.p[i]);
        const Pair g = mul2(dy.p[i], w.p[i]);
        s1 = add2(s1, g);
        s2 = fma2(g, xhat, s2);
    }
}
// dx of a piece; s1, s2: the row's sums divided by its length.  (Computed anew rather than kept: registers are dearer.)
__device__ __forceinline__ Vec piece_dx(const Vec &x, const Vec &dy, const Vec &w, float mean, float rstd, float s1, float s2) {
    Vec dx;
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i) {
        const Pair xhat = xhat_of(x.p[i], mean, rstd);
        const Pair g = fma2(dy.p[i], w.p[i], pair(-s1, -s1));
        dx.p[i] = mul2(fma2(xhat, pair(-s2, -s2), g), pair(rstd, rstd));
    }
    return dx;
}

// Rows of up to 256 elements: `lanes` lanes to a row, one piece to a lane.
constexpr int kLanesThreads = 256;

template <typename T, typename G, bool EVEN>
__global__ void __launch_bounds__(kLanesThreads)
layer_norm_backward_short_kernel(const NormBackArgs a, int lanes) {
    __shared__ alignas(16) float total[2 * 32 * kPiece];
    let_next_start();
    const Columns<EVEN, together(sizeof(T), sizeof(G))> c = {(int)threadIdx.x % lanes, lanes, a.dim};
    const int groups = kLanesThreads / lanes;
    const T *x0 = static_cast<const T *>(a.x);
    const G *dy0 = static_cast<const G *>(a.dy);
    const Vec w = load_piece(a.weight, c, 0, true);
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
        const Vec x = next_x.get(), dy = next_dy.get();
        const float mean = next_mean, rstd = next_rstd;
        send_for(row + step);
        Pair p1 = 0, p2 = 0;
        take_piece(x, dy, w, mean, rstd, sums, p1, p2);
        if (!a.dx) continue;
        const float s1 = lanes_sum(pair_sum(p1), lanes) * a.inv_dim, s2 = lanes_sum(pair_sum(p2), lanes) * a.inv_dim;
        const bool live = row < a.rows;
        store_piece(static_cast<T *>(a.dx) + (live ? row * a.ld_dx : 0), c, 0, live, piece_dx(x, dy, w, mean, rstd, s1, s2));
    }
    if (!a.parts) return;
    // the rows of a warp by exchange, the warps one after the other in shared memory
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i)
        for (int o = lanes; o < 32; o <<= 1) {
            sums.dw.p[i] = add2(sums.dw.p[i], __shfl_xor_sync(0xffffffffu, sums.dw.p[i], o));
            sums.db.p[i] = add2(sums.db.p[i], __shfl_xor_sync(0xffffffffu, sums.db.p[i], o));
        }
    for (int warp = 0; warp < kLanesThreads / 32; ++warp) {
        if ((int)threadIdx.x / 32 == warp && (int)threadIdx.x % 32 < lanes) {
            const Vec none = zeros(), dw = warp > 0 ? load_piece(total, c, 0, true) : none, db = warp > 0 ? load_piece(total + 32 * kPiece, c, 0, true) : none;
            store_piece(total, c, 0, true, sum_of(sums.dw, dw));
            store_piece(total + 32 * kPiece, c, 0, true, sum_of(sums.db, db));
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

// The sums of four values over a warp, each in the lanes whose bits 4 and 3 are its number: values are traded
// for other values' halves, six exchanges instead of twenty.
__device__ __forceinline__ float traded_sums(const float (&v)[4], int lane) {
    const bool high = lane & 16, odd = lane & 8;
    const float a = (high ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, high ? v[0] : v[2], 16);
    const float b = (high ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, high ? v[1] : v[3], 16);
    float c = (odd ? b : a) + __shfl_xor_sync(0xffffffffu, odd ? a : b, 8);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
    return c;
}

// Longer rows: a group of warps takes two rows at a time, U pieces of each to a thread; even rows lie in shared memory, where
// the next ones are on their way, and are read from there once for the sums and once for dx.  The groups of a block join
// their sums over rows in shared memory, so that one set of them leaves an SM.
constexpr int kPairsAhead = 2;

template <typename T, typename G, int U, bool EVEN, int WARPS>
__global__ void __launch_bounds__(32 * kGroupWarps)
layer_norm_backward_kernel(const NormBackArgs a, int warps) {
    constexpr int N = together(sizeof(T), sizeof(G));
    using AheadX = Slot<T, EVEN>;
    using AheadDy = Slot<G, EVEN>;
    constexpr int kBytes = AheadX::kBytes + AheadDy::kBytes;
    extern __shared__ __align__(16) unsigned char ahead[];  // [pairs ahead][2][U][both pieces of all threads]; at the end two sums of each column
    __shared__ alignas(16) float slots[2][kGroupWarps][4];
    let_next_start();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const Group group(WARPS ? WARPS : warps);
    const Columns<EVEN, N, 32 * WARPS> c = {group.t, 32 * warps, a.dim};
    const T *x0 = static_cast<const T *>(a.x);
    const G *dy0 = static_cast<const G *>(a.dy);
    const int64_t step = (int64_t)gridDim.x * group.count;  // of a group's rows; it takes rows row and row + step together
    int64_t row = (int64_t)blockIdx.x * group.count + group.index;
    const auto slot = [&](int stage, int r, int u) { return ahead + ((stage * 2 + r) * U + u) * (int)blockDim.x * kBytes; };
    const auto send_for = [&](int64_t first, int stage) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int64_t at = first + r * step;
            if (at >= a.rows) continue;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                AheadX::send_for(slot(stage, r, u), x0 + at * a.ld_x, c, u, threadIdx.x, blockDim.x);
                AheadDy::send_for(slot(stage, r, u) + blockDim.x * AheadX::kBytes, dy0 + at * a.ld_dy, c, u, threadIdx.x, blockDim.x);
            }
        }
        copies_end_group();
    };
    float next_mean[2] = {}, next_rstd[2] = {};
    const auto look_up = [&](int64_t first) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int64_t at = first + r * step;
            next_mean[r] = at < a.rows ? a.mean[at] : 0.f;
            next_rstd[r] = at < a.rows ? a.rstd[at] : 0.f;
        }
    };
    if constexpr (EVEN) {
        for (int i = 0; i < kPairsAhead; ++i) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    AheadX::clear(slot(i, r, u), c, u, threadIdx.x, blockDim.x);
                    AheadDy::clear(slot(i, r, u) + blockDim.x * AheadX::kBytes, c, u, threadIdx.x, blockDim.x);
                }
            send_for(row + 2 * i * step, i);
        }
    }
    look_up(row);
    Vec w[U];
    PieceSums sums[U] = {};
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = load_piece(a.weight, c, u, true);
    Piece<T, EVEN> odd_x[EVEN ? 1 : 2][U];
    Piece<G, EVEN> odd_dy[EVEN ? 1 : 2][U];
    // a piece of the pair's row r
    const auto get = [&](int stage, int r, int u, Vec &x, Vec &dy) {
        if constexpr (EVEN) {
            x = AheadX::get(slot(stage, r, u), x0, c, u, threadIdx.x, blockDim.x);
            dy = AheadDy::get(slot(stage, r, u) + blockDim.x * AheadX::kBytes, dy0, c, u, threadIdx.x, blockDim.x);
        } else {
            x = odd_x[r][u].get();
            dy = odd_dy[r][u].get();
        }
    };
    for (int stage = 0, turn = 0; row < a.rows; row += 2 * step, stage = stage + 1 == kPairsAhead ? 0 : stage + 1, turn ^= 1) {
        float mean[2], rstd[2], v[4];
        const bool both = row + step < a.rows;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            mean[r] = next_mean[r];
            rstd[r] = next_rstd[r];
        }
        if constexpr (EVEN) {
            copies_wait<kPairsAhead - 1>();
        } else {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const bool live = r == 0 || both;
                const int64_t at = live ? row + r * step : 0;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    odd_x[r][u].load(x0 + at * a.ld_x, c, u, live);
                    odd_dy[r][u].load(dy0 + at * a.ld_dy, c, u, live);
                }
            }
        }
        look_up(row + 2 * step);
        v[2] = v[3] = 0.f;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (r == 1 && !both) continue;
            Pair p1 = 0, p2 = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                Vec x, dy;
                get(stage, r, u, x, dy);
                take_piece(x, dy, w[u], mean[r], rstd[r], sums[u], p1, p2);
            }
            v[2 * r] = pair_sum(p1);
            v[2 * r + 1] = pair_sum(p2);
        }
        if (a.dx) {
            const float mine = traded_sums(v, lane);
            if (lane % 8 == 0) slots[turn][warp][lane / 8] = mine;
            group.sync();
            float4 all = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
            for (int i = 0; i < warps; ++i) {
                const float4 q = *reinterpret_cast<const float4 *>(slots[turn][group.index * warps + i]);
                all.x += q.x;
                all.y += q.y;
                all.z += q.z;
                all.w += q.w;
            }
            const float m1[2] = {all.x * a.inv_dim, all.z * a.inv_dim}, m2[2] = {all.y * a.inv_dim, all.w * a.inv_dim};
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (r == 1 && !both) continue;
                T *dx = static_cast<T *>(a.dx) + (row + r * step) * a.ld_dx;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    Vec x, dy;
                    get(stage, r, u, x, dy);
                    store_piece(dx, c, u, true, piece_dx(x, dy, w[u], mean[r], rstd[r], m1[r], m2[r]));
                }
            }
        }
        if constexpr (EVEN) send_for(row + 2 * kPairsAhead * step, stage);  // behind the last use of what was there
    }
    if (!a.parts) return;
    const int64_t pad = padded(a.dim);
    float *part = a.parts + (int64_t)blockIdx.x * 2 * pad, *joined = reinterpret_cast<float *>(ahead);
    __syncthreads();  // all copies have been waited for by those who sent for them
    for (int q = 0; q < group.count; ++q) {
        if (q == group.index) {
            const bool last = q + 1 == group.count;
            float *to = last ? part : joined;
#pragma unroll
            for (int u = 0; u < U; ++u) {  // the last group brings the sums out
                Vec dw = sums[u].dw, db = sums[u].db;
                if (q > 0) {
                    dw = sum_of(dw, load_piece(joined, c, u, true));
                    db = sum_of(db, load_piece(joined + pad, c, u, true));
                }
                store_piece(to, c, u, true, dw);
                store_piece(to + pad, c, u, true, db);
            }
        }
        if (q + 1 < group.count) __syncthreads();
    }
}

// Rows too long for that: the two sums of each row first, then columns by the tile, an element to an access; x and dy are
// read twice.  2048 x 12288 bf16 136 us (floor 23), fp32 153 (46); 2048 x 14336 bf16 154 (27).
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
            if (a.dx) dx0[row * a.ld_dx + c] = narrow<T>(rstd * (g * w[i] - fmaf(xhat, s.y, s.x)));
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
constexpr int kJoinLoads = 10;  // of a thread, together: those of 148 blocks at once

__global__ void __launch_bounds__(32 * kJoinWarps)
layer_norm_join_kernel(const NormBackArgs a, int parts) {
    __shared__ float slots[kJoinWarps][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const bool of_bias = blockIdx.y == 1;
    const int c = blockIdx.x * 32 + lane;
    float *g = of_bias ? a.dbias : a.dweight, *m = of_bias ? a.m_bias : a.m_weight, *v = of_bias ? a.v_bias : a.v_weight;
    const bool writes = warp == 0 && c < a.dim;
    float m_c = 0.f, v_c = 0.f;
    if (m && writes) m_c = __ldcg(m + c), v_c = __ldcg(v + c);  // what the kernel before this one leaves alone
    wait_for_previous();
    const int64_t pad = padded(a.dim);
    const float *from = a.parts + (of_bias ? pad : 0) + min(c, a.dim - 1);
    float s = 0.f;
    for (int first = warp; first < parts; first += kJoinLoads * kJoinWarps) {
        float q[kJoinLoads];  // (of a part that there is, and used or not: a load with a condition would wait for the one before)
#pragma unroll
        for (int j = 0; j < kJoinLoads; ++j) q[j] = __ldcg(from + (int64_t)min(first + j * kJoinWarps, parts - 1) * 2 * pad);
#pragma unroll
        for (int j = 0; j < kJoinLoads; ++j) s += first + j * kJoinWarps < parts ? q[j] : 0.f;
    }
    slots[warp][lane] = s;
    __syncthreads();
    if (!writes) return;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < kJoinWarps; ++i) s += slots[i][lane];
    if (g) g[c] = s;
    if (m) {
        fold1(s, m_c, v_c, a.fold.a, a.fold.b);
        m[c] = m_c;
        v[c] = v_c;
    }
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

template <typename T, typename O, int U, bool EVEN, int WARPS>
cudaError_t forward_groups(const NormArgs &a, const RowPlan &p, int sm_count, cudaStream_t stream) {
    const int threads = 32 * p.warps * p.groups;
    const size_t params = EVEN ? (size_t)64 * U * 32 * p.warps : (size_t)8 * a.dim;
    const size_t shared = params + (EVEN ? (size_t)kAhead * U * Piece<T, true>::kUnits * threads * 16 : 0);
    if (shared > 40 * 1024) {  // with the static part, more than a kernel has unasked
        static std::atomic<unsigned long long> ready{0};
        const cudaError_t e = allow_shared(layer_norm_kernel<T, O, U, EVEN, WARPS>, 200 * 1024, ready);
        if (e != cudaSuccess) return e;
    }
    const unsigned grid = grid_for((size_t)a.rows, (size_t)p.groups, sm_count, 1);
    layer_norm_kernel<T, O, U, EVEN, WARPS><<<grid, threads, shared, stream>>>(a, p.warps);
    return cudaGetLastError();
}

// Pieces to a thread and warps to a row: as many pieces as leave every SM eight warps, up to `most`; warps rounded up to
// a power of two where the compiler has to know them.  (With 8, 4 and 2 pieces, bf16: 16384 x 4096 48, 56 and 72 us; 8192 x 1024 13.0,
// 11.0 and 11.7, taken 4; 30000 x 512 28, 21 and 16, taken 2; 700 x 4096 6.9, 6.2 and 6.9.)
RowPlan plan_rows(int64_t rows, int pieces, int sm_count, int most, bool power) {
    RowPlan p;
    p.pieces = pieces;
    const auto warps_with = [&](int each) {
        int w = (pieces + 32 * each - 1) / (32 * each);
        while (power && (w & (w - 1))) ++w;
        return w;
    };
    p.each = most;
    while (p.each > 1 && (pieces <= 16 * p.each || rows * warps_with(p.each) < 8 * (int64_t)sm_count) && warps_with(p.each / 2) <= kGroupWarps)
        p.each /= 2;
    p.warps = warps_with(p.each);
    p.groups = 1;
    return p;
}

constexpr int most_even(size_t size) { return size == 2 ? 8 : 4; }  // pieces of even rows to a thread, x's elements of that size
constexpr int kMostOdd = 4;

template <typename T, typename O>
cudaError_t forward_even(const NormArgs &a, RowPlan &p, int sm_count, cudaStream_t stream) {
    if constexpr (most_even(sizeof(T)) == 8) {
        if (p.each == 8) return forward_groups<T, O, 8, true, 0>(a, p, sm_count, stream);
    }
    switch (p.each) {
        case 4: return forward_groups<T, O, 4, true, 0>(a, p, sm_count, stream);
        case 2: return forward_groups<T, O, 2, true, 0>(a, p, sm_count, stream);
        default: return forward_groups<T, O, 1, true, 0>(a, p, sm_count, stream);
    }
}
// (rows here have over 32 pieces and up to kLongPieces: one piece to a thread takes two warps at least, four take eight at most)
template <typename T, typename O, int U>
cudaError_t forward_odd(const NormArgs &a, RowPlan &p, int sm_count, cudaStream_t stream) {
    if constexpr (U > 1) {
        if (p.warps == 1) return forward_groups<T, O, U, false, 1>(a, p, sm_count, stream);
    }
    if constexpr (kLongPieces > 32 * 8 * U) {
        if (p.warps == 16) return forward_groups<T, O, U, false, 16>(a, p, sm_count, stream);
    }
    switch (p.warps) {
        case 2: return forward_groups<T, O, U, false, 2>(a, p, sm_count, stream);
        case 4: return forward_groups<T, O, U, false, 4>(a, p, sm_count, stream);
        default: return forward_groups<T, O, U, false, 8>(a, p, sm_count, stream);
    }
}

template <typename T, typename O>
cudaError_t forward(const NormArgs &a, int sm_count, cudaStream_t stream) {
    const int pieces = (int)(padded(a.dim) / kPiece);
    constexpr int N = together(sizeof(T), sizeof(O));
    const bool even = even_rows(a.x, a.dim, a.ld_x, sizeof(T), N) && even_rows(a.y, a.dim, a.ld_y, sizeof(O), N) && aligned(a.weight, 16) &&
                      aligned(a.bias, 16);
    if (pieces <= 32) {
        const int lanes = lanes_for(pieces), rows = kShortThreads / lanes;
        const unsigned grid = (unsigned)((a.rows + rows - 1) / rows);
        if (even) layer_norm_short_kernel<T, O, true><<<grid, kShortThreads, 0, stream>>>(a, lanes);
        else layer_norm_short_kernel<T, O, false><<<grid, kShortThreads, 0, stream>>>(a, lanes);
        return cudaGetLastError();
    }
    if (pieces > kLongPieces) {
        layer_norm_long_kernel<T, O><<<(unsigned)a.rows, kLongThreads, 0, stream>>>(a);
        return cudaGetLastError();
    }
    // (uneven: four pieces where there are rows enough for that, else one or two)
    RowPlan p = plan_rows(a.rows, pieces, sm_count, even ? most_even(sizeof(T)) : kMostOdd, !even);
    // rows side by side in a block, as many as its warps and an SM's shared memory have room for
    p.groups = kGroupWarps / p.warps;
    while (p.groups > 1 && a.rows < (int64_t)sm_count * p.groups) p.groups -= 1;
    if (even) return forward_even<T, O>(a, p, sm_count, stream);
    return p.each == 4 ? forward_odd<T, O, 4>(a, p, sm_count, stream)
                       : p.each == 2 ? forward_odd<T, O, 2>(a, p, sm_count, stream) : forward_odd<T, O, 1>(a, p, sm_count, stream);
}

// Blocks of the backward pass, whose sums the workspace holds; behind them two sums of each row where rows are long.
struct BackPlan : RowPlan {
    bool is_long;
    int64_t parts;
};
BackPlan plan_back(int64_t rows, int dim, int sm_count, bool even, bool wide) {
    BackPlan p;
    p.pieces = (int)(padded(dim) / kPiece);
    // two pieces to a thread (16384 x 4096 bf16 75 us, one 102; 32816 x 512 31, 36), one where there are few rows.  (One is better for some
    // rows that two leave places empty in: 4096 x 1600, seven warps of one piece 16.4 us, four of two 17.1.)
    p.each = p.pieces > 32 * kGroupWarps || (even && rows >= 2 * (int64_t)sm_count) ? 2 : 1;
    p.warps = (p.pieces + 32 * p.each - 1) / (32 * p.each);
    while (!even && p.pieces > 32 && (p.warps & (p.warps - 1))) ++p.warps;  // the compiler has to know them
    p.groups = 1;
    p.is_long = p.pieces > kLongPieces;
    int64_t most = sm_count;
    if (p.pieces <= 32) {
        p.groups = kLanesThreads / lanes_for(p.pieces);
        // two to an SM.  Three fit, too (72 to 80 registers), and are better where there are many long rows alone: 60000 x 256 bf16 27.8 us
        // with two, 24.7 with three (one 42, four 32), 65536 x 128 17.4 and 16.2; 23327 x 224 12.4 and 13.4, 15035 x 56 7.3 and 8.3
        most = 2 * (int64_t)sm_count;
    } else if (p.is_long) {
        const int64_t tiles = (dim + kTileColumns * kLanesThreads - 1) / (kTileColumns * kLanesThreads);
        most = (4 * (int64_t)sm_count + tiles - 1) / tiles;
    } else {
        // as many groups to a block as it has warps for (half as many, where even rows in fp32 fill shared memory: 4096 x 4096 38 us, else
        // 57), fewer where that would leave SMs without any
        p.groups = (wide && p.warps <= kGroupWarps / 2 ? kGroupWarps / 2 : kGroupWarps) / p.warps;
        while (p.groups > 1 && rows < (int64_t)sm_count * p.groups) p.groups -= 1;
    }
    p.parts = (rows + p.groups - 1) / p.groups;
    if (p.parts > most) p.parts = most;
    if (p.parts < 1) p.parts = 1;
    return p;
}

constexpr size_t kBackShared = 200 * 1024;
template <typename T, typename G>
size_t bytes_ahead(int each, int threads) {
    return (size_t)kPairsAhead * 2 * each * (Piece<T, true>::kUnits + Piece<G, true>::kUnits) * threads * 16;
}

template <typename T, typename G, int U, bool EVEN, int WARPS>
cudaError_t back_groups(const NormBackArgs &a, const BackPlan &p, cudaStream_t stream) {
    const int threads = 32 * p.warps * p.groups;
    size_t shared = EVEN ? bytes_ahead<T, G>(U, threads) : 0;
    const size_t joined = p.groups > 1 && a.parts ? (size_t)2 * padded(a.dim) * sizeof(float) : 0;
    if (shared < joined) shared = joined;
    if (shared > 40 * 1024) {  // with the static part, more than a kernel has unasked
        static std::atomic<unsigned long long> ready{0};
        const cudaError_t e = allow_shared(layer_norm_backward_kernel<T, G, U, EVEN, WARPS>, kBackShared, ready);
        if (e != cudaSuccess) return e;
    }
    layer_norm_backward_kernel<T, G, U, EVEN, WARPS><<<(unsigned)p.parts, threads, shared, stream>>>(a, p.warps);
    return cudaGetLastError();
}
template <typename T, typename G, bool EVEN>
cudaError_t launch_back(const NormBackArgs &a, const BackPlan &p, cudaStream_t stream) {
    if (p.pieces <= 32) {
        layer_norm_backward_short_kernel<T, G, EVEN><<<(unsigned)p.parts, kLanesThreads, 0, stream>>>(a, lanes_for(p.pieces));
        return cudaGetLastError();
    }
    if constexpr (EVEN) {
        return p.each == 2 ? back_groups<T, G, 2, true, 0>(a, p, stream) : back_groups<T, G, 1, true, 0>(a, p, stream);
    } else {
        if (p.each == 2) return back_groups<T, G, 2, false, 16>(a, p, stream);  // rows of over 512 pieces
        switch (p.warps) {
            case 2: return back_groups<T, G, 1, false, 2>(a, p, stream);
            case 4: return back_groups<T, G, 1, false, 4>(a, p, stream);
            case 8: return back_groups<T, G, 1, false, 8>(a, p, stream);
            default: return back_groups<T, G, 1, false, 16>(a, p, stream);
        }
    }
}

template <typename T, typename G>
cudaError_t backward(const NormBackArgs &a, int sm_count, cudaStream_t stream, int *launches) {
    constexpr int N = together(sizeof(T), sizeof(G));
    bool even = even_rows(a.x, a.dim, a.ld_x, sizeof(T), N) && even_rows(a.dy, a.dim, a.ld_dy, sizeof(G), N) &&
                (!a.dx || even_rows(a.dx, a.dim, a.ld_dx, sizeof(T), N)) && aligned(a.weight, 16);
    BackPlan p = plan_back(a.rows, a.dim, sm_count, even, even && sizeof(T) + sizeof(G) > 4);
    if (even && !p.is_long && p.pieces > 32 && bytes_ahead<T, G>(p.each, 32 * p.warps * p.groups) > kBackShared) {
        even = false;  // the longest rows of fp32 go the other way
        p = plan_back(a.rows, a.dim, sm_count, false, false);
    }
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
    const BackPlan p = plan_back(rows, dim, sm_count, false, false);
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
