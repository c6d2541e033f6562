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

namespace adama {
namespace {

// ---- groups of threads that share a row ---------------------------------------------------------
// Up to 32 lanes of a warp (a power of two), or the whole block.

__device__ __forceinline__ float lanes_sum(float x, int lanes) {
    for (int o = lanes / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// The sums of N values over the row's group, in every thread.
template <bool BLOCK, int N>
__device__ __forceinline__ void group_sums(float (&x)[N], int lanes, float (*slots)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = lanes_sum(x[i], BLOCK ? 32 : lanes);
    if (!BLOCK) return;
    const int lane = threadIdx.x % 32, warps = blockDim.x / 32;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) slots[threadIdx.x / 32][i] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = lanes_sum(lane < warps ? slots[lane][i] : 0.f, 32);
    __syncthreads();
}

__device__ __forceinline__ int piece_count(int column, int dim) {
    return column + kPiece <= dim ? kPiece : column < dim ? dim - column : 0;
}

// ---- forward -------------------------------------------------------------------------------------

// U pieces to a thread.  BLOCK: a row to a block, else to `lanes` lanes of a warp.  Exchanges between lanes are the
// dearest instructions here, and a row takes two chains of them in every warp that shares it: so a lane takes many
// pieces where there are rows enough for all SMs (4096 x 1600 fp32 to bf16: 17.3 us with one piece to a thread, @FWD@).
template <typename T, typename O, int U, bool BLOCK, bool EVEN>
__global__ void __launch_bounds__(BLOCK ? (U <= 2 ? 1024 : 256) : 128)
layer_norm_kernel(const NormArgs a, int lanes) {
    __shared__ float slots[32][1];
    const int width = BLOCK ? (int)blockDim.x : lanes, t = threadIdx.x % width;
    const int64_t row = BLOCK ? blockIdx.x : (int64_t)blockIdx.x * (blockDim.x / lanes) + threadIdx.x / lanes;
    const bool live = row < a.rows;
    const T *x = static_cast<const T *>(a.x);
    const Extent all = extent_of(x, a.rows, a.dim, a.ld_x);
    x += (live ? row : 0) * a.ld_x;
    Piece<T, EVEN> raw[U];
    float v[U][kPiece];
    int count[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = (t + u * width) * kPiece;
        count[u] = live ? piece_count(c, a.dim) : 0;
        raw[u].load(x + c, count[u], all);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u].get(x + (t + u * width) * kPiece, count[u], all, v[u]);
    Pair sums = 0;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < kPiece; i += 2) sums = add2(sums, pair(v[u][i], v[u][i + 1]));
    float s[1], other;
    split(sums, s[0], other);
    s[0] += other;
    group_sums<BLOCK, 1>(s, lanes, slots);
    const float mean = s[0] / (float)a.dim;  // (a product with 1/D would move the mean of equal values)
    sums = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (count[u] != kPiece) {  // elements behind the row: no distance from the mean
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (i >= count[u]) v[u][i] = mean;
        }
#pragma unroll
        for (int i = 0; i < kPiece; i += 2) {
            const Pair d = add2(pair(v[u][i], v[u][i + 1]), pair(-mean, -mean));
            sums = fma2(d, d, sums);
            split(d, v[u][i], v[u][i + 1]);
        }
    }
    split(sums, s[0], other);
    s[0] += other;
    group_sums<BLOCK, 1>(s, lanes, slots);
    const float rstd = 1.f / sqrtf(s[0] / (float)a.dim + a.eps);
    if (t == 0 && live) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    const Extent params_w = {reinterpret_cast<uintptr_t>(a.weight), reinterpret_cast<uintptr_t>(a.weight + a.dim)};
    const Extent params_b = {reinterpret_cast<uintptr_t>(a.bias), reinterpret_cast<uintptr_t>(a.bias + a.dim)};
    O *y = static_cast<O *>(a.y) + (live ? row : 0) * a.ld_y;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = (t + u * width) * kPiece;
        float w[kPiece], b[kPiece];
        Piece<float, EVEN> raw_w, raw_b;
        raw_w.load(a.weight + c, count[u], params_w);
        raw_b.load(a.bias + c, a.bias ? count[u] : 0, params_b);
        raw_w.get(a.weight + c, count[u], params_w, w);
        raw_b.get(a.bias + c, a.bias ? count[u] : 0, params_b, b);
#pragma unroll
        for (int i = 0; i < kPiece; i += 2) {
            const Pair xhat = mul2(pair(v[u][i], v[u][i + 1]), pair(rstd, rstd));
            split(fma2(xhat, pair(w[i], w[i + 1]), pair(b[i], b[i + 1])), v[u][i], v[u][i + 1]);
        }
        store_run<EVEN>(y + c, v[u], count[u], BLOCK ? 32 : lanes);
    }
}

// Rows that no block holds in registers: read three times, from L2 if they stay there.
constexpr int kLongThreads = 512;

template <typename T, typename O>
__global__ void __launch_bounds__(kLongThreads)
layer_norm_long_kernel(const NormArgs a) {
    __shared__ float slots[32][1];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x);
    const Extent all = extent_of(x, a.rows, a.dim, a.ld_x);
    x += row * a.ld_x;
    constexpr int kStep = kLongThreads * kPiece;
    const int first = threadIdx.x * kPiece;
    float s[1] = {0.f}, v[kPiece];
    for (int64_t c = first; c < a.dim; c += kStep) {
        load_piece<false>(x + c, piece_count((int)c, a.dim), all, v);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) s[0] += v[i];
    }
    group_sums<true, 1>(s, 32, slots);
    const float mean = s[0] / (float)a.dim;  // (a product with 1/D would move the mean of equal values)
    s[0] = 0.f;
    for (int64_t c = first; c < a.dim; c += kStep) {
        const int count = piece_count((int)c, a.dim);
        load_piece<false>(x + c, count, all, v);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            const float d = i < count ? v[i] - mean : 0.f;
            s[0] = fmaf(d, d, s[0]);
        }
    }
    group_sums<true, 1>(s, 32, slots);
    const float rstd = 1.f / sqrtf(s[0] / (float)a.dim + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    O *y = static_cast<O *>(a.y) + row * a.ld_y;
    const Extent params_w = {reinterpret_cast<uintptr_t>(a.weight), reinterpret_cast<uintptr_t>(a.weight + a.dim)};
    const Extent params_b = {reinterpret_cast<uintptr_t>(a.bias), reinterpret_cast<uintptr_t>(a.bias + a.dim)};
    for (int64_t c0 = 0; c0 < a.dim; c0 += kStep) {  // whole warps: they store together
        const int64_t c = c0 + first;
        const int count = c < a.dim ? piece_count((int)c, a.dim) : 0;
        float w[kPiece], b[kPiece] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        load_piece<false>(x + c, count, all, v);
        load_piece<false>(a.weight + c, count, params_w, w);
        if (a.bias) load_piece<false>(a.bias + c, count, params_b, b);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[i] = fmaf((v[i] - mean) * rstd, w[i], b[i]);
        store_run<false>(y + c, v, count, 32);
    }
}

// ---- backward ------------------------------------------------------------------------------------

// A block's sums in the workspace: dweight, then dbias, each padded to whole pieces.
__host__ __device__ inline int64_t padded(int dim) { return ((int64_t)dim + kPiece - 1) / kPiece * kPiece; }

// The sums of N values (2 or 4) over a warp, each in the lanes whose upper bits are its number: values are
// traded for other values' halves, six exchanges instead of twenty for four of them.
template <int N>
__device__ __forceinline__ float traded_sums(const float (&v)[N], int lane) {
    static_assert(N == 2 || N == 4, "values");
    const bool high = lane & 16, odd = lane & 8;
    float c = (high ? v[N / 2] : v[0]) + __shfl_xor_sync(0xffffffffu, high ? v[0] : v[N / 2], 16);
    if (N == 4) {
        const float b = (high ? v[N - 1] : v[1]) + __shfl_xor_sync(0xffffffffu, high ? v[1] : v[N - 1], 16);
        c = (odd ? b : c) + __shfl_xor_sync(0xffffffffu, odd ? c : b, 8);
    } else {
        c += __shfl_xor_sync(0xffffffffu, c, 8);
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
    return c;
}

// Sums over rows, of a thread's columns.
struct PieceSums {
    Pair dw[kPiece / 2], db[kPiece / 2];
};

__device__ __forceinline__ Pair xhat_of(float x0, float x1, float mean, float rstd) {
    return mul2(add2(pair(x0, x1), pair(-mean, -mean)), pair(rstd, rstd));
}
// A piece's part in its columns' sums and in its row's two.  Elements behind the row are 0 in dy and add nothing.
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
__device__ __forceinline__ void store_sums(float *p, const Pair (&v)[kPiece / 2], bool add) {
    float4 q[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        q[h] = add ? reinterpret_cast<const float4 *>(p)[h] : make_float4(0.f, 0.f, 0.f, 0.f);
        float a, b;
        split(v[2 * h], a, b);
        q[h].x += a;
        q[h].y += b;
        split(v[2 * h + 1], a, b);
        q[h].z += a;
        q[h].w += b;
        reinterpret_cast<float4 *>(p)[h] = q[h];
    }
}

// Rows of up to 256 elements: `lanes` lanes to a row, one piece to a lane.
constexpr int kLanesThreads = 256;

template <typename T, typename G, bool EVEN>
__global__ void __launch_bounds__(kLanesThreads)
layer_norm_backward_lanes_kernel(const NormBackArgs a, int lanes) {
    __shared__ alignas(16) float total[2 * 32 * kPiece];
    let_next_start();
    const int t = threadIdx.x % lanes, groups = kLanesThreads / lanes, c = t * kPiece, count = piece_count(c, a.dim);
    const T *x0 = static_cast<const T *>(a.x);
    const G *dy0 = static_cast<const G *>(a.dy);
    const Extent x_all = extent_of(x0, a.rows, a.dim, a.ld_x), dy_all = extent_of(dy0, a.rows, a.dim, a.ld_dy);
    const Extent params_w = {reinterpret_cast<uintptr_t>(a.weight), reinterpret_cast<uintptr_t>(a.weight + a.dim)};
    float w[kPiece];
    load_piece<EVEN>(a.weight + c, count, params_w, w);
    PieceSums sums = {};
    // all lanes of a warp go round together, the last rows of some being none
    for (int64_t base = (int64_t)blockIdx.x * groups; base < a.rows; base += (int64_t)gridDim.x * groups) {
        const int64_t row = base + threadIdx.x / lanes;
        const bool live = row < a.rows;
        const int n = live ? count : 0;
        float x[kPiece], dy[kPiece];
        Piece<T, EVEN> raw_x;
        Piece<G, EVEN> raw_dy;
        const T *px = x0 + (live ? row * a.ld_x : 0) + c;
        const G *pdy = dy0 + (live ? row * a.ld_dy : 0) + c;
        raw_x.load(px, n, x_all);
        raw_dy.load(pdy, n, dy_all);
        const float mean = live ? a.mean[row] : 0.f, rstd = live ? a.rstd[row] : 0.f;
        raw_x.get(px, n, x_all, x);
        raw_dy.get(pdy, n, dy_all, dy);
        Pair p1 = 0, p2 = 0;
        take_piece(x, dy, w, mean, rstd, sums, p1, p2);
        if (!a.dx) continue;
        float s1, s2, other;
        split(p1, s1, other);
        s1 = lanes_sum(s1 + other, lanes) * a.inv_dim;
        split(p2, s2, other);
        s2 = lanes_sum(s2 + other, lanes) * a.inv_dim;
        float dx[kPiece];
        piece_dx(x, dy, w, mean, rstd, s1, s2, dx);
        store_run<EVEN>(static_cast<T *>(a.dx) + (live ? row * a.ld_dx : 0) + c, dx, n, lanes);
    }
    if (!a.parts) return;
    // the rows of a warp by exchange, the warps one after the other in shared memory
    const int cols = lanes * kPiece;
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i)
        for (int o = lanes; o < 32; o <<= 1) {
            sums.dw[i] = add2(sums.dw[i], __shfl_xor_sync(0xffffffffu, sums.dw[i], o));
            sums.db[i] = add2(sums.db[i], __shfl_xor_sync(0xffffffffu, sums.db[i], o));
        }
    for (int warp = 0; warp < kLanesThreads / 32; ++warp) {
        if ((int)threadIdx.x / 32 == warp && (int)threadIdx.x % 32 < lanes) {
            store_sums(total + c, sums.dw, warp > 0);
            store_sums(total + cols + c, sums.db, warp > 0);
        }
        __syncthreads();
    }
    const int64_t pad = padded(a.dim);
    float *part = a.parts + (int64_t)blockIdx.x * 2 * pad;
    for (int i = threadIdx.x; i < a.dim; i += kLanesThreads) {
        part[i] = total[i];
        part[pad + i] = total[cols + i];
    }
}

// Longer rows: W warps to a row, two pieces to a thread, of ROWS rows at a time; the groups of a block join their sums
// in shared memory, so that one set of them leaves an SM.
constexpr int kBackPieces = 2;     // U
constexpr int kBackWarps = 16;     // of a block

template <typename T, typename G, int ROWS, bool EVEN>
__global__ void __launch_bounds__(32 * kBackWarps)
layer_norm_backward_kernel(const NormBackArgs a, int warps) {
    constexpr int U = kBackPieces;
    extern __shared__ __align__(16) float joined[];  // two sums of each column, where a block has several groups
    __shared__ alignas(16) float slots[2][kBackWarps][2 * ROWS];
    let_next_start();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, group = warp / warps, groups = (int)blockDim.x / 32 / warps;
    const int width = 32 * warps, t = threadIdx.x - group * width;
    const T *x0 = static_cast<const T *>(a.x);
    const G *dy0 = static_cast<const G *>(a.dy);
    const Extent x_all = extent_of(x0, a.rows, a.dim, a.ld_x), dy_all = extent_of(dy0, a.rows, a.dim, a.ld_dy);
    const Extent params_w = {reinterpret_cast<uintptr_t>(a.weight), reinterpret_cast<uintptr_t>(a.weight + a.dim)};
    float w[U][kPiece];
    PieceSums sums[U] = {};
    int count[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = (t + u * width) * kPiece;
        count[u] = piece_count(c, a.dim);
        load_piece<EVEN>(a.weight + c, count[u], params_w, w[u]);
    }
    const int64_t stride = (int64_t)gridDim.x * groups;
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * groups + group; row < a.rows; row += ROWS * stride, turn ^= 1) {
        Piece<T, EVEN> raw_x[ROWS][U];
        Piece<G, EVEN> raw_dy[ROWS][U];
        const T *px[ROWS];
        const G *pdy[ROWS];
        float mean[ROWS], rstd[ROWS], v[2 * ROWS];
        bool live[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int64_t at = row + r * stride;
            live[r] = at < a.rows;
            px[r] = x0 + (live[r] ? at * a.ld_x : 0) + t * kPiece;
            pdy[r] = dy0 + (live[r] ? at * a.ld_dy : 0) + t * kPiece;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                raw_x[r][u].load(px[r] + u * width * kPiece, live[r] ? count[u] : 0, x_all);
                raw_dy[r][u].load(pdy[r] + u * width * kPiece, live[r] ? count[u] : 0, dy_all);
            }
            mean[r] = live[r] ? a.mean[at] : 0.f;
            rstd[r] = live[r] ? a.rstd[at] : 0.f;
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            Pair s1 = 0, s2 = 0;
            float other;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x[kPiece], dy[kPiece];
                raw_x[r][u].get(px[r] + u * width * kPiece, live[r] ? count[u] : 0, x_all, x);
                raw_dy[r][u].get(pdy[r] + u * width * kPiece, live[r] ? count[u] : 0, dy_all, dy);
                take_piece(x, dy, w[u], mean[r], rstd[r], sums[u], s1, s2);
            }
            split(s1, v[2 * r], other);
            v[2 * r] += other;
            split(s2, v[2 * r + 1], other);
            v[2 * r + 1] += other;
        }
        if (!a.dx) continue;
        const float mine = traded_sums(v, lane);
        if (lane % (16 / ROWS) == 0) slots[turn][warp][lane / (16 / ROWS)] = mine;
        if (warps == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(width) : "memory");
        float all[2 * ROWS] = {};
        for (int i = 0; i < warps; ++i) {
#pragma unroll
            for (int q = 0; q < 2 * ROWS; ++q) all[q] += slots[turn][group * warps + i][q];
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            T *dx = static_cast<T *>(a.dx) + (live[r] ? (row + r * stride) * a.ld_dx : 0) + t * kPiece;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x[kPiece], dy[kPiece], out[kPiece];
                raw_x[r][u].get(px[r] + u * width * kPiece, live[r] ? count[u] : 0, x_all, x);
                raw_dy[r][u].get(pdy[r] + u * width * kPiece, live[r] ? count[u] : 0, dy_all, dy);
                piece_dx(x, dy, w[u], mean[r], rstd[r], all[2 * r] * a.inv_dim, all[2 * r + 1] * a.inv_dim, out);
                store_run<EVEN>(dx + u * width * kPiece, out, live[r] ? count[u] : 0, 32);
            }
        }
    }
    if (!a.parts) return;
    const int64_t pad = padded(a.dim);
    float *part = a.parts + (int64_t)blockIdx.x * 2 * pad;
    for (int q = 0; q < groups; ++q) {
        if (q == group) {
            float *to = q + 1 == groups ? part : joined;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t c = (int64_t)(t + u * width) * kPiece;
                if (count[u] == 0) continue;
                if (q > 0 && q + 1 == groups) {  // the last one brings them out
#pragma unroll
                    for (int i = 0; i < kPiece / 2; ++i) {
                        const float2 dw = *reinterpret_cast<const float2 *>(joined + c + 2 * i);
                        const float2 db = *reinterpret_cast<const float2 *>(joined + pad + c + 2 * i);
                        sums[u].dw[i] = add2(sums[u].dw[i], pair(dw.x, dw.y));
                        sums[u].db[i] = add2(sums[u].db[i], pair(db.x, db.y));
                    }
                }
                const bool add = q > 0 && q + 1 < groups;
                store_sums(to + c, sums[u].dw, add);
                store_sums(to + pad + c, sums[u].db, add);
            }
        }
        if (q + 1 < groups) __syncthreads();
    }
}

// Rows too long for that: the two sums of each row first, then columns by the tile.
template <typename T, typename G>
__global__ void __launch_bounds__(kLongThreads)
layer_norm_row_sums_kernel(const NormBackArgs a, float2 *sums) {
    __shared__ float slots[32][2];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x);
    const G *dy = static_cast<const G *>(a.dy);
    const Extent x_all = extent_of(x, a.rows, a.dim, a.ld_x), dy_all = extent_of(dy, a.rows, a.dim, a.ld_dy);
    const Extent params_w = {reinterpret_cast<uintptr_t>(a.weight), reinterpret_cast<uintptr_t>(a.weight + a.dim)};
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s[2] = {0.f, 0.f};
    for (int64_t c = threadIdx.x * kPiece; c < a.dim; c += kLongThreads * kPiece) {
        const int count = piece_count((int)c, a.dim);
        float v[kPiece], g[kPiece], w[kPiece];
        load_piece<false>(x + row * a.ld_x + c, count, x_all, v);
        load_piece<false>(dy + row * a.ld_dy + c, count, dy_all, g);
        load_piece<false>(a.weight + c, count, params_w, w);
#pragma unroll
        for (int i = 0; i < kPiece; ++i)
            if (i < count) {
                s[0] = fmaf(g[i], w[i], s[0]);
                s[1] = fmaf(g[i] * w[i], (v[i] - mean) * rstd, s[1]);
            }
    }
    group_sums<true, 2>(s, 32, slots);
    if (threadIdx.x == 0) sums[row] = make_float2(s[0] * a.inv_dim, s[1] * a.inv_dim);
}

template <typename T, typename G>
__global__ void __launch_bounds__(kLanesThreads)
layer_norm_tiles_kernel(const NormBackArgs a, const float2 *sums) {
    const int c = (blockIdx.x * kLanesThreads + threadIdx.x) * kPiece, count = piece_count(c, a.dim);
    const T *x0 = static_cast<const T *>(a.x);
    const G *dy0 = static_cast<const G *>(a.dy);
    const Extent x_all = extent_of(x0, a.rows, a.dim, a.ld_x), dy_all = extent_of(dy0, a.rows, a.dim, a.ld_dy);
    const Extent params_w = {reinterpret_cast<uintptr_t>(a.weight), reinterpret_cast<uintptr_t>(a.weight + a.dim)};
    float w[kPiece], dw[kPiece], db[kPiece];
    load_piece<false>(a.weight + c, count, params_w, w);
#pragma unroll
    for (int i = 0; i < kPiece; ++i) dw[i] = db[i] = 0.f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        float x[kPiece], g[kPiece], out[kPiece];
        load_piece<false>(x0 + row * a.ld_x + c, count, x_all, x);
        load_piece<false>(dy0 + row * a.ld_dy + c, count, dy_all, g);
        const float mean = a.mean[row], rstd = a.rstd[row];
        const float2 s = a.dx ? sums[row] : make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            const float xhat = (x[i] - mean) * rstd;
            db[i] += g[i];
            dw[i] = fmaf(g[i], xhat, dw[i]);
            out[i] = rstd * (g[i] * w[i] - fmaf(xhat, s.y, s.x));
        }
        if (a.dx) store_run<false>(static_cast<T *>(a.dx) + row * a.ld_dx + c, out, count, 32);
    }
    if (!a.parts) return;
    float *part = a.parts + (int64_t)blockIdx.y * 2 * padded(a.dim);
#pragma unroll
    for (int i = 0; i < kPiece; ++i)
        if (i < count) {
            part[c + i] = dw[i];
            part[padded(a.dim) + c + i] = db[i];
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

template <typename T, typename O, int U, bool EVEN>
void forward_rows(const NormArgs &a, int pieces, cudaStream_t stream) {
    const int warps = (pieces + 32 * U - 1) / (32 * U);
    if (warps == 1) layer_norm_kernel<T, O, U, false, EVEN><<<(unsigned)((a.rows + 3) / 4), 128, 0, stream>>>(a, 32);
    else layer_norm_kernel<T, O, U, true, EVEN><<<(unsigned)a.rows, 32 * warps, 0, stream>>>(a, 32);
}

template <typename T, typename O, bool EVEN>
cudaError_t forward(const NormArgs &a, int sm_count, cudaStream_t stream) {
    const int pieces = (int)(padded(a.dim) / kPiece);
    // as many pieces to a lane as leave every SM a dozen warps
    const auto enough = [&](int u) { return a.rows * ((pieces + 32 * u - 1) / (32 * u)) >= 12 * (int64_t)sm_count; };
    if (pieces <= 32) {
        const int lanes = lanes_for(pieces), rows = 128 / lanes;
        layer_norm_kernel<T, O, 1, false, EVEN><<<(unsigned)((a.rows + rows - 1) / rows), 128, 0, stream>>>(a, lanes);
    } else if (pieces > 2048) {
        layer_norm_long_kernel<T, O><<<(unsigned)a.rows, kLongThreads, 0, stream>>>(a);
    } else if (EVEN && pieces > 128 && enough(8)) {
        forward_rows<T, O, EVEN ? 8 : 4, EVEN>(a, pieces, stream);
    } else if (pieces > 64 && pieces <= 1024 && enough(4)) {
        forward_rows<T, O, 4, EVEN>(a, pieces, stream);
    } else if (pieces > 1024 || enough(2)) {
        forward_rows<T, O, 2, EVEN>(a, pieces, stream);
    } else {
        forward_rows<T, O, 1, EVEN>(a, pieces, stream);
    }
    return cudaGetLastError();
}
template <typename T, typename O>
cudaError_t forward(const NormArgs &a, int sm_count, cudaStream_t stream) {
    const bool even = even_rows(a.x, a.dim, a.ld_x, sizeof(T)) && even_rows(a.y, a.dim, a.ld_y, sizeof(O)) && aligned(a.weight, 16) &&
                      aligned(a.bias, 16);
    return even ? forward<T, O, true>(a, sm_count, stream) : forward<T, O, false>(a, sm_count, stream);
}

// Blocks of the backward pass, whose sums the workspace holds; behind them two sums of each row where rows are long.
struct BackPlan {
    int pieces, warps, groups;  // warps to a row, rows side by side in a block
    bool is_long;
    int64_t parts;
    size_t shared;
};
BackPlan plan_back(int64_t rows, int dim, int sm_count) {
    BackPlan p;
    p.pieces = (int)(padded(dim) / kPiece);
    p.warps = (p.pieces + 32 * kBackPieces - 1) / (32 * kBackPieces);
    p.groups = 1;
    p.is_long = p.warps > kBackWarps;
    p.shared = 0;
    int64_t most = sm_count;
    if (p.pieces <= 32) {
        p.groups = kLanesThreads / lanes_for(p.pieces);
        most = 4 * (int64_t)sm_count;
    } else if (p.is_long) {
        const int64_t tiles = (p.pieces + kLanesThreads - 1) / kLanesThreads;
        most = (4 * (int64_t)sm_count + tiles - 1) / tiles;
    } else {
        // as many rows to a block as it has warps for, fewer where that would leave SMs without any
        p.groups = kBackWarps / p.warps;
        while (p.groups > 1 && rows < (int64_t)sm_count * p.groups) p.groups -= 1;
        if (p.groups > 1) p.shared = (size_t)2 * padded(dim) * sizeof(float);
    }
    p.parts = (rows + p.groups - 1) / p.groups;
    if (p.parts > most) p.parts = most;
    if (p.parts < 1) p.parts = 1;
    return p;
}

template <typename T, typename G, bool EVEN>
void launch_back(const NormBackArgs &a, const BackPlan &p, cudaStream_t stream) {
    // two rows at a time where their pieces leave registers for it
    constexpr int kRows = EVEN && sizeof(T) == 2 && sizeof(G) == 2 ? 2 : 1;
    const unsigned grid = (unsigned)p.parts;
    if (p.pieces <= 32) layer_norm_backward_lanes_kernel<T, G, EVEN><<<grid, kLanesThreads, 0, stream>>>(a, lanes_for(p.pieces));
    else layer_norm_backward_kernel<T, G, kRows, EVEN><<<grid, 32 * p.warps * p.groups, p.shared, stream>>>(a, p.warps);
}

template <typename T, typename G>
cudaError_t backward(const NormBackArgs &a, int sm_count, cudaStream_t stream, int *launches) {
    const BackPlan p = plan_back(a.rows, a.dim, sm_count);
    const unsigned grid = (unsigned)p.parts;
    if (a.rows > 0) {
        if (p.is_long) {
            float2 *sums = reinterpret_cast<float2 *>(static_cast<float *>(a.workspace) + p.parts * 2 * padded(a.dim));
            if (a.dx) layer_norm_row_sums_kernel<T, G><<<(unsigned)a.rows, kLongThreads, 0, stream>>>(a, sums);
            const dim3 tiles((unsigned)((p.pieces + kLanesThreads - 1) / kLanesThreads), grid);
            layer_norm_tiles_kernel<T, G><<<tiles, kLanesThreads, 0, stream>>>(a, sums);
        } else {
            const bool even = even_rows(a.x, a.dim, a.ld_x, sizeof(T)) && even_rows(a.dy, a.dim, a.ld_dy, sizeof(G)) &&
                              (!a.dx || even_rows(a.dx, a.dim, a.ld_dx, sizeof(T))) && aligned(a.weight, 16);
            if (even) launch_back<T, G, true>(a, p, stream);
            else launch_back<T, G, false>(a, p, stream);
        }
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        *launches += p.is_long && a.dx ? 2 : 1;
    }
    if (a.parts) {
        const dim3 columns((unsigned)((a.dim + 31) / 32), 2);
        const int parts = a.rows > 0 ? (int)grid : 0;
        // (without a kernel of this call in front, in plain order)
        const cudaError_t e = a.rows > 0 ? launch_chained(layer_norm_join_kernel, columns, dim3(32 * kJoinWarps), 0, stream, a, parts)
                                         : (layer_norm_join_kernel<<<columns, 32 * kJoinWarps, 0, stream>>>(a, parts), cudaGetLastError());
        *launches += 1;
        return e;
    }
    return cudaSuccess;
}

}  // namespace

size_t norm_workspace_bytes(int64_t rows, int dim, int sm_count) {
    const BackPlan p = plan_back(rows, dim, sm_count);
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
