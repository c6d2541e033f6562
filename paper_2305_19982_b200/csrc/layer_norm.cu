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
#include "row_access.cuh"

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

template <typename T, typename O, int U, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? 1024 : 128)
layer_norm_kernel(const NormArgs a, int lanes) {
    __shared__ float slots[32][1];
    const int width = BLOCK ? (int)blockDim.x : lanes, t = threadIdx.x % width;
    const int64_t row = BLOCK ? blockIdx.x : (int64_t)blockIdx.x * (blockDim.x / lanes) + threadIdx.x / lanes;
    const bool live = row < a.rows;
    const T *x = static_cast<const T *>(a.x);
    const Extent all = extent_of(x, a.rows, a.dim, a.ld_x);
    x += (live ? row : 0) * a.ld_x;
    float v[U][kPiece];
    int count[U];
    float s[1] = {0.f};
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = (t + u * width) * kPiece;
        count[u] = live ? piece_count(c, a.dim) : 0;
        load_piece(x + c, count[u], all, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < kPiece; ++i) s[0] += v[u][i];
    group_sums<BLOCK, 1>(s, lanes, slots);
    const float mean = s[0] / (float)a.dim;  // (a product with 1/D would move the mean of equal values)
    s[0] = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            const float d = i < count[u] ? v[u][i] - mean : 0.f;
            v[u][i] = d;
            s[0] = fmaf(d, d, s[0]);
        }
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
        float w[kPiece], b[kPiece] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        load_piece(a.weight + c, count[u], params_w, w);
        if (a.bias) load_piece(a.bias + c, count[u], params_b, b);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[u][i] = fmaf(v[u][i] * rstd, w[i], b[i]);
        store_run(y + c, v[u], count[u], BLOCK ? 32 : lanes);
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
        load_piece(x + c, piece_count((int)c, a.dim), all, v);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) s[0] += v[i];
    }
    group_sums<true, 1>(s, 32, slots);
    const float mean = s[0] / (float)a.dim;  // (a product with 1/D would move the mean of equal values)
    s[0] = 0.f;
    for (int64_t c = first; c < a.dim; c += kStep) {
        const int count = piece_count((int)c, a.dim);
        load_piece(x + c, count, all, v);
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
        load_piece(x + c, count, all, v);
        load_piece(a.weight + c, count, params_w, w);
        if (a.bias) load_piece(a.bias + c, count, params_b, b);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[i] = fmaf((v[i] - mean) * rstd, w[i], b[i]);
        store_run(y + c, v, count, 32);
    }
}

// ---- backward ------------------------------------------------------------------------------------

// A block's sums in the workspace: dweight, then dbias, each padded to whole pieces.
__host__ __device__ inline int64_t padded(int dim) { return ((int64_t)dim + kPiece - 1) / kPiece * kPiece; }

constexpr int kLanesThreads = 256;  // of a block whose rows are shared by lanes of a warp

template <typename T, typename G, int U, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? 512 : kLanesThreads)
layer_norm_backward_kernel(const NormBackArgs a, int lanes) {
    __shared__ float slots[32][2];
    const int width = BLOCK ? (int)blockDim.x : lanes, t = threadIdx.x % width;
    const int groups = BLOCK ? 1 : (int)blockDim.x / lanes;
    const T *x0 = static_cast<const T *>(a.x);
    const G *dy0 = static_cast<const G *>(a.dy);
    const Extent x_all = extent_of(x0, a.rows, a.dim, a.ld_x), dy_all = extent_of(dy0, a.rows, a.dim, a.ld_dy);
    const Extent params_w = {reinterpret_cast<uintptr_t>(a.weight), reinterpret_cast<uintptr_t>(a.weight + a.dim)};
    float w[U][kPiece], dw[U][kPiece], db[U][kPiece];
    int count[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = (t + u * width) * kPiece;
        count[u] = piece_count(c, a.dim);
        load_piece(a.weight + c, count[u], params_w, w[u]);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) dw[u][i] = db[u][i] = 0.f;
    }
    const int64_t step = (int64_t)gridDim.x * groups;
    // all lanes of a warp go round together, the last rows of some being none
    for (int64_t base = (int64_t)blockIdx.x * groups; base < a.rows; base += step) {
        const int64_t row = BLOCK ? base : base + threadIdx.x / lanes;
        const bool live = row < a.rows;
        float x[U][kPiece], g[U][kPiece];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = (t + u * width) * kPiece, n = live ? count[u] : 0;
            load_piece(x0 + (live ? row * a.ld_x : 0) + c, n, x_all, x[u]);
            load_piece(dy0 + (live ? row * a.ld_dy : 0) + c, n, dy_all, g[u]);
        }
        const float mean = live ? a.mean[row] : 0.f, rstd = live ? a.rstd[row] : 0.f;
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                const float xhat = (x[u][i] - mean) * rstd;
                const bool in = live && i < count[u];
                x[u][i] = xhat;
                db[u][i] += g[u][i];
                dw[u][i] = in ? fmaf(g[u][i], xhat, dw[u][i]) : dw[u][i];
                g[u][i] *= w[u][i];
                s[0] += g[u][i];
                s[1] = in ? fmaf(g[u][i], xhat, s[1]) : s[1];
            }
        if (!a.dx) continue;
        group_sums<BLOCK, 2>(s, lanes, slots);
        s[0] *= a.inv_dim;
        s[1] *= a.inv_dim;
        T *dx = static_cast<T *>(a.dx) + (live ? row * a.ld_dx : 0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float out[kPiece];
#pragma unroll
            for (int i = 0; i < kPiece; ++i) out[i] = rstd * (g[u][i] - fmaf(x[u][i], s[1], s[0]));
            store_run(dx + (t + u * width) * kPiece, out, live ? count[u] : 0, BLOCK ? 32 : lanes);
        }
    }
    if (!a.parts) return;
    const int64_t pad = padded(a.dim);
    float *part = a.parts + (int64_t)blockIdx.x * 2 * pad;
    if (BLOCK) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t c = (int64_t)(t + u * width) * kPiece;
            if (count[u] == 0) continue;
            float4 *pw = reinterpret_cast<float4 *>(part + c), *pb = reinterpret_cast<float4 *>(part + pad + c);
            pw[0] = make_float4(dw[u][0], dw[u][1], dw[u][2], dw[u][3]);
            pw[1] = make_float4(dw[u][4], dw[u][5], dw[u][6], dw[u][7]);
            pb[0] = make_float4(db[u][0], db[u][1], db[u][2], db[u][3]);
            pb[1] = make_float4(db[u][4], db[u][5], db[u][6], db[u][7]);
        }
        return;
    }
    // the groups of a warp by exchange, the warps one after the other in shared memory
    __shared__ float total[BLOCK ? 1 : 2 * U * 32 * kPiece];
    const int cols = U * lanes * kPiece;
    for (int i = threadIdx.x; i < 2 * cols; i += blockDim.x) total[i] = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < kPiece; ++i)
            for (int o = lanes; o < 32; o <<= 1) {
                dw[u][i] += __shfl_xor_sync(0xffffffffu, dw[u][i], o);
                db[u][i] += __shfl_xor_sync(0xffffffffu, db[u][i], o);
            }
    for (int warp = 0; warp < (int)blockDim.x / 32; ++warp) {
        __syncthreads();
        if ((int)threadIdx.x / 32 != warp || (int)threadIdx.x % 32 >= lanes) continue;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                total[(t + u * lanes) * kPiece + i] += dw[u][i];
                total[cols + (t + u * lanes) * kPiece + i] += db[u][i];
            }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.dim; i += blockDim.x) {
        part[i] = total[i];
        part[pad + i] = total[cols + i];
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
        load_piece(x + row * a.ld_x + c, count, x_all, v);
        load_piece(dy + row * a.ld_dy + c, count, dy_all, g);
        load_piece(a.weight + c, count, params_w, w);
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
    load_piece(a.weight + c, count, params_w, w);
#pragma unroll
    for (int i = 0; i < kPiece; ++i) dw[i] = db[i] = 0.f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        float x[kPiece], g[kPiece], out[kPiece];
        load_piece(x0 + row * a.ld_x + c, count, x_all, x);
        load_piece(dy0 + row * a.ld_dy + c, count, dy_all, g);
        const float mean = a.mean[row], rstd = a.rstd[row];
        const float2 s = a.dx ? sums[row] : make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            const float xhat = (x[i] - mean) * rstd;
            db[i] += g[i];
            dw[i] = fmaf(g[i], xhat, dw[i]);
            out[i] = rstd * (g[i] * w[i] - fmaf(xhat, s.y, s.x));
        }
        if (a.dx) store_run(static_cast<T *>(a.dx) + row * a.ld_dx + c, out, count, 32);
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

// Pieces of a thread, by the row's length: lanes of a warp share rows of up to 32 pieces, blocks longer ones.
int lanes_for(int pieces) {
    int lanes = 1;
    while (lanes < pieces) lanes *= 2;
    return lanes;
}
constexpr int kBlockPieces = 1024;      // forward: one piece to a thread up to here, two up to twice that
constexpr int kBackBlockPieces = 512;   // backward: the same
constexpr int kJoinParts = 2;           // blocks of the backward pass to an SM, whose sums are joined

template <typename T, typename O>
cudaError_t forward(const NormArgs &a, cudaStream_t stream) {
    const int pieces = (int)(padded(a.dim) / kPiece);
    if (pieces <= 32) {
        const int lanes = lanes_for(pieces), rows = 128 / lanes;
        layer_norm_kernel<T, O, 1, false><<<(unsigned)((a.rows + rows - 1) / rows), 128, 0, stream>>>(a, lanes);
    } else if (pieces <= kBlockPieces) {
        layer_norm_kernel<T, O, 1, true><<<(unsigned)a.rows, (pieces + 31) / 32 * 32, 0, stream>>>(a, 32);
    } else if (pieces <= 2 * kBlockPieces) {
        layer_norm_kernel<T, O, 2, true><<<(unsigned)a.rows, (pieces + 63) / 64 * 32, 0, stream>>>(a, 32);
    } else {
        layer_norm_long_kernel<T, O><<<(unsigned)a.rows, kLongThreads, 0, stream>>>(a);
    }
    return cudaGetLastError();
}

// What the workspace holds: the blocks' sums, behind them two sums of each row where rows are long.
struct BackPlan {
    int pieces;
    bool is_long;
    int64_t parts;
};
BackPlan plan_back(int64_t rows, int dim, int sm_count) {
    BackPlan p;
    p.pieces = (int)(padded(dim) / kPiece);
    p.is_long = p.pieces > 2 * kBackBlockPieces;
    const int64_t most = (int64_t)sm_count * kJoinParts;
    if (p.pieces <= 32) {
        const int groups = kLanesThreads / lanes_for(p.pieces);
        p.parts = (rows + groups - 1) / groups;
    } else {
        p.parts = rows;
    }
    if (p.is_long) {
        const int64_t tiles = (p.pieces + kLanesThreads - 1) / kLanesThreads;
        const int64_t each = (2 * most + tiles - 1) / tiles;
        if (p.parts > each) p.parts = each;
    }
    if (p.parts > most) p.parts = most;
    if (p.parts < 1) p.parts = 1;
    return p;
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
        } else if (p.pieces <= 32) {
            layer_norm_backward_kernel<T, G, 1, false><<<grid, kLanesThreads, 0, stream>>>(a, lanes_for(p.pieces));
        } else if (p.pieces <= kBackBlockPieces) {
            layer_norm_backward_kernel<T, G, 1, true><<<grid, (p.pieces + 31) / 32 * 32, 0, stream>>>(a, 32);
        } else {
            layer_norm_backward_kernel<T, G, 2, true><<<grid, (p.pieces + 63) / 64 * 32, 0, stream>>>(a, 32);
        }
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        *launches += p.is_long && a.dx ? 2 : 1;
    }
    if (a.parts) {
        const dim3 columns((unsigned)((a.dim + 31) / 32), 2);
        layer_norm_join_kernel<<<columns, 32 * kJoinWarps, 0, stream>>>(a, a.rows > 0 ? (int)grid : 0);
        *launches += 1;
    }
    return cudaGetLastError();
}

}  // namespace

size_t norm_workspace_bytes(int64_t rows, int dim, int sm_count) {
    const BackPlan p = plan_back(rows, dim, sm_count);
    return (size_t)p.parts * 2 * padded(dim) * sizeof(float) + (p.is_long ? (size_t)rows * sizeof(float2) : 0);
}

cudaError_t launch_layer_norm(const NormArgs &a, cudaStream_t stream) {
    if (a.x_dtype == ADAMA_F32)
        return a.y_dtype == ADAMA_F32 ? forward<float, float>(a, stream) : forward<float, __nv_bfloat16>(a, stream);
    return a.y_dtype == ADAMA_F32 ? forward<__nv_bfloat16, float>(a, stream) : forward<__nv_bfloat16, __nv_bfloat16>(a, stream);
}

cudaError_t launch_layer_norm_backward(const NormBackArgs &a, int sm_count, cudaStream_t stream, int *launches) {
    if (a.x_dtype == ADAMA_F32)
        return a.dy_dtype == ADAMA_F32 ? backward<float, float>(a, sm_count, stream, launches)
                                       : backward<float, __nv_bfloat16>(a, sm_count, stream, launches);
    return a.dy_dtype == ADAMA_F32 ? backward<__nv_bfloat16, float>(a, sm_count, stream, launches)
                                   : backward<__nv_bfloat16, __nv_bfloat16>(a, sm_count, stream, launches);
}

}  // namespace adama
