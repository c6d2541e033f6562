// Embedding lookup, out[t] = scale*table[ids[t]], and its gradient by sorted tokens:
//     g[i] = scale * sum over the tokens t with ids[t] = i of dy[t]
// written to a whole table (zeros in the other rows), added to one, or folded into the moments of the rows
// that occur (m += a*g, v += b*g^2: the sum is complete before it is squared; a row without tokens has g = 0 and
// is not touched, so that the traffic is that of the tokens, not of the vocabulary).
//
// The tokens are sorted by id, equal ones in their order.  The sorted tokens are cut into chunks; a warp takes
// a chunk's columns 256 at a time and sums equal neighbours in registers, in fp32.  A run of equal tokens that
// lies inside a chunk is finished there; the parts of one that crosses chunks go to the workspace, and a second
// kernel adds them in order; one that only reaches into the next chunk is finished by the warp that has its
// beginning.  So a token that occurs thousands of times is spread over the card like any others, no sum is made by
// atomics (the counts of the sort are, and whole numbers do not care for an order), and results do not depend on scheduling.
//
// The lookup of 16384 x 4096 bf16 takes 32 us = 5.6 TB/s, bound by HBM (7 x 1600: 2.1 us).  Gradients: 32768 x 4096 bf16 into a
// whole bf16 table of 32000 rows 113 us = 4.6 TB/s; 60000 x 1024 fp32 added 92 us = 5.1 TB/s; 4096 x 1600 bf16 folded 24 us =
// 2.8 TB/s: short ones are four or five kernels that wait for each other, each some 4 us long.
#include "adama_device.cuh"
#include "chained.cuh"
#include "row_access.cuh"
#include "row_writer.cuh"
#include "tensor_table.cuh"

namespace adama {
namespace {

constexpr int kTile = 32 * kPiece;  // columns of a warp

// ---- lookup --------------------------------------------------------------------------------------

constexpr int kLookupWarps = 4;
constexpr int kLookupPieces = 4;  // of a lane, all loaded before the first is stored

template <typename T, typename O, bool EVEN>
__global__ void __launch_bounds__(32 * kLookupWarps)
embedding_kernel(const EmbeddingArgs a, int groups) {
    const int lane = threadIdx.x % 32;
    const int64_t task = (int64_t)blockIdx.x * kLookupWarps + threadIdx.x / 32;
    const int64_t token = task / groups;
    const int first = (int)(task - token * groups) * kLookupPieces * kTile;
    if (token >= a.tokens) return;
    const int64_t id = a.ids[token];
    const bool inside = id >= 0 && id < a.vocab;
    const Columns<EVEN, together(sizeof(T), sizeof(O)), 32> c = {lane, 32, a.dim - first};
    const T *row = static_cast<const T *>(a.table) + (inside ? id * a.ld_table : 0) + first;
    O *out = static_cast<O *>(a.out) + token * a.ld_out + first;
    Piece<T, EVEN> raw[kLookupPieces];
#pragma unroll
    for (int u = 0; u < kLookupPieces; ++u) raw[u].load(row, c, u, inside);
    const float other = id < 0 ? 0.f : NAN;
#pragma unroll
    for (int u = 0; u < kLookupPieces; ++u) {
        Vec v = raw[u].get();
#pragma unroll
        for (int i = 0; i < kPiece / 2; ++i) v.p[i] = inside ? mul2(v.p[i], pair(a.scale, a.scale)) : pair(other, other);
        store_piece(out, c, u, true, v);
    }
    if (!inside && id >= 0 && first == 0 && lane == 0) record_bad_target(a.status, token);
}

// ---- sorting by id ---------------------------------------------------------------------------------
// Ids outside the table get the key `vocab` and come last.

__device__ __forceinline__ unsigned key_of(const EmbeddingGradArgs &a, int64_t id) {
    return id >= 0 && id < a.vocab ? (unsigned)id : (unsigned)a.vocab;
}
// Several of a thread's tokens are loaded together, the last token again where there are no more: a load with a condition
// waits for the one before it.

// Up to kRankTokens tokens: a token's place is the number of tokens that come before it, counted over all
// of them.  32 tokens to a block, whose warps share the count.  (The whole gradient by this and by the digits below: 4096 x 1600 of
// 50257 ids 24 and 29 us, 5500 x 256 20 and 20, 8000 x 256 25 and 21; 4096 x 64 of 500 ids, which one pass sorts, 14 and 13.)
constexpr int kRankTokens = 5120;
constexpr int kRankWarps = 16;

__global__ void __launch_bounds__(32 * kRankWarps)
embedding_rank_kernel(const EmbeddingGradArgs a) {
    __shared__ alignas(16) unsigned keys[kRankTokens];
    __shared__ int counts[kRankWarps][32];
    let_next_start();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, tokens = (int)a.tokens;
    const int groups = (tokens + 31) / 32;  // of 32 tokens
    constexpr int kThreads = 32 * kRankWarps, kLoads = 4;
    for (int first = threadIdx.x; first < 32 * groups; first += kLoads * kThreads) {
        int64_t id[kLoads];
#pragma unroll
        for (int q = 0; q < kLoads; ++q) id[q] = a.ids[min(first + q * kThreads, tokens - 1)];
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int i = first + q * kThreads;
            if (i < 32 * groups) keys[i] = i < tokens ? key_of(a, id[q]) : 0xffffffffu;
        }
    }
    __syncthreads();
    const int t = blockIdx.x * 32 + lane;
    const unsigned mine = keys[t];
    int before = 0;
    for (int g = warp; g < groups; g += kRankWarps) {
        if (g != (int)blockIdx.x) {
            const unsigned limit = mine + (g < (int)blockIdx.x ? 1u : 0u);  // equal ones in front count
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const uint4 k = *reinterpret_cast<const uint4 *>(keys + 32 * g + j);
                before += (k.x < limit) + (k.y < limit) + (k.z < limit) + (k.w < limit);
            }
        } else {
            for (int j = 0; j < 32; ++j) before += keys[32 * g + j] < mine + (j < lane ? 1u : 0u);
        }
    }
    counts[warp][lane] = before;
    __syncthreads();
    if (warp != 0 || t >= tokens) return;
    int place = 0;
#pragma unroll
    for (int i = 0; i < kRankWarps; ++i) place += counts[i][lane];
    a.keys[place] = mine;
    a.order[place] = (unsigned)t;
    if (mine == (unsigned)a.vocab && a.ids[t] >= 0) record_bad_target(a.status, t);
}

// More: passes over digits of the key, from the lowest on, each of which keeps the order of equal digits.  A block
// has neighbouring tokens; how many of each digit every block has is counted ahead of a pass (of the first one by a kernel
// of its own, of the others as the tokens get their new places).
constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSortWarps = 8;
constexpr int kSortThreads = 32 * kSortWarps;
constexpr int kSortBlocks = 64;  // at most
constexpr int kSortPasses = 4;   // for keys of 31 bits and the one behind them
constexpr int kRounds = 4;       // of 32 tokens, loaded together

struct SortPass {
    const unsigned *keys, *order;  // null in the first pass: from the ids
    unsigned *keys_out, *order_out;
    int *counts, *next_counts;  // [blocks][digits]; next: null in the last pass
    int shift, next_shift, mask;
    int per;  // tokens of a block, a multiple of kSortThreads
};

// Counts for the first pass; the other passes' counts (`others` ints behind them) become 0.
__global__ void __launch_bounds__(kSortThreads)
embedding_digits_kernel(const EmbeddingGradArgs a, const SortPass p, int *others, int other_ints) {
    __shared__ int counts[kDigits];
    let_next_start();
    for (int i = threadIdx.x; i < kDigits; i += kSortThreads) counts[i] = 0;
    for (int i = blockIdx.x * kSortThreads + threadIdx.x; i < other_ints; i += gridDim.x * kSortThreads) others[i] = 0;
    __syncthreads();
    const int64_t begin = (int64_t)blockIdx.x * p.per, end = begin + p.per < a.tokens ? begin + p.per : a.tokens;
    for (int64_t first = begin + threadIdx.x; first < end; first += kRounds * kSortThreads) {
        int64_t id[kRounds];
#pragma unroll
        for (int q = 0; q < kRounds; ++q) id[q] = a.ids[min(first + q * kSortThreads, end - 1)];
#pragma unroll
        for (int q = 0; q < kRounds; ++q)
            if (first + q * kSortThreads < end) {
                const unsigned key = key_of(a, id[q]);
                atomicAdd(&counts[key >> p.shift & p.mask], 1);
                if (key == (unsigned)a.vocab && id[q] >= 0) record_bad_target(a.status, first + q * kSortThreads);
            }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kDigits; i += kSortThreads) p.counts[blockIdx.x * kDigits + i] = counts[i];
}

__global__ void __launch_bounds__(kSortThreads)
embedding_scatter_kernel(const EmbeddingGradArgs a, const SortPass p) {
    __shared__ int place[kSortWarps][kDigits];  // where a warp's next token of a digit goes
    __shared__ int warp_total[kSortWarps];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int i = threadIdx.x; i < kSortWarps * kDigits; i += kSortThreads) (&place[0][0])[i] = 0;
    let_next_start();
    wait_for_previous();
    __syncthreads();
    const int64_t begin = (int64_t)blockIdx.x * p.per + (int64_t)warp * (p.per / kSortWarps);
    int64_t end = begin + p.per / kSortWarps;
    if (end > a.tokens) end = a.tokens;
    unsigned key[kRounds], token[kRounds];
    const auto load = [&](int64_t base) {
        if (p.keys) {
#pragma unroll
            for (int i = 0; i < kRounds; ++i) {
                const int64_t t = min(base + 32 * i + lane, end - 1);
                key[i] = p.keys[t];
                token[i] = p.order[t];
            }
        } else {
            int64_t id[kRounds];
#pragma unroll
            for (int i = 0; i < kRounds; ++i) id[i] = a.ids[min(base + 32 * i + lane, end - 1)];
#pragma unroll
            for (int i = 0; i < kRounds; ++i) {
                key[i] = key_of(a, id[i]);
                token[i] = (unsigned)(base + 32 * i + lane);
            }
        }
    };
    for (int64_t base = begin; base < end; base += 32 * kRounds) {
        load(base);
#pragma unroll
        for (int i = 0; i < kRounds; ++i)
            if (base + 32 * i + lane < end) atomicAdd(&place[warp][key[i] >> p.shift & p.mask], 1);
    }
    // a thread has two neighbouring digits: tokens of smaller digits, and of its digits in blocks before this one
    int total[2] = {0, 0}, earlier[2] = {0, 0};
#pragma unroll 16
    for (int b = 0; b < (int)gridDim.x; ++b) {
        const int2 n = *reinterpret_cast<const int2 *>(p.counts + b * kDigits + 2 * threadIdx.x);
        if (b < (int)blockIdx.x) {
            earlier[0] += n.x;
            earlier[1] += n.y;
        }
        total[0] += n.x;
        total[1] += n.y;
    }
    int at = total[0] + total[1];
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int x = __shfl_up_sync(0xffffffffu, at, o);
        if (lane >= o) at += x;
    }
    if (lane == 31) warp_total[warp] = at;
    __syncthreads();
    at -= total[0] + total[1];
    for (int w = 0; w < warp; ++w) at += warp_total[w];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        int next = at + earlier[q];
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
            int &slot = place[w][2 * threadIdx.x + q];
            const int n = slot;
            slot = next;
            next += n;
        }
        at += total[q];
    }
    __syncthreads();
    for (int64_t base = begin; base < end; base += 32 * kRounds) {
        if (begin + 32 * kRounds < end) load(base);  // else they are still here
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            const bool in = base + 32 * i + lane < end;
            const int digit = in ? (int)(key[i] >> p.shift & p.mask) : kDigits;
            const unsigned same = __match_any_sync(0xffffffffu, digit);
            const int rank = __popc(same & ((1u << lane) - 1));
            int to = 0;
            if (in) to = place[warp][digit] + rank;
            __syncwarp();
            if (in && rank == 0) place[warp][digit] += __popc(same);
            __syncwarp();
            if (in) {
                p.keys_out[to] = key[i];
                p.order_out[to] = token[i];
                if (p.next_counts) atomicAdd(p.next_counts + to / p.per * kDigits + (key[i] >> p.next_shift & p.mask), 1);
            }
        }
    }
}

// ---- sums of equal tokens --------------------------------------------------------------------------

enum GradMode { kWrite, kAdd, kFold };

// What a finished sum of a warp's columns of one tile meets in memory.
template <typename O, int MODE, bool EVEN, int N>
struct Target {
    using First = Slot<O, EVEN>;       // of kAdd: the table; of kFold: m, then v behind it
    static constexpr int kBytes = 32 * (MODE == kAdd ? First::kBytes : MODE == kFold ? 2 * First::kBytes : 0);
    const EmbeddingGradArgs &a;
    int64_t at;  // of the row's tile

    __device__ __forceinline__ Target(const EmbeddingGradArgs &args, unsigned key, int tile) : a(args), at((int64_t)key * args.ld_grad + tile) {}
    __device__ __forceinline__ void send_for(unsigned char *slot, const Columns<EVEN, N, 32> &c, int lane) const {
        if constexpr (MODE == kAdd) First::send_for(slot, static_cast<const O *>(a.grad) + at, c, 0, lane, 32);
        if constexpr (MODE == kFold) {
            First::send_for(slot, a.m + at, c, 0, lane, 32);
            First::send_for(slot + 32 * First::kBytes, a.v + at, c, 0, lane, 32);
        }
    }
    __device__ __forceinline__ void finish(const unsigned char *slot, const Columns<EVEN, N, 32> &c, int lane, const Vec &sum) const {
        Vec g;
#pragma unroll
        for (int i = 0; i < kPiece / 2; ++i) g.p[i] = mul2(sum.p[i], pair(a.scale, a.scale));
        if constexpr (MODE == kFold) {
            Vec x = First::get(slot, a.m + at, c, 0, lane, 32), y = First::get(slot + 32 * First::kBytes, a.v + at, c, 0, lane, 32);
#pragma unroll
            for (int i = 0; i < kPiece / 2; ++i) {
                x.p[i] = fma2(pair(a.fold.a, a.fold.a), g.p[i], x.p[i]);  // as fold1
                y.p[i] = fma2(mul2(pair(a.fold.b, a.fold.b), g.p[i]), g.p[i], y.p[i]);
            }
            store_piece(a.m + at, c, 0, true, x);
            store_piece(a.v + at, c, 0, true, y);
        } else {
            if constexpr (MODE == kAdd) {
                const Vec x = First::get(slot, static_cast<const O *>(a.grad) + at, c, 0, lane, 32);
#pragma unroll
                for (int i = 0; i < kPiece / 2; ++i) g.p[i] = add2(g.p[i], x.p[i]);
            }
            store_piece(static_cast<O *>(a.grad) + at, c, 0, true, g);
        }
    }
};
__device__ __forceinline__ void add_to(Vec &sum, const Vec &x) {
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i) sum.p[i] = add2(sum.p[i], x.p[i]);
}

// Part `slot` of chunk b: 0 continues the chunk before, 1 begins in b and goes on behind it.  A tile of it lies by lanes, whatever
// columns they have, so that none asks which there are.
__device__ __forceinline__ uint4 *part_of(const EmbeddingGradArgs &a, int64_t b, int slot, int tile) {
    return reinterpret_cast<uint4 *>(a.parts + (2 * b + slot) * a.pad + tile);
}
__device__ __forceinline__ void store_part(uint4 *part, int lane, const Vec &sum) {
    uint4 w[2];
    pack_words(sum, w);
    part[lane] = w[0];
    part[32 + lane] = w[1];
}
__device__ __forceinline__ Vec load_part(const uint4 *part, int lane) {
    const uint4 w[2] = {part[lane], part[32 + lane]};
    return widened(w);
}

constexpr int kGradWarps = 4;

constexpr int kZeroRows = 8;  // rows of a warp, of those that may have no token

// chunk: tokens of a warp, up to 16: a lane each for them and for the next chunk's.  The first zero_blocks blocks zero the rows that have no token.
// A warp's tokens are on their way to shared memory some at a time, with what their sums will meet; the loop over them is
// not unrolled (a batch of four in registers cost little calls 10 us of fetching instructions).
template <int MODE>
constexpr int kDepthOf = MODE == kWrite ? 6 : 4;

template <typename G, typename O, int MODE, bool EVEN>
__global__ void __launch_bounds__(32 * kGradWarps, 8)
embedding_grad_kernel(const EmbeddingGradArgs a, int chunk, int tiles, unsigned zero_blocks) {
    using Given = Slot<G, EVEN>;
    constexpr int N = together(sizeof(G), sizeof(O));
    using Meets = Target<O, MODE, EVEN, N>;
    constexpr int kGiven = 32 * Given::kBytes, kSlot = kGiven + Meets::kBytes, kDepth = kDepthOf<MODE>;
    extern __shared__ __align__(16) unsigned char slots[];  // [warps][kDepth][kSlot]
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    wait_for_previous();
    let_next_start();  // the sorted tokens are there for the next kernel, too
    if (MODE == kWrite && blockIdx.x < zero_blocks) {
        const int64_t first = ((int64_t)blockIdx.x * kGradWarps + warp) * kZeroRows;
        const int64_t row = first + lane;
        int64_t lo = 0, hi = lane < kZeroRows ? a.tokens : 0;  // the first token whose key is not below the row
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if ((int64_t)a.keys[mid] < row) lo = mid + 1;
            else hi = mid;
        }
        const bool empty = lane < kZeroRows && row < a.vocab && (lo == a.tokens || (int64_t)a.keys[lo] != row);
        unsigned todo = __ballot_sync(0xffffffffu, empty);
        for (; todo; todo &= todo - 1)
            fill_zeros(static_cast<O *>(a.grad) + (first + __ffs(todo) - 1) * a.ld_grad, a.dim, lane, 32);
        return;
    }
    const int64_t task = (int64_t)(blockIdx.x - zero_blocks) * kGradWarps + warp, b = task / tiles;
    const int64_t start = b * chunk;
    if (start >= a.tokens) return;
    const int tile = (int)(task - b * tiles) * kTile;
    const Columns<EVEN, N, 32> c = {lane, 32, a.dim - tile};
    const int n = (int)(a.tokens - start < chunk ? a.tokens - start : chunk);
    const unsigned none = 0xffffffffu, out = (unsigned)a.vocab;
    const bool there = lane < 2 * chunk && start + lane < a.tokens;  // its tokens, then the next chunk's
    const unsigned key = there ? a.keys[start + lane] : none, token = there ? a.order[start + lane] : 0;
    const unsigned ahead = start > 0 ? a.keys[start - 1] : none;
    const unsigned far_ahead = start > chunk ? a.keys[start - chunk - 1] : none;
    const unsigned first_key = __shfl_sync(0xffffffffu, key, 0), last_key = __shfl_sync(0xffffffffu, key, n - 1);
    unsigned next = __shfl_down_sync(0xffffffffu, key, 1);
    if (lane == 31) next = none;
    unsigned ends = __ballot_sync(0xffffffffu, lane < n && next != key);
    const int live = __popc(__ballot_sync(0xffffffffu, lane < n && key != out));  // the others come last
    bool open = first_key == ahead;  // the first run continues the chunk before
    int j = 0;
    if (open && ends && far_ahead != first_key && __ffs(ends) < chunk) {  // begun there and ended here, not filling the chunk: its warp sees to it
        j = __ffs(ends);
        open = false;
    }
    // the last run's tokens in the next chunk, where it begins here and does not fill that
    const bool goes_on = live == n && !(ends >> (n - 1) & 1) && !(open && ends == 0);
    int extra = goes_on ? __popc(__ballot_sync(0xffffffffu, lane >= n && key == last_key)) : 0;
    if (extra == chunk) extra = 0;
    const int count = live + extra;
    if (extra) ends |= 1u << (count - 1);
    const G *dy = static_cast<const G *>(a.dy) + tile;
    Vec sum = zeros();
    unsigned char *const mine = slots + warp * (kDepth * kSlot);
    const auto send_for = [&](int at, int slot) {
        const unsigned t = __shfl_sync(0xffffffffu, token, at & 31), k = __shfl_sync(0xffffffffu, key, at & 31);
        if (at < count) {
            Given::send_for(mine + slot * kSlot, dy + (int64_t)t * a.ld_dy, c, 0, lane, 32);
            if (MODE != kWrite && (ends >> at & 1)) Meets(a, k, tile).send_for(mine + slot * kSlot + kGiven, c, lane);
        }
        copies_end_group();
    };
    for (int i = 0; i < kDepth; ++i) send_for(j + i, i);
    int slot = 0;
#pragma unroll 1
    for (; j < count; ++j) {
        const unsigned t = __shfl_sync(0xffffffffu, token, j), k = __shfl_sync(0xffffffffu, key, j);
        copies_wait<kDepth - 1>();
        add_to(sum, Given::get(mine + slot * kSlot, dy + (int64_t)t * a.ld_dy, c, 0, lane, 32));
        if (ends >> j & 1) {
            if (open) store_part(part_of(a, b, 0, tile), lane, sum);
            else Meets(a, k, tile).finish(mine + slot * kSlot + kGiven, c, lane, sum);
            open = false;
            sum = zeros();
        }
        __syncwarp();
        send_for(j + kDepth, slot);  // behind the last use of what was there
        slot = slot + 1 == kDepth ? 0 : slot + 1;
    }
    if (live == n && extra == 0 && !(ends >> (n - 1) & 1)) store_part(part_of(a, b, open ? 0 : 1, tile), lane, sum);
}

// Runs that fill chunks: a block looks at 32 chunks for those that begin one, and joins the parts of these for one tile;
// a warp to each, or the block to one of many parts.
constexpr int kJoinWarps = 8;
// parts up to which a warp adds them alone (32768 x 4096: 113 us, up to 4 113, up to 40 125; 4096 x 1600: 24, 25, 25)
constexpr int kJoinAlone = 12;
constexpr int kJoinLoads = 4;   // parts of a lane, together

template <typename O, int MODE, bool EVEN, int N>
__global__ void __launch_bounds__(32 * kJoinWarps)
embedding_join_kernel(const EmbeddingGradArgs a, int chunk) {
    using Meets = Target<O, MODE, EVEN, N>;
    __shared__ Pair sums[kJoinWarps][kTile / 2];
    __shared__ alignas(16) unsigned char slots[kJoinWarps][Meets::kBytes ? Meets::kBytes : 16];
    __shared__ int64_t last_of[32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int tile = blockIdx.y * kTile;
    const Columns<EVEN, N, 32> c = {lane, 32, a.dim - tile};
    const unsigned none = 0xffffffffu;
    const int64_t first = (int64_t)blockIdx.x * 32, start = (first + lane) * chunk, end = start + chunk;
    // The sort has ended when this kernel may start (the sums wait for it first): the runs are looked up while the sums are
    // still being made, and what the first one of a warp will meet is sent for.  A run begins in a chunk and fills the
    // next one: the same key at its own end and at that chunk's, another one in front of it.  (The keys come from L2: it is the
    // sums that have waited for the sort, not this kernel.)
    const unsigned key = end <= a.tokens ? __ldcg(a.keys + end - 1) : none, far = end + chunk <= a.tokens ? __ldcg(a.keys + end + chunk - 1) : none - 1;
    const unsigned before = start > 0 && start <= a.tokens ? __ldcg(a.keys + start - 1) : none;
    unsigned todo = __ballot_sync(none, key == far && key != before && key != (unsigned)a.vocab), of_warp = 0, of_block = 0;
    for (int turn = 0; todo; todo &= todo - 1) {  // (all warps see the same)
        const int which = __ffs(todo) - 1;
        const unsigned k = __shfl_sync(none, key, which);
        // the chunk in which the run ends, among the next 32 or, of a long run, by ever closer looks at 32 places
        int64_t last = first + which, end_chunk = (a.tokens + chunk - 1) / chunk, apart = 1;
        do {
            const int64_t at = (last + (lane + 1) * apart) * chunk;
            const unsigned more = __ballot_sync(none, at < a.tokens && __ldcg(a.keys + min(at, a.tokens - 1)) == k);
            const int run = more == none ? 32 : __ffs(~more) - 1;
            last += run * apart;
            if (apart == 1 && run < 32) break;
            if (run < 32 && last + apart < end_chunk) end_chunk = last + apart;  // it ends before that one
            apart = (end_chunk - last + 31) / 32;
        } while (end_chunk - last > 1);
        if (lane == 0) last_of[which] = last;  // (every warp writes the same)
        if (last - first - which > kJoinAlone) of_block |= 1u << which;
        else if (turn++ % kJoinWarps == warp) of_warp |= 1u << which;
    }
    __syncwarp();
    const int ahead = of_warp ? __ffs(of_warp) - 1 : -1;
    if (ahead >= 0) Meets(a, __shfl_sync(none, key, ahead), tile).send_for(slots[warp], c, lane);
    copies_end_group();
    wait_for_previous();
    // (a turn's last parts are loaded again where there are no more: a load with a condition waits for the one before it)
    const auto sum_parts = [&](Vec &sum, int64_t from, int64_t to) {
        for (; from < to; from += kJoinLoads) {
            Vec q[kJoinLoads];
#pragma unroll
            for (int j = 0; j < kJoinLoads; ++j) q[j] = load_part(part_of(a, min(from + j, to - 1), 0, tile), lane);
#pragma unroll
            for (int j = 0; j < kJoinLoads; ++j)
#pragma unroll
                for (int i = 0; i < kPiece / 2; ++i) sum.p[i] = add2(sum.p[i], from + j < to ? q[j].p[i] : 0);
        }
    };
    for (; of_warp; of_warp &= of_warp - 1) {
        const int which = __ffs(of_warp) - 1;
        const Meets meets(a, __shfl_sync(none, key, which), tile);
        if (which != ahead) {
            meets.send_for(slots[warp], c, lane);
            copies_end_group();
        }
        Vec sum = load_part(part_of(a, first + which, 1, tile), lane);
        sum_parts(sum, first + which + 1, last_of[which] + 1);
        copies_wait<0>();
        meets.finish(slots[warp], c, lane, sum);
    }
    copies_wait<0>();
    for (; of_block; of_block &= of_block - 1) {
        const int which = __ffs(of_block) - 1;
        const int64_t b = first + which, parts = last_of[which] - b;
        Vec sum = warp == 0 ? load_part(part_of(a, b, 1, tile), lane) : zeros();
        sum_parts(sum, b + 1 + parts * warp / kJoinWarps, b + 1 + parts * (warp + 1) / kJoinWarps);
#pragma unroll
        for (int q = 0; q < kPiece / 2; ++q) sums[warp][q * 32 + lane] = sum.p[q];
        __syncthreads();
        if (warp == 0) {
            const Meets meets(a, __shfl_sync(none, key, which), tile);
            meets.send_for(slots[0], c, lane);
            copies_end_group();
            for (int w = 1; w < kJoinWarps; ++w)
#pragma unroll
                for (int q = 0; q < kPiece / 2; ++q) sum.p[q] = add2(sum.p[q], sums[w][q * 32 + lane]);
            copies_wait<0>();
            meets.finish(slots[0], c, lane, sum);
        }
        __syncthreads();
    }
}

// ---- launches --------------------------------------------------------------------------------------

template <typename T, typename O>
cudaError_t lookup(const EmbeddingArgs &a, cudaStream_t stream) {
    const int groups = (a.dim + kLookupPieces * kTile - 1) / (kLookupPieces * kTile);
    const unsigned blocks = (unsigned)((a.tokens * groups + kLookupWarps - 1) / kLookupWarps);
    constexpr int N = together(sizeof(T), sizeof(O));
    if (even_rows(a.table, a.dim, a.ld_table, sizeof(T), N) && even_rows(a.out, a.dim, a.ld_out, sizeof(O), N))
        embedding_kernel<T, O, true><<<blocks, 32 * kLookupWarps, 0, stream>>>(a, groups);
    else
        embedding_kernel<T, O, false><<<blocks, 32 * kLookupWarps, 0, stream>>>(a, groups);
    return cudaGetLastError();
}

// Sizes of the parts of the workspace, each a multiple of 16 bytes.
size_t up16(size_t n) { return (n + 15) / 16 * 16; }

// Tokens to a chunk: 16 where that makes warps enough.  (With 8 and with 16: 32768 x 4096 127 and 113 us, 65536 x 256 52 and 48,
// 4096 x 1600 24.0 and 24.8, 8000 x 256 25 and 29.)
int chunk_for(int64_t tokens, int tiles, int sm_count) { return tokens * tiles / 16 < (int64_t)14 * sm_count ? 8 : 16; }
struct GradPlan {
    int tiles, chunk;
    int64_t chunks, pad;
    size_t list, parts;  // bytes of a list of the tokens, of the runs' parts
    bool by_rank;
};
GradPlan plan_grad(int64_t tokens, int dim, int sm_count) {
    GradPlan p;
    p.tiles = (dim + kTile - 1) / kTile;
    p.chunk = chunk_for(tokens, p.tiles, sm_count);
    p.chunks = (tokens + p.chunk - 1) / p.chunk;
    p.pad = (int64_t)p.tiles * kTile;
    p.list = up16((size_t)tokens * sizeof(unsigned));
    p.parts = p.chunks > 1 ? (size_t)p.chunks * 2 * p.pad * sizeof(float) : 0;
    p.by_rank = tokens <= kRankTokens;
    return p;
}

cudaError_t sort_tokens(EmbeddingGradArgs &a, const GradPlan &p, unsigned char *ws, cudaStream_t stream, int *launches) {
    unsigned *lists[4];
    for (int i = 0; i < 4; ++i) lists[i] = reinterpret_cast<unsigned *>(ws + i * p.list);
    a.keys = lists[0];
    a.order = lists[1];
    if (p.by_rank) {
        embedding_rank_kernel<<<(unsigned)((a.tokens + 31) / 32), 32 * kRankWarps, 0, stream>>>(a);
        *launches += 1;
        return cudaGetLastError();
    }
    int bits = 1;
    while (bits < 32 && a.vocab >> bits) ++bits;  // the key `vocab` included
    const int passes = (bits + kDigitBits - 1) / kDigitBits, each = (bits + passes - 1) / passes;
    int *counts = reinterpret_cast<int *>(ws + 4 * p.list);
    SortPass s = {};
    s.mask = (1 << each) - 1;
    int64_t per = (a.tokens + kSortBlocks - 1) / kSortBlocks;
    if (per < 1024) per = 1024;
    s.per = (int)((per + kSortThreads - 1) / kSortThreads * kSortThreads);
    const unsigned blocks = (unsigned)((a.tokens + s.per - 1) / s.per);
    constexpr int kInts = kSortBlocks * kDigits;  // counts of a pass
    s.counts = counts;
    embedding_digits_kernel<<<blocks, kSortThreads, 0, stream>>>(a, s, counts + kInts, (passes - 1) * kInts);
    cudaError_t e = cudaGetLastError();
    *launches += 1;
    int to = passes % 2 ? 0 : 2;  // the last pass writes lists 0 and 1
    for (int i = 0; i < passes && e == cudaSuccess; ++i, to ^= 2) {
        s.counts = counts + i * kInts;
        s.next_counts = i + 1 < passes ? counts + (i + 1) * kInts : nullptr;
        s.shift = i * each;
        s.next_shift = (i + 1) * each;
        s.keys_out = lists[to];
        s.order_out = lists[to + 1];
        e = launch_chained(embedding_scatter_kernel, dim3(blocks), dim3(kSortThreads), 0, stream, a, s);
        *launches += 1;
        s.keys = lists[to];
        s.order = lists[to + 1];
    }
    return e;
}

template <typename G, typename O, int MODE, bool EVEN>
cudaError_t sums(const EmbeddingGradArgs &a, const GradPlan &p, cudaStream_t stream, int *launches) {
    const int64_t sum_blocks = (p.chunks * p.tiles + kGradWarps - 1) / kGradWarps;
    const int64_t zero_blocks = MODE == kWrite ? (a.vocab + kZeroRows * kGradWarps - 1) / (kZeroRows * kGradWarps) : 0;
    if (sum_blocks + zero_blocks == 0) return cudaSuccess;
    const dim3 grid((unsigned)(sum_blocks + zero_blocks)), block(32 * kGradWarps);
    const size_t shared = (size_t)kGradWarps * kDepthOf<MODE> * (32 * Slot<G, EVEN>::kBytes + Target<O, MODE, EVEN, 8>::kBytes);
    cudaError_t e = cudaSuccess;
    if (shared > 40 * 1024) {  // more than a kernel has unasked
        static std::atomic<unsigned long long> ready{0};
        e = allow_shared(embedding_grad_kernel<G, O, MODE, EVEN>, (int)shared, ready);
        if (e != cudaSuccess) return e;
    }
    if (a.tokens > 0) {
        e = launch_chained(embedding_grad_kernel<G, O, MODE, EVEN>, grid, block, shared, stream, a, p.chunk, p.tiles, (unsigned)zero_blocks);
    } else {  // no sort in front
        embedding_grad_kernel<G, O, MODE, EVEN><<<grid, block, shared, stream>>>(a, p.chunk, p.tiles, (unsigned)zero_blocks);
        e = cudaGetLastError();
    }
    if (e != cudaSuccess) return e;
    *launches += 1;
    if (p.chunks > 1) {
        const dim3 joins((unsigned)((p.chunks + 31) / 32), (unsigned)p.tiles);
        e = launch_chained(embedding_join_kernel<O, MODE, EVEN, together(sizeof(G), sizeof(O))>, joins, dim3(32 * kJoinWarps), 0, stream, a, p.chunk);
        *launches += 1;
    }
    return e;
}
template <typename G, typename O, int MODE>
cudaError_t sums(const EmbeddingGradArgs &a, const GradPlan &p, cudaStream_t stream, int *launches) {
    constexpr int N = together(sizeof(G), sizeof(O));
    const bool even = even_rows(a.dy, a.dim, a.ld_dy, sizeof(G), N) &&
                      (MODE == kFold ? even_rows(a.m, a.dim, a.ld_grad, 4, N) && aligned(a.v, 16) : even_rows(a.grad, a.dim, a.ld_grad, sizeof(O), N));
    return even ? sums<G, O, MODE, true>(a, p, stream, launches) : sums<G, O, MODE, false>(a, p, stream, launches);
}
template <typename G>
cudaError_t sums(const EmbeddingGradArgs &a, const GradPlan &p, cudaStream_t stream, int *launches) {
    if (a.m) return sums<G, float, kFold>(a, p, stream, launches);
    if (a.grad_dtype == ADAMA_F32)
        return a.accumulate ? sums<G, float, kAdd>(a, p, stream, launches) : sums<G, float, kWrite>(a, p, stream, launches);
    return a.accumulate ? sums<G, __nv_bfloat16, kAdd>(a, p, stream, launches) : sums<G, __nv_bfloat16, kWrite>(a, p, stream, launches);
}

}  // namespace

cudaError_t launch_embedding(const EmbeddingArgs &a, cudaStream_t stream) {
    if (a.table_dtype == ADAMA_F32)
        return a.out_dtype == ADAMA_F32 ? lookup<float, float>(a, stream) : lookup<float, __nv_bfloat16>(a, stream);
    return a.out_dtype == ADAMA_F32 ? lookup<__nv_bfloat16, float>(a, stream) : lookup<__nv_bfloat16, __nv_bfloat16>(a, stream);
}

size_t embedding_workspace_bytes(int64_t tokens, int dim, int sm_count) {
    const GradPlan p = plan_grad(tokens, dim, sm_count);
    return p.list * (p.by_rank ? 2 : 4) + (p.by_rank ? 0 : kSortPasses * kSortBlocks * kDigits * sizeof(int)) + p.parts;
}

cudaError_t launch_embedding_grad(EmbeddingGradArgs a, int sm_count, cudaStream_t stream, int *launches) {
    const GradPlan p = plan_grad(a.tokens, a.dim, sm_count);
    unsigned char *ws = static_cast<unsigned char *>(a.workspace);
    a.pad = p.pad;
    a.parts = reinterpret_cast<float *>(ws + p.list * (p.by_rank ? 2 : 4) + (p.by_rank ? 0 : kSortPasses * kSortBlocks * kDigits * sizeof(int)));
    if (a.tokens > 0) {
        const cudaError_t e = sort_tokens(a, p, ws, stream, launches);
        if (e != cudaSuccess) return e;
    }
    return a.dy_dtype == ADAMA_F32 ? sums<float>(a, p, stream, launches) : sums<__nv_bfloat16>(a, p, stream, launches);
}

}  // namespace adama
