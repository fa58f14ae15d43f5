// psops_xent_kernels.cuh -- softmax cross entropy of a linear head and its
// gradients (C entries: psops_xent.cu).
//
// A call first lists the tokens that count (psops_xent_index_kernel) and
// gathers their hidden states, padded with zeros to whole tiles
// (psops_xent_gather_kernel); everything after works on these "compact" rows,
// so that tokens without a loss cost nothing and their contents cannot reach a
// result.  The number of compact rows is known on the device only.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "psops_umma.cuh"

namespace {

constexpr int kTileRows = 256;                   // compact rows are padded to this
constexpr int kTileCols = 256;                   // a piece of the vocabulary is a multiple of this
constexpr int kStepK = 64;                       // of the summed axis, a step of a product
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct XentControl {
    int rows;                                    // tokens that count
    unsigned tickets;
    float unscale;                               // gradient sums * unscale = gradients
    int error;
    int shares;                                  // dh: its sum over the vocabulary in so many shares
    int share_rows;                              // rows between the shares' sums
    int dw_shares;                               // dw, where it is split: its sum over the tokens in so many shares
};

struct IndexParams {
    const long long *targets;
    const float *grad;                           // NULL in the forward pass
    XentControl *control;
    int *row_of;                                 // compact row -> token
    int *compact_of;                             // token -> compact row, or -1
    int *label;                                  // compact row -> label
    float *row_scale;                            // compact row -> what its 16-bit gradients are multiplied with (backward)
    float *rows_out, *lse_out;                   // zeroed where a token is left out (forward)
    const float *lse, *rows;                     // (backward) by token; rows may be NULL
    float *row_label;                            // (backward) compact row -> exp(-rows) - 1, or 2 where rows are not given
    float *row_lse;                              // (backward) by compact row, times log2 e
    int tokens;
    int vocab;
    int reduction;
    float headroom;                              // largest |dlogits| that the 16-bit type should see
    int tiles_across, steps, sum_rows, pairs;    // dh: tiles of its columns, steps of the shortest piece, room for sums, CTAs or pairs of them
    int dw_tiles, dw_most, dw_pairs;             // dw, where it is split: tiles, most shares (0: not split), pairs of CTAs
};

constexpr int kMostShares = 32;
constexpr int kShareCost = 4;                    // a tile's start and end, in steps
constexpr int kShareJoin = 6;                    // a tile's sums written and read once more, that many tiles to a step

// dh has few tiles where there are few rows, and its sum over the vocabulary is
// long: it is split into shares, as many as bring the rounds of tiles to the
// least time (8 x 4 tiles on 74 pairs: one share leaves 42 pairs idle, two
// shares ten; measured 183 -> 100 us for 1,950 rows, 32,003 entries, dim 1000).
// By a whole warp, each lane looking at one number of shares; ties go to the fewest.
__device__ __forceinline__ int best_shares(int tiles, int steps, int most, int pairs)
{
    static_assert(kMostShares <= 32, "a lane for each");
    const int s = (threadIdx.x & 31) + 1;
    const long long rounds = ((long long)tiles * s + pairs - 1) / pairs;
    const long long t = rounds * ((steps + s - 1) / s + kShareCost) + (long long)tiles * s / kShareJoin;
    const unsigned mine = s > most || t >= 0xffffffffll ? 0xffffffffu : (unsigned)t;
    const unsigned least = __reduce_min_sync(0xffffffffu, mine);
    return least == 0xffffffffu ? 1 : __ffs((int)__ballot_sync(0xffffffffu, mine == least));
}

constexpr int kIndexThreads = 1024;

using umma::after_the_kernel_before;

// Elements [8 g, 8 g + 8) of a row of `n` 16-bit values, zeros beyond its end.
__device__ __forceinline__ uint4 eight_of_row(const uint16_t *row, int g, int n, bool aligned)
{
    if (aligned && g * 8 + 8 <= n) return *reinterpret_cast<const uint4 *>(row + g * 8);
    uint32_t e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = g * 8 + j < n ? row[g * 8 + j] : 0u;
    return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
}

// Where the hidden states come from and go to.
struct GatherParams {
    const uint16_t *h;
    long long ld;
    int dim, padded;
    bool aligned;
    uint16_t *out;
};

// Hidden states of the tokens that count, in rows of `padded` (a multiple of 64)
// elements; zero rows up to a whole step of the products.  A thread per 16 bytes.
__device__ __forceinline__ void gather_rows(const GatherParams &G, int rows, const int *row_of)
{
    const unsigned groups = G.padded / 8;
    const long long whole = (long long)(max(1, rows) + kStepK - 1) / kStepK * kStepK * groups;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < whole; i += (long long)gridDim.x * blockDim.x) {
        const int r = (int)(i / groups), g = (int)(i - (long long)r * groups);
        uint4 u = make_uint4(0, 0, 0, 0);
        if (r < rows) u = eight_of_row(G.h + row_of[r] * G.ld, g, G.dim, G.aligned);
        reinterpret_cast<uint4 *>(G.out)[i] = u;
    }
}

// One block lists the tokens that count, in order: each warp a stretch of them.
// GATHER: with no more than kListTokens tokens every block makes the list for
// itself, the first one also writes it down, and all of them gather: one launch
// instead of two.  In a CUDA graph, one / two, us, loss and gradients of x 512 x
// 3,000: 1,024 tokens 18.8 / 20.1 and 38.1 / 40.1, 8,192 tokens 43.4 / 44 and
// 102.8 / 102.6.
constexpr int kListTokens = 8192;
template <bool GATHER>
__global__ void __launch_bounds__(kIndexThreads) psops_xent_index_kernel(const IndexParams P, const GatherParams G)
{
    __shared__ int own_row_of[GATHER ? kListTokens : 1];
    __shared__ int warp_sum[32];
    __shared__ float warp_top[32];
    after_the_kernel_before();
    const bool writes = !GATHER || blockIdx.x == 0;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per = (P.tokens + kIndexThreads - 1) / kIndexThreads * 32;
    const int first = min(P.tokens, warp * per), last = min(P.tokens, first + per);
    int mine = 0;
    float top = 0.0f;
#pragma unroll 4
    for (int t = first + lane; t < last; t += 32) {
        const long long y = P.targets[t];
        if (y >= 0 && y < P.vocab) {
            ++mine;
            if (P.grad != nullptr && P.reduction == PSOPS_PER_TOKEN) {
                const float g = fabsf(P.grad[t]);
                if (g < INFINITY) top = fmaxf(top, g);       // one that overflowed must not scale the others out of range
            }
        }
    }
    mine = __reduce_add_sync(0xffffffffu, mine);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    if (lane == 0) {
        warp_sum[warp] = mine;
        warp_top[warp] = top;
    }
    __syncthreads();
    int at = 0, total = 0;
    top = 0.0f;
#pragma unroll
    for (int w = 0; w < 32; ++w) {
        if (w < warp) at += warp_sum[w];
        total += warp_sum[w];
        top = fmaxf(top, warp_top[w]);
    }
    // What the 16-bit logits' gradients are multiplied with, and what undoes it in
    // the fp32 sums.  One gradient for all tokens stays out of the 16 bits (its own
    // rounding would be the same for every token and add up); gradients per token
    // are scaled by a power of two that brings the largest finite one to (1/2, 1] * headroom.
    float up = P.headroom;
    if (P.grad != nullptr) {
        float undo;
        if (P.reduction != PSOPS_PER_TOKEN) {
            undo = (P.reduction == PSOPS_MEAN ? __fdiv_rn(P.grad[0], (float)max(1, total)) : P.grad[0]) / P.headroom;
        } else {
            int e = 0;
            if (top > 0.0f) e = min(120, max(-100, ilogbf(top) + 1));
            up = ldexpf(P.headroom, -e);
            undo = 1.0f / up;
        }
        if (total == 0) undo = 0.0f;                 // no token, no gradient, even if the upstream one is not finite
        if (writes && threadIdx.x == 0) P.control->unscale = undo;
    }
#pragma unroll 2
    for (int t0 = first; t0 < last; t0 += 32) {
        const int t = t0 + lane;
        const long long y = t < last ? P.targets[t] : -1;
        const bool in = y >= 0 && y < P.vocab;
        const unsigned votes = __ballot_sync(0xffffffffu, in);
        if (in) {
            const int r = at + __popc(votes & ((1u << lane) - 1u));
            if (GATHER) own_row_of[r] = t;
            if (writes) {
                P.row_of[r] = t;
                P.label[r] = (int)y;
                P.compact_of[t] = r;
                if (P.grad != nullptr) {
                    P.row_scale[r] = P.reduction == PSOPS_PER_TOKEN ? P.grad[t] * up : up;
                    P.row_lse[r] = P.lse[t] * kLog2e;
                    P.row_label[r] = P.rows != nullptr ? expm1f(-P.rows[t]) : 2.0f;
                }
            }
        } else if (writes && t < last) {
            P.compact_of[t] = -1;
            if (P.rows_out != nullptr) P.rows_out[t] = 0.0f;
            if (P.lse_out != nullptr) P.lse_out[t] = 0.0f;
        }
        at += __popc(votes);
    }
    const int tiles = max(1, (total + kTileRows - 1) / kTileRows);
    int shares = 1;
    if (P.grad != nullptr && writes && warp == 0)
        shares = best_shares(tiles * P.tiles_across, P.steps, min(min(kMostShares, P.steps), P.sum_rows / (tiles * kTileRows)), P.pairs);
    int dw_shares = 1;
    if (P.dw_most > 1 && writes && warp == 0) {
        const int steps = (max(1, total) + kStepK - 1) / kStepK;
        dw_shares = best_shares(P.dw_tiles, steps, min(P.dw_most, steps), P.dw_pairs);
    }
    if (writes && threadIdx.x == 0) {
        P.control->dw_shares = dw_shares;
        P.control->rows = total;
        P.control->tickets = 0;
        P.control->share_rows = tiles * kTileRows;
        P.control->shares = shares;
    }
    if (GATHER) {
        __syncthreads();
        gather_rows(G, total, own_row_of);
    }
}

constexpr int kCopyThreads = 256;

// The gathering alone, behind the list.
__global__ void __launch_bounds__(kCopyThreads) psops_xent_gather_kernel(const GatherParams G, const XentControl *control, const int *row_of)
{
    after_the_kernel_before();
    gather_rows(G, control->rows, row_of);
}

// Rows of w that cannot be read in place.
__global__ void __launch_bounds__(kCopyThreads) psops_xent_pack_kernel(const uint16_t *w, long long ld, long long rows, int dim,
                                                                       int padded, bool aligned, uint16_t *out)
{
    after_the_kernel_before();
    const unsigned groups = padded / 8;
    for (long long i = (long long)blockIdx.x * kCopyThreads + threadIdx.x; i < rows * groups; i += (long long)gridDim.x * kCopyThreads) {
        const long long r = i / groups;
        reinterpret_cast<uint4 *>(out)[i] = eight_of_row(w + r * ld, (int)(i - r * groups), dim, aligned);
    }
}

// Rows of dw that could not be written in place.
__global__ void __launch_bounds__(kCopyThreads) psops_xent_unpack_kernel(const uint16_t *in, int padded, long long rows, int dim,
                                                                         uint16_t *dw, long long ld)
{
    after_the_kernel_before();
    const long long warps = (long long)gridDim.x * (kCopyThreads / 32);
    for (long long r = (long long)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); r < rows; r += warps)
#pragma unroll 4
        for (int d = threadIdx.x & 31; d < dim; d += 32) dw[r * ld + d] = in[r * padded + d];
}

// ---------------------------------------------------------------------------
// Products on the tensor cores
//
// One kernel does all of them, persistent, a pair of CTAs to a 256 x 256 tile
// of the result, 64 of the summed axis a step:
//
//   job       rows of the result   columns        summed over    what becomes of a tile
//   kLoss     compact rows         vocabulary     dim            softmax maxima and sums
//   kDlogits  compact rows         vocabulary     dim            the logits' gradient, 16 bits
//   kDh       compact rows         dim            vocabulary     fp32 sums, added up over pieces
//   kDw       vocabulary           dim            compact rows   dw, 16 bits
//   kDwLong   the same, from a call of more tokens than one chain of sums may have
//   kDwSums   the same, the summed axis in shares                fp32 sums
//
// Warp 0 of each CTA copies its share of both operands (of a pair: 128 rows of
// A and 128 of B, 32 KB a step), one thread of the first CTA issues the
// products, warps 4 to 11 of each CTA turn the other one of two 256-column
// accumulators into the job's output meanwhile.  kDh and kDw read operands whose
// summed axis runs across the rows in memory: the copies bring 64 x 64 boxes,
// and the product's descriptors say so; nothing is transposed.
//
// With 128 tokens or fewer half of a pair's rows would be empty; the first
// three jobs then run with single CTAs on 128 x 256 tiles.  In a CUDA graph, single
// CTAs / pairs, us, loss and gradients: 64 x 4,096 x 32,768 61 / 74 and 188 / 206,
// 128 x 1,024 x 32,000 25 / 29 and 75 / 75, 128 x 512 x 300 18 / 18 and 30 / 30;
// few tiles of a long sum would rather have two SMs each: 32 x 1,000 x 3,000
// 22 / 20 and 36 / 33.
// ---------------------------------------------------------------------------
enum Job { kLoss = 0, kDlogits = 1, kDh = 2, kDw = 3, kDwLong = 4, kDwSums = 5 };

constexpr int kTile = 256, kHalf = 128;
constexpr int kOperandBytes = kHalf * kStepK * 2;                // 128 rows of A or B
constexpr int kOutBytes = 32 * 128;                              // a warp's 32 rows of 128 bytes on their way out
constexpr int kOutWarps = 8;
constexpr int kProductThreads = 384;
constexpr int kSingleTokens = kHalf;                             // up to here single CTAs
// A pair: 32 KB a stage for each CTA, five of them, and two outputs a warp; a
// single CTA: 48 KB a stage, four of them, one output.
template <bool PAIR> struct ProductShape {
    static constexpr int kCtas = PAIR ? 2 : 1, kRows = kHalf * kCtas;
    static constexpr int kStages = PAIR ? 5 : 4, kOuts = PAIR ? 2 : 1;
    static constexpr int kStageBytes = kOperandBytes * (PAIR ? 2 : 3);
    static constexpr int kShared = kStages * kStageBytes + kOutWarps * kOuts * kOutBytes + 1024;       // 1024: alignment
};
// The tensor cores cut off what does not fit into a running sum, so a chain of n
// products of 16 elements each ends nearer to zero than it should, by c n 2^-24 of
// its value: at most a unit in the last place per product, c <= 2.  Measured for
// logits of 16 that lean to their label: c = 0.26 to 0.38 (bf16) and 0.35 to 0.97
// (fp16, whose products have more bits to lose); where all products have one sign
// up to 0.49 and 1.5, and up to 1.6 in dw's sums over 300,000 tokens, of either type.
// So sums are made of chains of at most so many steps, which are added up in fp32,
// to nearest (logits and dw in registers, the fp32 sums where they lie; dw has a
// variant for it, since the registers cost it 452 bytes of spills):
//   a logit: 12 steps, n <= 48, since the loss is fp32;
//   dh, dw: 128 steps, n <= 512: at most 6e-5 of the value, an eighth of fp16's unit
//   roundoff.  One chain of 131,072 terms left dh 1.2e-4 too small, one of 300,000 dw
//   1.8e-3.
constexpr int kLogitSteps = 12, kSumSteps = 128;
constexpr int kChainTokens = kSumSteps * kStepK;                 // a call of more takes kDwLong
// For the logits the middle of the loss is also put back, with the factor that they
// are multiplied with anyway: what is left of the loss's error is mostly below 5e-7.
// Where nothing was cut off (a logit of one product), the factor itself is the
// error: 0.3 and 0.6 of 48 2^-24, 9e-7 and 1.7e-6 of the logit.
template <class T> constexpr float kCutOff = 0.3f * 0x1p-24f;
template <> constexpr float kCutOff<__half> = 0.6f * 0x1p-24f;
constexpr int kGroupTiles = 8;                                   // row tiles that share columns in L2

struct ProductParams {
    XentControl *control;
    int columns;                                 // kLoss, kDlogits: entries of the piece; kDh, kDw: padded dim
    int depth;                                   // kLoss, kDlogits: padded dim; kDh: entries of the piece
    int result_rows;                             // kDw, kDwSums: entries of the piece
    int dw_share_rows;                           // kDwSums: rows between the shares' sums
    int first;                                   // first vocabulary entry of the piece
    bool add;                                    // kDh: add to the sums of the pieces before (else false)
    const int *label;
    const float *row_lse, *row_scale, *row_label;
    float2 *stats;                               // (max, sum of exp2) by 128 vocabulary entries and compact row, base 2
    long long stats_ld;
    float *label_logit;
};

// 32 bits, approximate: off by some units in the last place of the result, numbers
// below 2^-126 as zero.  A probability's error from its logit, 16 times 2^-24 and
// more, is larger, and one below 2^-126 adds nothing to a sum that has a 1 in it.
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <class T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    uint32_t u;
    memcpy(&u, &h, 4);
    return u;
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    uint32_t u;
    memcpy(&u, &h, 4);
    return u;
}

// x = value where at == j; written out so that the registers of a row are not put into memory to be indexed
__device__ __forceinline__ void take_if(float &x, int at, int j, uint32_t value)
{
    asm("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, %2;\n\t@p mov.b32 %0, %3;\n\t}" : "+f"(x) : "r"(at), "r"(j), "r"(value));
}

struct Work { int m, n, split; };                // tile of the result, share of the summed axis

// Tiles in bands of kGroupTiles row tiles, column by column, so that the pairs
// running at one time share both operands in L2.
__device__ __forceinline__ Work work_of(int i, int tiles_m, int tiles_n)
{
    const int tiles = tiles_m * tiles_n;
    Work w;
    w.split = i / tiles;
    i -= w.split * tiles;
    const int band = i / (kGroupTiles * tiles_n);
    const int in_band = i - band * kGroupTiles * tiles_n;
    const int high = min(kGroupTiles, tiles_m - band * kGroupTiles);
    w.n = in_band / high;
    w.m = band * kGroupTiles + in_band - w.n * high;
    return w;
}

template <class T, int JOB, bool PAIR>
__global__ void __launch_bounds__(kProductThreads, 1)
psops_xent_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                          const __grid_constant__ CUtensorMap map_out, const ProductParams P)
{
    constexpr bool kAAcross = JOB == kDw || JOB == kDwLong || JOB == kDwSums, kBAcross = JOB == kDh || kAAcross;
    constexpr bool kSums = JOB == kDh || JOB == kDwSums, kLogits = JOB == kLoss || JOB == kDlogits;
    constexpr int kChainSteps = kLogits ? kLogitSteps : kSumSteps;
    using S = ProductShape<PAIR>;
    constexpr int kStages = S::kStages, kStageBytes = S::kStageBytes, kRows = S::kRows;
    constexpr uint32_t kInstruction = umma::instruction(__is_same(T, __nv_bfloat16), kAAcross, kBAcross, kRows, kTile);

    extern __shared__ uint8_t raw[];
    __shared__ alignas(8) uint64_t bar_full[kStages], bar_empty[kStages], bar_sum[2], bar_free[2];
    __shared__ uint32_t tensor_base_slot;
    __shared__ int failed_slot;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? umma::cta_rank() : 0;
    volatile int *failed = &failed_slot;
    const uint32_t stages = (umma::shared_address(raw) + 1023u) & ~1023u;
    const uint32_t outs = stages + kStages * kStageBytes;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            umma::barrier_init(umma::shared_address(&bar_full[s]), 1);
            umma::barrier_init(umma::shared_address(&bar_empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            umma::barrier_init(umma::shared_address(&bar_sum[b]), 1);
            umma::barrier_init(umma::shared_address(&bar_free[b]), S::kCtas * kOutWarps);
        }
        failed_slot = 0;
        umma::barrier_init_done();
        umma::prefetch_map(&map_a);
        umma::prefetch_map(&map_b);
    }
    if (warp == 2) umma::tensor_memory_take<PAIR>(umma::shared_address(&tensor_base_slot));
    umma::fence_before();
    __syncthreads();
    umma::cluster_sync();
    umma::fence_after();
    const uint32_t tensor_base = tensor_base_slot;

    after_the_kernel_before();
    const int rows = P.control->rows;
    const int some_rows = max(1, rows);
    const int tiles_m = ((kAAcross ? P.result_rows : JOB == kDh ? rows : some_rows) + kRows - 1) / kRows;
    const int tiles_n = (P.columns + kTile - 1) / kTile;
    const int steps = ((kAAcross ? some_rows : P.depth) + kStepK - 1) / kStepK;
    const int splits = JOB == kDh ? P.control->shares : JOB == kDwSums ? P.control->dw_shares : 1;
    const int share = (steps + splits - 1) / splits;                                   // steps of the longest share
    const int fewest = (share + kChainSteps - 1) / kChainSteps;                        // chains of like length
    const int chain = (share + fewest - 1) / fewest;
    const float put_back = 1.0f + kCutOff<T> * (float)(chain * (kStepK / 16)), unit = kLog2e * put_back;
    const int works = tiles_m * tiles_n * splits;
    const int pair = blockIdx.x / S::kCtas, pairs = gridDim.x / S::kCtas;

    if (warp == 0) {
        // ---- copies in (all lanes wait, one issues)
        int s = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int i = pair; i < works && ok; i += pairs) {
            const Work w = work_of(i, tiles_m, tiles_n);
            const int k_first = (int)((long long)steps * w.split / splits), k_last = (int)((long long)steps * (w.split + 1) / splits);
            const int m0 = w.m * kRows + (int)rank * kHalf, n0 = w.n * kTile + (int)rank * kHalf;
            for (int k = k_first; k < k_last; ++k) {
                ok = __all_sync(0xffffffffu, umma::barrier_wait(umma::shared_address(&bar_empty[s]), phase ^ 1u, failed));
                if (!ok) break;
                if (umma::elected()) {
                    const uint32_t full = umma::in_cta(umma::shared_address(&bar_full[s]), 0);
                    if (rank == 0) umma::barrier_expect(umma::shared_address(&bar_full[s]), S::kCtas * kStageBytes);
                    const uint32_t a = stages + s * kStageBytes, b = a + kOperandBytes;
                    if (kAAcross) {
                        umma::tensor_load<PAIR>(a, &map_a, m0, k * kStepK, full);
                        umma::tensor_load<PAIR>(a + umma::kAcross, &map_a, m0 + 64, k * kStepK, full);
                    } else {
                        umma::tensor_load<PAIR>(a, &map_a, k * kStepK, m0, full);
                    }
#pragma unroll
                    for (int part = 0; part < (PAIR ? 1 : 2); ++part) {        // 128 rows of B each
                        const uint32_t to = b + part * kOperandBytes;
                        const int n = n0 + part * kHalf;
                        if (kBAcross) {
                            umma::tensor_load<PAIR>(to, &map_b, n, k * kStepK, full);
                            umma::tensor_load<PAIR>(to + umma::kAcross, &map_b, n + 64, k * kStepK, full);
                        } else {
                            umma::tensor_load<PAIR>(to, &map_b, k * kStepK, n, full);
                        }
                    }
                }
                __syncwarp();
                if (++s == kStages) { s = 0; phase ^= 1u; }
            }
        }
        if (!ok) __nanosleep(1000000);               // copies in flight land long before
    } else if (warp == 1 && rank == 0) {
        // ---- products (all lanes wait, one issues)
        int s = 0, buffer = 0;
        uint32_t phase = 0, buffer_phase = 0;
        bool ok = true;
        const uint64_t first_a = umma::operand(stages, kAAcross), first_b = umma::operand(stages + kOperandBytes, kBAcross);
        for (int i = pair; i < works && ok; i += pairs) {
            const Work w = work_of(i, tiles_m, tiles_n);
            const int k_first = (int)((long long)steps * w.split / splits), k_last = (int)((long long)steps * (w.split + 1) / splits);
            int link = 0;                                          // place within a chain of sums
            for (int k = k_first; k < k_last; ++k) {
                if (link == 0) {
                    ok = __all_sync(0xffffffffu, umma::barrier_wait(umma::shared_address(&bar_free[buffer]), buffer_phase ^ 1u, failed));
                    if (!ok) break;
                    umma::fence_after();
                }
                ok = __all_sync(0xffffffffu, umma::barrier_wait(umma::shared_address(&bar_full[s]), phase, failed));
                if (!ok) break;
                umma::fence_after();
                const bool ends = link == chain - 1 || k == k_last - 1;
                if (umma::elected()) {
                    const uint32_t sums = tensor_base + buffer * kTile;
                    const uint64_t da = first_a + (uint32_t)s * (kStageBytes >> 4), db = first_b + (uint32_t)s * (kStageBytes >> 4);
#pragma unroll
                    for (int j = 0; j < kStepK / 16; ++j)  // 16 of the summed axis: 32 bytes along a row, or two groups of 8 rows
                        umma::multiply<PAIR>(sums, da + (kAAcross ? j * 128 : j * 2), db + (kBAcross ? j * 128 : j * 2), kInstruction, link > 0 || j > 0);
                    umma::products_arrive<PAIR>(umma::shared_address(&bar_empty[s]));
                    if (ends) umma::products_arrive<PAIR>(umma::shared_address(&bar_sum[buffer]));
                }
                __syncwarp();
                if (++s == kStages) { s = 0; phase ^= 1u; }
                link = ends ? 0 : link + 1;
                if (ends && ++buffer == 2) { buffer = 0; buffer_phase ^= 1u; }
            }
        }
    } else if (warp >= 4) {
        // ---- results: this warp has 32 rows (its quarter of tensor memory) and 128 columns
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t own_outs = outs + (warp - 4) * S::kOuts * kOutBytes;
        int turn = 0;                                // which of them is written next
        const float unscale = kAAcross && !kSums ? P.control->unscale : 1.0f;
        const int share_rows = JOB == kDh ? P.control->share_rows : JOB == kDwSums ? P.dw_share_rows : 0;
        int buffer = 0;
        uint32_t phase = 0;
        for (int i = pair; i < works; i += pairs) {
            const Work w = work_of(i, tiles_m, tiles_n);
            const int row0 = w.m * kRows + (int)rank * kHalf + quarter * 32, row = row0 + lane;
            const int col0 = w.n * kTile + half * kHalf;
            int y = -1;
            float lse = 0.0f, g = 0.0f, at_label = 2.0f;
            if (kLogits) {
                if (row < rows) y = P.label[row] - P.first - col0;
                if (JOB == kDlogits && row < rows) {
                    lse = P.row_lse[row];
                    g = P.row_scale[row];
                    at_label = P.row_label[row];
                }
            }
            const uint32_t quarter_base = tensor_base + ((uint32_t)(quarter * 32) << 16) + half * kHalf;
            float top = -INFINITY, sum = 0.0f;
            bool add = P.add;
            // 64 columns from column c of this warp's, as bit patterns in u
            auto finish = [&](int c, uint32_t *u) {
                const int left = P.columns - (col0 + c);       // columns that exist from here on
                if (JOB == kLoss) {
                    if (left < 64) {
#pragma unroll
                        for (int j = 0; j < 64; ++j)
                            if (j >= left) u[j] = 0xff800000u;       // -inf
                    }
                    if (y >= c && y < c + 64) {
                        float mine = 0.0f;
#pragma unroll
                        for (int j = 0; j < 64; ++j) take_if(mine, y - c, j, u[j]);
                        P.label_logit[row] = mine * put_back;
                    }
                    float high = top;
#pragma unroll
                    for (int j = 0; j < 64; ++j) high = fmaxf(high, __uint_as_float(u[j]));
                    const float ref = high > -INFINITY ? high * unit : 0.0f;
                    sum *= exp2_fast((top > -INFINITY ? top * unit : -INFINITY) - ref);
#pragma unroll
                    for (int j = 0; j < 64; ++j) sum += exp2_fast(fmaf(__uint_as_float(u[j]), unit, -ref));
                    top = high;
                } else {
                    if (JOB == kDlogits) {
                        const int hit = y - c;
#pragma unroll
                        for (int j = 0; j < 64; ++j)
                            u[j] = __float_as_uint(exp2_fast(fmaf(__uint_as_float(u[j]), unit, -lse)));
                        if (hit >= 0 && hit < 64) {
#pragma unroll
                            for (int j = 0; j < 64; ++j)
                                if (j == hit) u[j] = __float_as_uint(at_label > 1.0f ? __uint_as_float(u[j]) - 1.0f : at_label);
                        }
#pragma unroll
                        for (int j = 0; j < 64; ++j) u[j] = __float_as_uint(__uint_as_float(u[j]) * g);
                        if (left < 64 || row0 + 32 > rows) {           // rows and columns that are only padding become zeros
                            const int mine = row < rows ? left : 0;
#pragma unroll
                            for (int j = 0; j < 64; ++j)
                                if (j >= mine) u[j] = 0u;
                        }
                    } else if (!kSums) {
#pragma unroll
                        for (int j = 0; j < 64; ++j) u[j] = __float_as_uint(__uint_as_float(u[j]) * unscale);
                    }
                    const bool wanted = JOB == kDlogits ? row0 < (some_rows + kStepK - 1) / kStepK * kStepK
                                        : JOB == kDh ? row0 < rows : row0 < P.result_rows;
                    constexpr int kBoxes = kSums ? 2 : 1;         // 128 bytes a row: 32 fp32 or 64 16-bit columns
#pragma unroll
                    for (int box = 0; box < kBoxes; ++box) {
                        const uint32_t out = own_outs + turn * kOutBytes;
                        turn = (turn + 1) % S::kOuts;
                        if (lane == 0) umma::stores_read<S::kOuts - 1>();
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            uint4 v;
                            if (kSums)
                                v = make_uint4(u[32 * box + 4 * j], u[32 * box + 4 * j + 1], u[32 * box + 4 * j + 2], u[32 * box + 4 * j + 3]);
                            else {
                                uint32_t p[4];
#pragma unroll
                                for (int q = 0; q < 4; ++q) {
                                    const int at = 8 * j + 2 * q;
                                    p[q] = pack2<T>(__uint_as_float(u[at]), __uint_as_float(u[at + 1]));
                                }
                                v = make_uint4(p[0], p[1], p[2], p[3]);
                            }
                            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(out + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(v.x),
                                         "r"(v.y), "r"(v.z), "r"(v.w)
                                         : "memory");
                        }
                        umma::copies_see_shared();
                        __syncwarp();
                        if (lane == 0) {
                            const int x = col0 + c + box * 32;
                            if (wanted && (JOB == kDlogits || x < P.columns)) {
                                if (kSums && add) umma::tensor_add(&map_out, x, w.split * share_rows + row0, out);
                                else umma::tensor_store(&map_out, x, w.split * share_rows + row0, out);
                            }
                            umma::stores_commit();
                        }
                    }
                }
            };
            const int k_first = (int)((long long)steps * w.split / splits), k_last = (int)((long long)steps * (w.split + 1) / splits);
            const int chains = (k_last - k_first + chain - 1) / chain;
            bool ok = true;
            // the accumulator of the next chain: there, and given back when it is in registers
            auto take = [&]() {
                ok = __all_sync(0xffffffffu, umma::barrier_wait(umma::shared_address(&bar_sum[buffer]), phase, failed));
                umma::fence_after();
                return ok;
            };
            auto give = [&]() {
                umma::fence_before();
                __syncwarp();
                if (lane == 0) umma::barrier_arrive_at(umma::in_cta(umma::shared_address(&bar_free[buffer]), 0));
            };
            if constexpr (kLogits || JOB == kDwLong) {
                uint32_t total[kHalf];
#pragma unroll 1
                for (int q = 0; q < chains; ++q) {
                    if (!take()) break;
                    const uint32_t sums = quarter_base + buffer * kTile;
                    if (q == 0) {
#pragma unroll
                        for (int c = 0; c < kHalf; c += 32) umma::tensor_memory_load(sums + c, total + c);
                        umma::tensor_memory_loaded<kHalf>(total);
                    } else {
#pragma unroll
                        for (int c = 0; c < kHalf; c += 16) {
                            uint32_t t[16];
                            umma::tensor_memory_load16(sums + c, t);
                            umma::tensor_memory_loaded<16>(t);
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                total[c + j] = __float_as_uint(__uint_as_float(total[c + j]) + __uint_as_float(t[j]));
                        }
                    }
                    give();
                    if (++buffer == 2) { buffer = 0; phase ^= 1u; }
                }
                if (!ok) break;
                finish(0, total);
                finish(64, total + 64);
            } else {
#pragma unroll 1
                for (int q = 0; q < chains; ++q) {
                    if (!take()) break;
                    if (q > 0) {                         // always in the same order: the chain before lies in memory
                        add = true;
                        if (lane == 0) umma::stores_done();
                    }
                    const uint32_t sums = quarter_base + buffer * kTile;
#pragma unroll 1
                    for (int c = 0; c < kHalf; c += 64) {
                        uint32_t u[64];
                        umma::tensor_memory_load(sums + c, u);
                        umma::tensor_memory_load(sums + c + 32, u + 32);
                        umma::tensor_memory_loaded<64>(u);
                        if (c == kHalf - 64) give();
                        finish(c, u);
                    }
                    if (++buffer == 2) { buffer = 0; phase ^= 1u; }
                }
                if (!ok) break;
            }
            if (JOB == kLoss && row < rows)
                P.stats[(long long)((P.first + col0) / kHalf) * P.stats_ld + row] = make_float2(top > -INFINITY ? top * unit : -INFINITY, sum);
        }
        if (lane == 0) umma::stores_done();
    }
    __syncwarp();
    umma::fence_before();
    __syncthreads();
    umma::cluster_sync();                        // nobody reads the other's shared or tensor memory any more
    umma::fence_after();
    if (warp == 2) umma::tensor_memory_give<PAIR>(tensor_base);
    if (threadIdx.x == 0 && *failed) atomicExch(&P.control->error, 1);
}

// ---------------------------------------------------------------------------
// Joining the pieces
// ---------------------------------------------------------------------------
constexpr int kJoinRows = 32, kJoinParts = 32;   // a block: 32 compact rows, each joined by 32 threads

struct JoinParams {
    const float2 *stats;
    long long stats_ld;
    int parts;
    XentControl *control;
    const int *row_of;
    const float *label_logit;
    float *rows_out, *lse_out, *loss;
    double *partials;                            // one per block
    int reduction;
};

__device__ __forceinline__ void join(float &top, float &sum, float top2, float sum2)
{
    // maxima leave NaN out, sums carry it on
    const float both = fmaxf(top, top2), ref = both > -INFINITY ? both : 0.0f;
    sum = sum * exp2f(top - ref) + sum2 * exp2f(top2 - ref);
    top = both;
}

// lse and loss of every row from its parts' maxima and sums; the block that
// comes last adds up the loss, always in the same order.
__global__ void __launch_bounds__(kJoinRows * kJoinParts) psops_xent_join_kernel(const JoinParams P)
{
    __shared__ float tops[kJoinParts][kJoinRows + 1], sums[kJoinParts][kJoinRows + 1];
    __shared__ double row_loss[kJoinRows];
    __shared__ bool last;
    after_the_kernel_before();
    const int rows = P.control->rows;
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int r = blockIdx.x * kJoinRows + lane;
    float top = -INFINITY, sum = 0.0f;
    if (r < rows)
        for (int k = part; k < P.parts; k += 8 * kJoinParts) {
            float2 s[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                s[j] = k + j * kJoinParts < P.parts ? P.stats[(k + j * kJoinParts) * P.stats_ld + r] : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) join(top, sum, s[j].x, s[j].y);
        }
    tops[part][lane] = top;
    sums[part][lane] = sum;
    __syncthreads();
    // warp `part` joins the parts of row `part`, a lane for each
    top = tops[lane][part];
    sum = sums[lane][part];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const float top2 = __shfl_xor_sync(0xffffffffu, top, off), sum2 = __shfl_xor_sync(0xffffffffu, sum, off);
        join(top, sum, top2, sum2);
    }
    if (lane == 0) {
        const int row = blockIdx.x * kJoinRows + part;
        double loss = 0.0;
        if (row < rows) {
            const float lse = P.control->error ? NAN : (top + log2f(sum)) * kLn2, mine = lse - P.label_logit[row];
            const int t = P.row_of[row];
            if (P.rows_out != nullptr) P.rows_out[t] = mine;
            if (P.lse_out != nullptr) P.lse_out[t] = lse;
            loss = mine;
        }
        row_loss[part] = loss;
    }
    __syncthreads();
    if (part == 0) {
        double loss = row_loss[lane];
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, off);
        if (lane == 0) {
            P.partials[blockIdx.x] = loss;
            __threadfence();
            last = atomicAdd(&P.control->tickets, 1u) == gridDim.x - 1;
        }
    }
    __syncthreads();
    if (!last || threadIdx.x >= 32) return;
    __threadfence();
    if (lane == 0) P.control->tickets = 0;
    if (P.loss == nullptr) return;
    double total = 0.0;
    for (unsigned b = lane; b < gridDim.x; b += 32) total += __ldcg(P.partials + b);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
    if (lane == 0) *P.loss = P.control->error ? NAN : P.reduction == PSOPS_MEAN ? (float)(total / (double)max(1, rows)) : (float)total;
}

// dh in the caller's rows from the compact sums, rounded once; zero where a
// token is left out.  DW: dw from its shares' sums (row for row).  The launch for
// dh is a call's last one and runs for dw alone too (with no rows then): where a
// product gave up it leaves no numbers in either rather than wrong ones.
struct OutParams {
    const float *sums;
    long long sums_ld;
    const XentControl *control;
    const int *compact_of;
    int rows, dim, dw_share_rows;
    bool aligned;
    void *out;
    long long ld;
    void *dw;                                    // dh's launch: dw, or NULL
    long long dw_ld, dw_rows;
};

template <class T, bool DW>
__global__ void __launch_bounds__(kCopyThreads) psops_xent_out_kernel(const OutParams P)
{
    after_the_kernel_before();
    const bool error = P.control->error != 0;
    const float counts = error ? NAN : P.control->unscale, left_out = error ? NAN : 0.0f;      // an unscale that is not finite stays with the tokens that count
    const int shares = DW ? P.control->dw_shares : P.control->shares, dim = P.dim;
    const long long share = (DW ? P.dw_share_rows : P.control->share_rows) * P.sums_ld;
    const unsigned groups = (dim + 3) / 4;
    for (long long i = (long long)blockIdx.x * kCopyThreads + threadIdx.x; i < (long long)P.rows * groups; i += (long long)gridDim.x * kCopyThreads) {
        const int t = (int)(i / groups), d = (int)(i - (long long)t * groups) * 4;
        const int r = DW ? t : P.compact_of[t];
        T *out = (T *)P.out + t * P.ld + d;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        const float unscale = r >= 0 ? counts : left_out;
        if (r >= 0) {
            const float *in = P.sums + r * P.sums_ld + d;
#pragma unroll 4
            for (int s = 0; s < shares; ++s) {
                const float4 a = *reinterpret_cast<const float4 *>(in + s * share);
                v.x += a.x; v.y += a.y; v.z += a.z; v.w += a.w;
            }
        }
        const uint2 u = make_uint2(pack2<T>(v.x * unscale, v.y * unscale), pack2<T>(v.z * unscale, v.w * unscale));
        if (P.aligned && d + 4 <= dim) {
            *reinterpret_cast<uint2 *>(out) = u;
        } else {
            T e[4];
            memcpy(e, &u, 8);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (d + j < dim) out[j] = e[j];
        }
    }
    if (DW || !error || P.dw == nullptr) return;
    const uint16_t nothing = (uint16_t)pack2<T>(NAN, NAN);
    for (long long i = (long long)blockIdx.x * kCopyThreads + threadIdx.x; i < P.dw_rows * dim; i += (long long)gridDim.x * kCopyThreads) {
        const long long v = i / dim;
        ((uint16_t *)P.dw)[v * P.dw_ld + (i - v * dim)] = nothing;
    }
}

} // namespace
