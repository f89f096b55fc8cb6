// Softmax cross entropy of an output layer, for n workers' tokens at once, with its gradients, and without the logits in memory.
//
//   z_i = W h_i,  lse_i = log sum_v exp(z_iv),  loss_w = mean over the labelled tokens of worker w of (lse_i - z_i,label)
//   dz_iv = (exp(z_iv - lse_i) - [v = label_i]) * grad_w / count_w,  dh_i = sum_v dz_iv W_v,  dW^(w)_v = sum_i in w dz_iv h_i
//
// Forward: tiles of z = W H' stay in registers; a tile leaves, per token, its largest logit and its sum of exponentials, which a
// second kernel joins over the vocabulary.  Backward: for some workers after the others, the tiles of z again, from
// which dz goes to scratch as 16-bit words, and from there into the two products.  (The logits kept as 32-bit numbers would save a
// quarter of the products for rows * vocab * 8 bytes of traffic, and as 16-bit numbers would spoil exp(z).)
//
// dz at the label, p - 1, is minus the sum of the token's other probabilities too, and made so where that is below 1/2: where the label is
// nearly certain, 1 - p is far smaller than what the rounding of lse to 32 bits leaves uncertain of p (a token whose loss was 4e-5 beside
// a log-sum of 190 had gradients 16 % off).  The tiles that make dz add the others up; the word of such a label is written when the whole
// vocabulary is there.  Only where one worker's dz is too large for the scratch does it go by pieces of the vocabulary, with a pass over
// the logits before them for the sums.
//
// All but the smallest are bound by the matrix cores: 8 x 1024 tokens of 768 against 50,257 words in bf16 take 2.47 ms for four products
// of 632 GFLOP, 1.02 PFLOP/s with everything between them (the library's largest plain product: 1.54); in 32 bits 4 x 511 tokens
// 1.9 ms, of which 0.19 are the words of W made twice, at the rate of a copy.  A handful of tokens (4 x 5 of 256, 4,001 words)
// takes 51 us, eleven launches of 2.3 to 9 us that each wait for the one before.
//
// Words: tensors of 16 bits are multiplied as they are; those of 32 bits as pairs of 16-bit floats (22 bits), scaled by the power of two
// that takes the tensor's largest finite number to 2^14.  dz is kept without grad_w / count_w (which the products' results are
// multiplied by), as words of the same kind: 8 or 11 bits beside 16-bit tensors, 22 beside 32-bit ones; in 16-bit floats times 2^14, so
// that probabilities down to 2^-38 are not lost.
#include <math.h>
#include <algorithm>
#include <new>
#include <type_traits>
#include <utility>

#include "sams_gemm.h"
#include "sams_train.h"

struct sams_xent {
    int32_t n, type, train;
    int64_t t_max, dim, vocab, piece, dz_bytes;
    hipStream_t stream;
    sams::Scratch scratch;
    int64_t h, w, dz, dh, part, token, at_label, inv, amax, exps;
};

namespace sams {

using namespace gemm;

constexpr int64_t kXentPieceBytes = (int64_t)1 << 30;        // of dz, of some workers' tokens or one piece of the vocabulary
// of one worker's dz, if there is as much memory: by pieces the backward pass of 16,384 tokens of 768 and 50,257 words takes 5.0 ms, whole 3.9
constexpr int64_t kXentWorkerBytes = (int64_t)4 << 30;
constexpr int kAmaxBlocks = 1024;
constexpr float kLog2e = 1.44269504088896340736f;

constexpr int64_t kPartBytes = (int64_t)256 << 20;          // of partial sums of dh, at most (but one for every token)
constexpr int kMaxSplit = 64;
constexpr int64_t kMostBlocks = 1 << 20;                    // workgroups of 256 that go from row to row

template <int KIND> __host__ __device__ constexpr int dz_exponent() { return KIND == BF16 ? 0 : 14; }
template <int T> constexpr int kind_of() { return T == SAMS_F32 ? SPLIT : T == SAMS_BF16 ? BF16 : F16; }

__device__ __forceinline__ bool takes_part(const int64_t *labels, int64_t row, int64_t vocab)
{
    return (uint64_t)labels[row] < (uint64_t)vocab;
}

// largest finite |value| over the rows (those that take no part left out), one result per block: of H in the first blocks, of W in the others
__global__ void __launch_bounds__(256) k_xent_amax(const float *h, Rows hs, int64_t t, int64_t rows, const int64_t *labels, const float *w, int64_t w_row,
                                                   int64_t vocab, int64_t dim, float *amax)
{
    __shared__ float best[4];
    const bool of_w = blockIdx.x >= kAmaxBlocks;
    const int block = of_w ? blockIdx.x - kAmaxBlocks : blockIdx.x;
    const int64_t count = of_w ? vocab : rows;
    float m = 0.f;
    for (int64_t r = block * (int64_t)4 + (threadIdx.x >> 6); r < count; r += kAmaxBlocks * 4) {
        const float *p;
        if (of_w) {
            p = w + r * w_row;
        } else {
            if (!takes_part(labels, r, vocab)) continue;
            p = h + r / t * hs.worker + r % t * hs.row;
        }
        for (int64_t i = (threadIdx.x & 63) * 4; i < dim; i += 256) {
            uint32_t raw[4];
            load_piece<SAMS_F32>(p, i, dim, raw);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = fabsf(__builtin_bit_cast(float, raw[e]));
                m = v <= 3.402823466e38f ? fmaxf(m, v) : m;
            }
        }
    }
    m = wave_max(m);
    if ((threadIdx.x & 63) == 0) best[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) amax[blockIdx.x] = fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3]));
}

// what k_xent_pack packs: rows of a tensor into rows of words; rows that take no part (labels given) become zeros, whatever they hold
struct Packed {
    const void *src;
    Rows at;
    int64_t t, rows;                    // rows of a worker, rows; none: nothing to pack
    const int64_t *labels;
    uint16_t *out;
};

// H by the first blocks, W by the next, and grad_w / count_w (0 where a worker has no labelled token) by the last n, where asked for
template <int T, int KIND>
__global__ void __launch_bounds__(256) k_xent_pack(Packed H, unsigned blocks_h, Packed W, unsigned blocks_w, int64_t dim, int64_t vocab, const float *amax, int32_t *exps,
                                                   const int64_t *labels, int64_t t, const float *grad, float *inv)
{
    if (blockIdx.x >= blocks_h + blocks_w) {
        __shared__ int64_t counts[4];
        const int64_t worker = blockIdx.x - blocks_h - blocks_w;
        int c = 0;
        for (int64_t i = threadIdx.x; i < t; i += 256) c += takes_part(labels, worker * t + i, vocab);
#pragma unroll
        for (int o = 32; o; o >>= 1) c += __shfl_xor(c, o);
        if ((threadIdx.x & 63) == 0) counts[threadIdx.x >> 6] = c;
        __syncthreads();
        const int64_t count = counts[0] + counts[1] + counts[2] + counts[3];
        if (threadIdx.x == 0) inv[worker] = count ? (grad ? grad[worker] : 1.f) / (float)count : 0.f;
        return;
    }
    const bool of_w = blockIdx.x >= blocks_h;
    const Packed p = of_w ? W : H;
    const unsigned block = of_w ? blockIdx.x - blocks_h : blockIdx.x, blocks = of_w ? blocks_w : blocks_h;
    const int lane = threadIdx.x & 63;
    float scale = 1.f;
    if constexpr (KIND == SPLIT) {
        float m = 0.f;
        static_assert(kAmaxBlocks % 256 == 0, "");
#pragma unroll
        for (int i = 0; i < kAmaxBlocks / 256; ++i) {
            const float4 a = ((const float4 *)(amax + (of_w ? kAmaxBlocks : 0)))[i * 64 + lane];
            m = fmaxf(m, fmaxf(fmaxf(a.x, a.y), fmaxf(a.z, a.w)));
        }
        m = wave_max(m);
        int e = 0;
        if (m > 0) {
            (void)frexpf(m, &e);
            e = 15 - e;                                              // the largest at 2^14 to 2^15
            if (e > 126) e = 126;
        }
        scale = ldexpf(1.f, e);
        if (block == 0 && threadIdx.x == 0) exps[of_w] = e;
    }
    const int64_t width = row_numbers<KIND>(dim), ld = row_words<KIND>(dim);
    for (int64_t r = block * (int64_t)4 + (threadIdx.x >> 6); r < p.rows; r += blocks * (int64_t)4) {
        const bool used = !p.labels || takes_part(p.labels, r, vocab);
        const typename TypeOf<T>::type *from = (const typename TypeOf<T>::type *)p.src + r / p.t * p.at.worker + r % p.t * p.at.row;
        for (int64_t i = lane * 8; i < width; i += 512) {
            float v[8];
            load8<T>(from, i, used ? dim : 0, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= scale;
            put8<KIND>(p.out + r * ld, i, v);
        }
    }
}

// 1 / the scale of H (0), of W (1), of both (2).  Of both, at least 2^-126: a product of words is below 2^48, and a logit of 2^-78 in place of
// a smaller one moves nothing, whereas 0 would make NaN of the -infinity that stands for words which are none.
template <int KIND>
__device__ __forceinline__ float unscale(const int32_t *exps, int which)
{
    if constexpr (KIND != SPLIT) return 1.f;
    return ldexpf(1.f, -(which == 0 ? exps[0] : which == 1 ? exps[1] : min(exps[0] + exps[1], 126)));
}

// (largest, sum of 2^(number - largest)) of two sets of numbers
__device__ __forceinline__ float2 join_sums(float2 a, float2 b)
{
    const float top = fmaxf(a.x, b.x), base = top == -INFINITY ? 0.f : top;
    return make_float2(top, a.y * __builtin_amdgcn_exp2f(a.x - base) + b.y * __builtin_amdgcn_exp2f(b.x - base));
}

// Whether the workgroups go from tile to tile, the next tile's first stage on its way while the sums of one are made: 16-bit words do (8192 x
// 50257 x 768: 655 -> 618 us; 4096 x 32000 x 1024: 257 -> 245), pairs, whose tiles of 256 leave no registers for it, gain nothing
// (2044 x 50257 x 768: 464, 461).
template <int KIND> constexpr bool kStatsInTurn = KIND != SPLIT;

// Bound by the matrix cores, and by the exponentials while these wait: 8192 tokens of 768 and 50,257
// words 611 us, 1.03 PFLOP/s in bf16; pairs 0.34.
//
// Per token and tile of the vocabulary: the largest logit, in units of log 2, and the sum of 2^(logit - largest) over the words but the
// label.  A lane holds numbers of one token (32 of a tile's 64), so that the maximum and the sum run over its registers.  The label's
// product is left in `at_label`, as it is, by the lane that holds it: see token_loss.
template <class S, int KIND>
__global__ void __launch_bounds__(S::THREADS) k_xent_stats(Operand W, Operand H, int64_t dim, uint32_t first, uint32_t tiles_v, uint32_t tiles_t, const int32_t *exps, const int64_t *labels,
                                                           float2 *part, float *at_label)
{
    __shared__ __align__(16) char lds[S::LDS_BYTES];
    typedef Product<S, KIND, false, false> Logits;
    constexpr bool ON = kStatsInTurn<KIND>;
    float2 *joined = (float2 *)(lds + (ON ? (S::STAGES - 1) * Logits::STAGE : 0));           // [WAVES_M][BN]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / S::WAVES_N, wn = wave % S::WAVES_N;
    const uint32_t tiles = tiles_v * tiles_t;
    uint32_t id = first + blockIdx.x, mi, ni, batch;
    tile_place(id, tiles, tiles_v, tiles_t, mi, ni, batch);
    Logits logits;
    logits.start(W, (int64_t)mi * S::BM, H, (int64_t)ni * S::BN, 0, dim, lds);
    for (;;) {
        const int64_t m0 = (int64_t)mi * S::BM, n0 = (int64_t)ni * S::BN;
        const uint32_t tile_v = mi;
        int64_t at[S::NI];                                               // the tokens' labels, under way during the product
#pragma unroll
        for (int j = 0; j < S::NI; ++j) {
            const int64_t row = n0 + (wn * S::NI + j) * 32 + (lane & 31);
            at[j] = row < H.size ? labels[row] : -1;
        }
        f32x16 acc[S::MI][S::NI];
        clear<S>(acc);
        logits.finish(acc, dim, lds);
        if constexpr (ON) {
            id += gridDim.x;
            if (id < tiles) {
                tile_place(id, tiles, tiles_v, tiles_t, mi, ni, batch);
                logits.start(W, (int64_t)mi * S::BM, H, (int64_t)ni * S::BN, 0, dim, lds);
            }
        }
        int label[S::NI];                                                // where they lie among the wavefront's words; -1: elsewhere
#pragma unroll
        for (int j = 0; j < S::NI; ++j) {
            asm volatile("" : "+v"(at[j]));                              // not looked at before
            const int64_t in = at[j] - m0 - wm * S::MI * 32;
            label[j] = at[j] < W.size && in >= 0 && in < S::MI * 32 ? (int)in : -1;
        }
        const float f = kLog2e * unscale<KIND>(exps, 2);
        if (m0 + S::BM > W.size) {                                       // rows past the vocabulary
#pragma unroll
            for (int i = 0; i < S::MI; ++i)
#pragma unroll
                for (int q = 0; q < 16; ++q)
                    if (m0 + (wm * S::MI + i) * 32 + 8 * (q >> 2) + 4 * (lane >> 5) + (q & 3) >= W.size)
#pragma unroll
                        for (int j = 0; j < S::NI; ++j) acc[i][j][q] = -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < S::NI; ++j) {
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int i = 0; i < S::MI; ++i)
#pragma unroll
                for (int q = 0; q < 16; ++q) top = fmaxf(top, acc[i][j][q]);
            if (__any(label[j] >= 0)) {
                const int own = label[j] >= 0 && (label[j] >> 2 & 1) == lane >> 5 ? label[j] & ~4 : -1;
                float z = 0.f;
#pragma unroll
                for (int i = 0; i < S::MI; ++i)
#pragma unroll
                    for (int q = 0; q < 16; ++q)
                        if (own == i * 32 + 8 * (q >> 2) + (q & 3)) {
                            z = acc[i][j][q];
                            acc[i][j][q] = -INFINITY;
                        }
                if (own >= 0) at_label[n0 + (wn * S::NI + j) * 32 + (lane & 31)] = z;
            }
            top = fmaxf(top, __shfl_xor(top, 32)) * f;
            const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int i = 0; i < S::MI; ++i)
#pragma unroll
                for (int q = 0; q < 16; ++q) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][q], f, -base));
            sum += __shfl_xor(sum, 32);
            if (lane < 32) joined[wm * S::BN + (wn * S::NI + j) * 32 + lane] = make_float2(top, sum);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < S::BN; i += S::THREADS) {
            float2 a = joined[i];
#pragma unroll
            for (int w = 1; w < S::WAVES_M; ++w) a = join_sums(a, joined[w * S::BN + i]);
            if (n0 + i < H.size) part[tile_v * H.size + n0 + i] = a;
        }
        if (!ON || id >= tiles) return;
        __syncthreads();                                             // the stage that `joined` lies in is loaded next
    }
}

// What the tiles left of 16 tokens (a line of `part`) joined over the vocabulary by a workgroup, each tile's by one of 16 threads in turn;
// the first 16 threads get their token's.
//
// With S the sum of 2^(z_v - top) over the words but the label, and d = top - z_label, a token's loss is log(1 + S 2^d).  d comes from
// the label's product by one fma, against the same rounded `top` that the terms of S were taken against, so that the loss keeps its
// digits where the label is nearly certain, however large the logits, and is never below 0.
struct TokenSums { float top, rest, d; };
template <int KIND>
__device__ __forceinline__ TokenSums token_sums(const float2 *part, int tiles_v, const float *at_label, const int32_t *exps, int64_t first, int64_t end, int64_t rows,
                                                float2 (&joined)[4][16])
{
    const int r = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int64_t row = first + r;
    float2 sums = make_float2(-INFINITY, 0.f);
    if (row < end)
#pragma unroll 4
        for (int i = g; i < tiles_v; i += 16) sums = join_sums(sums, part[i * rows + row]);
#pragma unroll
    for (int o = 16; o < 64; o <<= 1) sums = join_sums(sums, make_float2(__shfl_xor(sums.x, o), __shfl_xor(sums.y, o)));
    if ((threadIdx.x & 63) < 16) joined[threadIdx.x >> 6][r] = sums;
    __syncthreads();
    sums = join_sums(join_sums(joined[0][r], joined[1][r]), join_sums(joined[2][r], joined[3][r]));
    const float top = sums.x == -INFINITY ? 0.f : sums.x;
    return TokenSums{top, sums.y, row < end ? -__builtin_fmaf(at_label[row], kLog2e * unscale<KIND>(exps, 2), -top) : 0.f};
}

template <int KIND>
__device__ __forceinline__ float token_loss(const float2 *part, int tiles_v, const float *at_label, const int32_t *exps, const int64_t *labels, int64_t first, int64_t end,
                                            int64_t rows, int64_t vocab, float *lse, float2 (&joined)[4][16])
{
    const TokenSums k = token_sums<KIND>(part, tiles_v, at_label, exps, first, end, rows, joined);
    const int64_t row = first + threadIdx.x;
    if (threadIdx.x >= 16 || row >= end) return 0.f;
    if (!takes_part(labels, row, vocab)) {
        lse[row] = 0.f;
        return 0.f;
    }
    const float log_sum = log2f(k.rest + exp2f(-k.d));
    lse[row] = (k.top + log_sum) * (1.f / kLog2e);
    return k.d > 32.f ? (k.d + log_sum) * (1.f / kLog2e) : log1pf(k.rest * exp2f(k.d));      // (2^d may be too large where 2^-d is small)
}

template <int KIND>
__global__ void __launch_bounds__(256) k_xent_join(const float2 *part, int tiles_v, const float *at_label, const int32_t *exps, const int64_t *labels, int64_t rows, int64_t vocab, float *lse,
                                                   float *token)
{
    __shared__ float2 joined[4][16];
    for (int64_t first = blockIdx.x * (int64_t)16; first < rows; first += gridDim.x * (int64_t)16) {
        const float loss = token_loss<KIND>(part, tiles_v, at_label, exps, labels, first, rows, rows, vocab, lse, joined);
        if (threadIdx.x < 16 && first + threadIdx.x < rows) token[first + threadIdx.x] = loss;
        __syncthreads();
    }
}

// The same and the mean over a worker's tokens in one launch, a workgroup per worker, where there are few (kJoinTokens, kJoinTiles): 1.5 us
// less of 48.8 for 4 x 5 tokens.
constexpr int kJoinTokens = 64, kJoinTiles = 2048;
template <int KIND>
__global__ void __launch_bounds__(256) k_xent_join_few(const float2 *part, int tiles_v, const float *at_label, const int32_t *exps, const int64_t *labels, int t, int64_t rows, int64_t vocab, float *lse,
                                                       float *loss)
{
    __shared__ float2 joined[4][16];
    const int64_t begin = blockIdx.x * (int64_t)t;
    float sum = 0.f;
    int count = 0;
    for (int i = 0; i < t; i += 16) {
        sum += token_loss<KIND>(part, tiles_v, at_label, exps, labels, begin + i, begin + t, rows, vocab, lse, joined);
        if (threadIdx.x < 16 && i + threadIdx.x < t) count += takes_part(labels, begin + i + threadIdx.x, vocab);
        __syncthreads();
    }
    if (threadIdx.x >= 16) return;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) { sum += __shfl_xor(sum, o); count += __shfl_xor(count, o); }
    if (threadIdx.x == 0) loss[blockIdx.x] = count ? sum / (float)count : 0.f;
}

// a worker's mean; tokens are added up in the same order every time
__global__ void __launch_bounds__(256) k_xent_loss(const float *token, const int64_t *labels, int64_t t, int64_t vocab, float *loss)
{
    __shared__ float sums[4];
    __shared__ int64_t counts[4];
    float s = 0.f;
    int c = 0;
    for (int64_t i = threadIdx.x; i < t; i += 256) {
        s += token[blockIdx.x * t + i];
        c += takes_part(labels, blockIdx.x * t + i, vocab);
    }
    s = wave_sum(s);
#pragma unroll
    for (int o = 32; o; o >>= 1) c += __shfl_xor(c, o);
    if ((threadIdx.x & 63) == 0) { sums[threadIdx.x >> 6] = s; counts[threadIdx.x >> 6] = c; }
    __syncthreads();
    if (threadIdx.x) return;
    const int64_t count = counts[0] + counts[1] + counts[2] + counts[3];
    loss[blockIdx.x] = count ? (sums[0] + sums[1] + sums[2] + sums[3]) / (float)count : 0.f;
}

// dz over the vocabulary or one piece of it (W: the piece), a row of words per token.  703 us at 8192 x 50,257 x 768 in bf16, 0.90 PFLOP/s: beside
// the product an exponential each, and 823 MB written, a wavefront's rows through LDS so that they leave in whole lines.
//
// rest == NULL: dz at the label is p - 1 for now, and `sums` [tiles_v][rows] gets each token's sum over the tile of the others; else `rest` is
// the sum over all.
struct Token { float base; int label; float rest; };                 // log2 of the scale less the log-sum; the label's place in the tile; the others' sum, if known
constexpr int kNoLabel = -1;
// whether dz at the label is -rest (in dz's scale)
template <int KIND> __device__ __forceinline__ bool mostly_label(float rest) { return rest < 0.5f * (float)(1 << dz_exponent<KIND>()); }
template <class S, int KIND>
__global__ void __launch_bounds__(S::THREADS) k_xent_dz(Operand W, Operand H, int64_t dim, Launch launch, uint32_t tiles_v, uint32_t tiles_t, const int32_t *exps, const int64_t *labels, int64_t v0,
                                                        int64_t vocab, const float *lse, uint16_t *dz, const float *rest, float *sums)
{
    __shared__ __align__(16) char lds[S::LDS_BYTES];
    __shared__ Token tokens[S::BN];
    __shared__ float joined[S::WAVES_M][S::BN];
    uint32_t mi, ni, batch;
    tile_place(launch, tiles_v, tiles_t, mi, ni, batch);
    const int64_t m0 = (int64_t)mi * S::BM, n0 = (int64_t)ni * S::BN;
    static_assert(S::BN <= S::THREADS, "a thread for each of the tile's tokens");
    const int64_t row = n0 + threadIdx.x;
    const bool mine = threadIdx.x < S::BN && row < H.size;
    int64_t label = mine ? labels[row] : -1;                         // under way during the product
    float log_sum = mine ? lse[row] : 0.f;
    f32x16 acc[S::MI][S::NI];
    clear<S>(acc);
    tile_product<S, KIND, false, false>(acc, W, m0, H, n0, 0, dim, lds);
    asm volatile("" : "+v"(label), "+v"(log_sum));                   // not looked at before
    if (threadIdx.x < S::BN) {
        const int64_t at = label - v0 - m0;
        const bool part = label >= 0 && label < vocab;               // elsewhere 2^(0 - infinity) = 0
        const bool here = part && at >= 0 && at < S::BM;
        tokens[threadIdx.x] = Token{part ? dz_exponent<KIND>() - log_sum * kLog2e : -INFINITY, here ? (int)at : kNoLabel, here && rest ? rest[row] : INFINITY};
    }
    __syncthreads();
    const float f = kLog2e * unscale<KIND>(exps, 2), one = (float)(1 << dz_exponent<KIND>());
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / S::WAVES_N, wn = wave % S::WAVES_N;
    float sum[S::NI];
    int block = -1;
    const int limit = W.size - m0 < S::BM ? (int)(W.size - m0) : S::BM;          // of the tile's words, in the vocabulary
    constexpr int BYTES = KIND == SPLIT ? 4 : 2;
    const int64_t row_bytes = row_words<KIND>(W.size) * 2;
    char *corner = (char *)dz + n0 * row_bytes + m0 * BYTES;
    store_rows<S, BYTES, KIND == SPLIT>(
        acc, lds,
        [&](int n) {
            const Token k = tokens[n];
            sum[++block] = 0.f;
            return std::make_pair(k, __any(k.label != kNoLabel) != 0);
        },
        [&](const std::pair<Token, bool> &kl, int m, const float (&z)[4]) {
            const Token &k = kl.first;
            float g[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) g[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[e], f, k.base));
            if (limit < S::BM) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (m + e >= limit) g[e] = 0.f;
            }
            float four = (g[0] + g[1]) + (g[2] + g[3]);
            if (kl.second) {
                float others[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool it = m + e == k.label;
                    others[e] = it ? 0.f : g[e];
                    g[e] = it ? (mostly_label<KIND>(k.rest) ? -k.rest : g[e] - one) : g[e];
                }
                four = (others[0] + others[1]) + (others[2] + others[3]);
            }
            sum[block] += four;
            return pack_words<KIND>(g);
        },
        [&](int n, int at, u32x4 w) {
            if (n0 + n < H.size && m0 * BYTES + at < row_bytes) *(u32x4 *)(corner + n * row_bytes + at) = w;
        });
    if (rest) return;
#pragma unroll
    for (int j = 0; j < S::NI; ++j) {
        sum[j] += __shfl_xor(sum[j], 32);
        if (lane < 32) joined[wm][(wn * S::NI + j) * 32 + lane] = sum[j];
    }
    __syncthreads();
    if (!mine) return;
    float all = joined[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < S::WAVES_M; ++w) all += joined[w][threadIdx.x];
    sums[mi * H.size + row] = all;
}

// The words of nearly certain labels, minus the sum of the others: 16 tokens by a workgroup, each tile's sums by one of 16 threads in turn.
template <int KIND>
__global__ void __launch_bounds__(256) k_xent_dz_label(const float *sums, int tiles_v, const int64_t *labels, int64_t rows, int64_t vocab, uint16_t *dz, int64_t ld)
{
    __shared__ float joined[4][16];
    const int r = threadIdx.x & 15, g = threadIdx.x >> 4;
    for (int64_t first = blockIdx.x * (int64_t)16; first < rows; first += gridDim.x * (int64_t)16) {
        const int64_t row = first + r;
        float sum = 0.f;
        if (row < rows)
#pragma unroll 4
            for (int i = g; i < tiles_v; i += 16) sum += sums[i * rows + row];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if ((threadIdx.x & 63) < 16) joined[threadIdx.x >> 6][r] = sum;
        __syncthreads();
        sum = (joined[0][r] + joined[1][r]) + (joined[2][r] + joined[3][r]);
        __syncthreads();
        if (threadIdx.x >= 16 || row >= rows || !takes_part(labels, row, vocab) || !mostly_label<KIND>(sum)) continue;
        const float v[4] = {-sum, 0.f, 0.f, 0.f};
        const auto w = pack_words<KIND>(v);
        const int64_t label = labels[row];
        if constexpr (KIND == SPLIT) {
            uint16_t *p = dz + row * ld + (label >> 5) * 64 + (label & 31);
            p[0] = (uint16_t)w[0];
            p[32] = (uint16_t)w[2];
        } else {
            dz[row * ld + label] = (uint16_t)w[0];
        }
    }
}

// The same sums from the log-sums' parts, in dz's scale: 1 - p = S 2^d / (1 + S 2^d).
template <int KIND>
__global__ void __launch_bounds__(256) k_xent_rest(const float2 *part, int tiles_v, const float *at_label, const int32_t *exps, int64_t rows, float *rest)
{
    __shared__ float2 joined[4][16];
    for (int64_t first = blockIdx.x * (int64_t)16; first < rows; first += gridDim.x * (int64_t)16) {
        const TokenSums k = token_sums<KIND>(part, tiles_v, at_label, exps, first, rows, rows, joined);
        if (threadIdx.x < 16 && first + threadIdx.x < rows) rest[first + threadIdx.x] = (float)(1 << dz_exponent<KIND>()) * (k.rest / (k.rest + exp2f(-k.d)));
        __syncthreads();
    }
}

// dW of one worker and piece.  ADD: to what is there, as 32-bit numbers.  Both operands lie with their k's, the tokens, as rows; a worker's
// products are its own, so that there are tiles enough without a split of k.  682 us at 8 x 1024 x 50,257 x 768 in bf16, 0.93 PFLOP/s,
// with 617 MB written.
template <class S, int KIND, int T, bool ADD>
__global__ void __launch_bounds__(S::THREADS) k_xent_dw(const uint16_t *dz, int64_t piece, const uint16_t *h, int64_t dim, int64_t t, Launch launch, uint32_t tiles_d, uint32_t tiles_v,
                                                        const int32_t *exps, const float *inv, typename TypeOf<T>::type *dw, Rows ds)
{
    typedef typename TypeOf<T>::type E;
    __shared__ __align__(16) char lds[S::LDS_BYTES];
    uint32_t mi, ni, batch;
    tile_place(launch, tiles_d, tiles_v, mi, ni, batch);
    const int64_t m0 = (int64_t)mi * S::BM, n0 = (int64_t)ni * S::BN, worker = batch;
    const int64_t ldz = row_words<KIND>(piece), ldh = row_words<KIND>(dim);
    const Operand Z{dz + worker * t * ldz, ldz, piece}, H{h + worker * t * ldh, ldh, dim};
    f32x16 acc[S::MI][S::NI];
    clear<S>(acc);
    tile_product<S, KIND, true, true>(acc, H, m0, Z, n0, 0, t, lds);
    const float f = inv[worker] / (float)(1 << dz_exponent<KIND>()), fh = unscale<KIND>(exps, 0);       // apart: together they may be too small
    E *out = dw + worker * ds.worker + n0 * ds.row;
    typedef typename std::conditional<ADD, float, E>::type Staged;
    store_rows<S, sizeof(Staged), false>(
        acc, lds, [](int) { return 0; },
        [&](int, int, const float (&v)[4]) {
            const float r[4] = {v[0] * f * fh, v[1] * f * fh, v[2] * f * fh, v[3] * f * fh};
            return pack_numbers<Staged>(r);
        },
        [&](int n, int at, u32x4 w) {
            const int64_t i = m0 + at / (int)sizeof(Staged);
            if (n0 + n >= piece || i >= dim) return;
            E *row = out + n * ds.row;
            if constexpr (ADD) {
                float v[4];
                __builtin_memcpy(v, &w, 16);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + e < dim) row[i + e] = (E)((float)row[i + e] + v[e]);
            } else {
                store_numbers(row, i, dim, w);
            }
        });
}

// dh over one piece, its vocabulary cut into parts; a part's sums are added to those of the pieces before.  part: [parts][rows][pitch]
// The result has few tiles (96 of 256 x 256 for 8192 tokens of 768) and k is the vocabulary: the parts make them enough for the chip.
// 578 us at 8192 x 50,257 x 768 in bf16, 1.09 PFLOP/s, and 24 us to join the parts.
template <class S, int KIND>
__global__ void __launch_bounds__(S::THREADS) k_xent_dh(const uint16_t *dz, int64_t piece, Operand W, int64_t rows, Launch launch, uint32_t tiles_d, uint32_t tiles_t, int first, float *part,
                                                        int64_t pitch, uint32_t parts)
{
    __shared__ __align__(16) char lds[S::LDS_BYTES];
    uint32_t mi, ni, batch;
    tile_place(launch, tiles_d, tiles_t, mi, ni, batch);
    const int64_t m0 = (int64_t)mi * S::BM, n0 = (int64_t)ni * S::BN;
    const int64_t steps = (piece + tile_k<KIND>() - 1) / tile_k<KIND>();
    const int64_t lo = steps * batch / parts * tile_k<KIND>(), hi = steps * (batch + 1) / parts * tile_k<KIND>();
    const Operand Z{dz, row_words<KIND>(piece), rows};
    f32x16 acc[S::MI][S::NI];
    clear<S>(acc);
    tile_product<S, KIND, true, false>(acc, W, m0, Z, n0, lo, (hi < piece ? hi : piece) - lo, lds);
    float *out = part + (batch * rows + n0) * pitch + m0;
    store_rows<S, 4, false>(acc, lds, [](int) { return 0; }, [](int, int, const float (&v)[4]) { return pack_numbers<float>(v); },
                            [&](int n, int at, u32x4 w) {
                                if (n0 + n >= rows || m0 + at / 4 >= pitch) return;
                                float *o = out + n * pitch + at / 4, v[4];
                                __builtin_memcpy(v, &w, 16);
                                const float4 was = first ? make_float4(0.f, 0.f, 0.f, 0.f) : *(const float4 *)o;
                                *(float4 *)o = make_float4(was.x + v[0], was.y + v[1], was.z + v[2], was.w + v[3]);
                            });
}

// joins the parts, in ascending order; a wavefront per row
template <int KIND, int T>
__global__ void __launch_bounds__(256) k_xent_dh_join(const float *part, int parts, int64_t rows, int64_t pitch, int64_t t, int64_t dim, const int32_t *exps, const float *inv,
                                                      typename TypeOf<T>::type *dh, Rows ds)
{
    for (int64_t row = blockIdx.x * (int64_t)4 + (threadIdx.x >> 6); row < rows; row += gridDim.x * (int64_t)4) {
        const float f = inv[row / t] / (float)(1 << dz_exponent<KIND>()), fw = unscale<KIND>(exps, 1);   // apart: together they may be too small
        typename TypeOf<T>::type *out = dh + row / t * ds.worker + row % t * ds.row;
        constexpr int N = kPiece<T>;
        for (int64_t i = (threadIdx.x & 63) * N; i < dim; i += 64 * N) {
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = 0.f;
#pragma unroll 4
            for (int p = 0; p < parts; ++p) {
                const float *at = part + (p * rows + row) * pitch + i;
#pragma unroll
                for (int e = 0; e < N; e += 4) {
                    const float4 a = i + e < pitch ? *(const float4 *)(at + e) : make_float4(0.f, 0.f, 0.f, 0.f);
                    v[e] += a.x; v[e + 1] += a.y; v[e + 2] += a.z; v[e + 3] += a.w;
                }
            }
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = v[e] * f * fw;
            store_piece<T>(out, i, dim, v);
        }
    }
}

static int64_t dz_words(int64_t vocab) { return (vocab + 255) / 256 * 256; }       // room for a token's, in numbers
static int64_t dh_pitch(int64_t dim) { return (dim + 3) / 4 * 4; }

// the tile of dh's product over one piece, and the parts that the vocabulary is cut into for it
static TileChoice dh_tiles(bool pairs, int64_t rows, int64_t dim, int64_t piece)
{
    const int64_t bytes = rows * dh_pitch(dim) * 4, room = kPartBytes / bytes, most = std::min<int64_t>(kMaxSplit, (piece + 255) / 256);
    return choose_tiles(pairs, 1, dim, rows, false, piece, (int)std::max<int64_t>(1, std::min(room, most)), bytes * 2 / 4000.0);      // 4 TB/s
}

// H and W as operands, packed where the tensors themselves are not fit to be loaded from; backward: H without the rows that take no part,
// and inv
template <int T, int KIND>
static int enqueue_operands(sams_xent *c, int64_t t, const void *h, Rows hs, const void *w, int64_t w_row, const int64_t *labels, bool backward, const float *grad, Operand *H,
                            Operand *W)
{
    const int64_t rows = c->n * t, ld = row_words<KIND>(c->dim);
    float *amax = c->scratch.at<float>(c->amax);
    auto fit = [&](int64_t row, const void *p) { return KIND != SPLIT && c->dim % 8 == 0 && row % 8 == 0 && row <= kMaxRowWords && aligned16(p); };
    Packed ph = {h, hs, t, rows, labels, c->scratch.at<uint16_t>(c->h)}, pw = {w, Rows{0, w_row}, c->vocab, c->vocab, nullptr, c->scratch.at<uint16_t>(c->w)};
    *H = Operand{ph.out, ld, rows};
    *W = Operand{pw.out, ld, c->vocab};
    if (!backward && (c->n == 1 || hs.worker == t * hs.row) && fit(hs.row, h)) {
        *H = Operand{(const uint16_t *)h, hs.row, rows};
        ph.rows = 0;
    }
    if (fit(w_row, w)) {
        *W = Operand{(const uint16_t *)w, w_row, c->vocab};
        pw.rows = 0;
    }
    if (rows == 0) ph.rows = pw.rows = 0;
    const unsigned blocks_h = ph.rows ? grid_for(ph.rows, 4, 2048) : 0, blocks_w = pw.rows ? grid_for(pw.rows, 4, 4096) : 0, blocks = blocks_h + blocks_w + (backward ? c->n : 0);
    if (KIND == SPLIT && rows)
        hipLaunchKernelGGL(k_xent_amax, dim3(2 * kAmaxBlocks), dim3(256), 0, c->stream, (const float *)h, hs, t, rows, labels, (const float *)w, w_row, c->vocab, c->dim, amax);
    if (blocks)
        hipLaunchKernelGGL((k_xent_pack<T, KIND>), dim3(blocks), dim3(256), 0, c->stream, ph, blocks_h, pw, blocks_w, c->dim, c->vocab, amax, c->scratch.at<int32_t>(c->exps), labels, t,
                           grad, c->scratch.at<float>(c->inv));
    SAMS_HIP(hipGetLastError());
    return SAMS_OK;
}

// the log-sums' parts of rows tokens; the tiles of the vocabulary
template <int KIND>
static uint32_t enqueue_stats(sams_xent *c, const Operand &W, const Operand &H, const int64_t *labels)
{
    uint32_t tv = 0;
    with_tile<KIND>(choose_tiles(KIND == SPLIT, 1, c->vocab, H.size, false, c->dim, 1, 0).shape, [&](auto shape) {
        typedef decltype(shape) S;
        tv = (uint32_t)((c->vocab + S::BM - 1) / S::BM);
        const uint32_t tt = (uint32_t)((H.size + S::BN - 1) / S::BN);
        auto launch = [&](dim3 grid, uint32_t first) {
            hipLaunchKernelGGL((k_xent_stats<S, KIND>), grid, dim3(S::THREADS), 0, c->stream, W, H, c->dim, first, tv, tt, c->scratch.at<int32_t>(c->exps), labels,
                               c->scratch.at<float2>(c->part), c->scratch.at<float>(c->at_label));
        };
        if (kStatsInTurn<KIND>) launch(dim3(at_once<S>(tv * tt)), 0);
        else in_launches((int64_t)tv * tt, S::THREADS, [&](dim3 grid, Launch l) { launch(grid, l.first); });
    });
    return tv;
}

template <int T>
static int enqueue_forward(sams_xent *c, int64_t t, const void *h, Rows hs, const void *w, int64_t w_row, const int64_t *labels, float *loss, float *lse)
{
    constexpr int KIND = kind_of<T>();
    const int64_t rows = c->n * t;
    float *token = c->scratch.at<float>(c->token), *at_label = c->scratch.at<float>(c->at_label);
    const int32_t *exps = c->scratch.at<int32_t>(c->exps);
    if (rows) {
        Operand H, W;
        SAMS_TRY((enqueue_operands<T, KIND>(c, t, h, hs, w, w_row, labels, false, nullptr, &H, &W)));
        float2 *part = c->scratch.at<float2>(c->part);
        const uint32_t tv = enqueue_stats<KIND>(c, W, H, labels);
        if (t <= kJoinTokens && tv <= kJoinTiles) {
            hipLaunchKernelGGL(k_xent_join_few<KIND>, dim3((unsigned)c->n), dim3(256), 0, c->stream, part, (int)tv, at_label, exps, labels, (int)t, rows, c->vocab, lse, loss);
            SAMS_HIP(hipGetLastError());
            return SAMS_OK;
        }
        hipLaunchKernelGGL(k_xent_join<KIND>, dim3((unsigned)grid_for(rows, 16, kMostBlocks)), dim3(256), 0, c->stream, part, (int)tv, at_label, exps, labels, rows, c->vocab, lse, token);
    }
    hipLaunchKernelGGL(k_xent_loss, dim3((unsigned)c->n), dim3(256), 0, c->stream, token, labels, t, c->vocab, loss);
    SAMS_HIP(hipGetLastError());
    return SAMS_OK;
}

template <int T>
static int enqueue_backward(sams_xent *c, int64_t t, const void *h, Rows hs, const void *w, int64_t w_row, const int64_t *labels, const float *lse, const float *grad,
                            void *dh, Rows dhs, void *dw, Rows dws, int dw_type, int accumulate)
{
    constexpr int KIND = kind_of<T>();
    typedef typename TypeOf<T>::type E;
    const int32_t *exps = c->scratch.at<int32_t>(c->exps);
    uint16_t *dz = c->scratch.at<uint16_t>(c->dz);
    Operand allH, W;
    SAMS_TRY((enqueue_operands<T, KIND>(c, t, h, hs, w, w_row, labels, true, grad, &allH, &W)));
    float *part = c->scratch.at<float>(c->dh), *sums = c->scratch.at<float>(c->part), *rest = nullptr;
    const int64_t pitch = dh_pitch(c->dim), whole = dz_words(c->vocab), worker_bytes = t * whole * type_size(c->type);
    // as many workers at a time as the scratch has room for, evenly; or a worker by pieces of the vocabulary
    const bool pieces = t && (worker_bytes > c->dz_bytes || whole > kMaxRowWords / 2);
    const int64_t most = pieces ? 1 : worker_bytes ? std::min<int64_t>(c->n, c->dz_bytes / worker_bytes) : c->n, turns = (c->n + most - 1) / most, each = (c->n + turns - 1) / turns;
    for (int64_t first = 0; first < c->n; first += each) {
        const int64_t workers = std::min(each, c->n - first), rows = workers * t, row0 = first * t, size = pieces ? c->piece : c->vocab;
        const int64_t *label = labels + row0;
        const float *log_sums = lse + row0, *inv = c->scratch.at<float>(c->inv) + first;
        const Operand H{allH.p + row0 * allH.ld, allH.ld, rows};
        if (pieces) {
            rest = c->scratch.at<float>(c->token);
            const uint32_t tv = enqueue_stats<KIND>(c, W, H, label);
            hipLaunchKernelGGL(k_xent_rest<KIND>, dim3((unsigned)grid_for(rows, 16, kMostBlocks)), dim3(256), 0, c->stream, c->scratch.at<float2>(c->part), (int)tv, c->scratch.at<float>(c->at_label),
                               exps, rows, rest);
        }
        const TileChoice hidden = rows ? dh_tiles(KIND == SPLIT, rows, c->dim, size) : TileChoice{2, 0};
        const int parts = hidden.parts;
        for (int64_t v0 = 0; v0 < c->vocab; v0 += size) {
            const int64_t piece = std::min(size, c->vocab - v0);
            const Operand Wp{W.p + v0 * W.ld, W.ld, piece};
            if (rows)
                with_tile<KIND>(choose_tiles(KIND == SPLIT, 1, piece, rows, false, c->dim, 1, 0).shape, [&](auto shape) {
                    typedef decltype(shape) S;
                    const uint32_t tv = (uint32_t)((piece + S::BM - 1) / S::BM), tt = (uint32_t)((rows + S::BN - 1) / S::BN);
                    in_launches((int64_t)tv * tt, S::THREADS, [&](dim3 grid, Launch l) {
                        hipLaunchKernelGGL((k_xent_dz<S, KIND>), grid, dim3(S::THREADS), 0, c->stream, Wp, H, c->dim, l, tv, tt, exps, label, v0, c->vocab, log_sums, dz, rest, sums);
                    });
                    if (!rest)
                        hipLaunchKernelGGL(k_xent_dz_label<KIND>, dim3((unsigned)grid_for(rows, 16, kMostBlocks)), dim3(256), 0, c->stream, sums, (int)tv, label, rows, c->vocab, dz, row_words<KIND>(piece));
                });
            with_tile<KIND>(choose_tiles(KIND == SPLIT, workers, c->dim, piece, false, t, 1, 0).shape, [&](auto shape) {
                typedef decltype(shape) S;
                const uint32_t td = (uint32_t)((c->dim + S::BM - 1) / S::BM), tv = (uint32_t)((piece + S::BN - 1) / S::BN);
                auto weight = [&](auto kernel, auto *out) {
                    in_launches((int64_t)td * tv * workers, S::THREADS, [&](dim3 grid, Launch l) {
                        hipLaunchKernelGGL(kernel, grid, dim3(S::THREADS), 0, c->stream, dz, piece, H.p, c->dim, t, l, td, tv, exps, inv, out + first * dws.worker + v0 * dws.row, dws);
                    });
                };
                if (dw_type == SAMS_F32 && accumulate) weight(k_xent_dw<S, KIND, SAMS_F32, true>, (float *)dw);
                else if (dw_type == SAMS_F32) weight(k_xent_dw<S, KIND, SAMS_F32, false>, (float *)dw);
                else if (accumulate) weight(k_xent_dw<S, KIND, T, true>, (E *)dw);
                else weight(k_xent_dw<S, KIND, T, false>, (E *)dw);
            });
            if (rows)
                with_tile<KIND>(hidden.shape, [&](auto shape) {
                    typedef decltype(shape) S;
                    const uint32_t td = (uint32_t)((c->dim + S::BM - 1) / S::BM), tt = (uint32_t)((rows + S::BN - 1) / S::BN);
                    in_launches((int64_t)td * tt * parts, S::THREADS, [&](dim3 grid, Launch l) {
                        hipLaunchKernelGGL((k_xent_dh<S, KIND>), grid, dim3(S::THREADS), 0, c->stream, dz, piece, Operand{Wp.p, Wp.ld, c->dim}, rows, l, td, tt, v0 == 0, part, pitch,
                                           (uint32_t)parts);
                    });
                });
            SAMS_HIP(hipGetLastError());
        }
        if (rows)
            hipLaunchKernelGGL((k_xent_dh_join<KIND, T>), dim3((unsigned)grid_for(rows, 4, kMostBlocks)), dim3(256), 0, c->stream, part, parts, rows, pitch, t, c->dim, exps, inv,
                               (E *)dh + first * dhs.worker, dhs);
        SAMS_HIP(hipGetLastError());
    }
    return SAMS_OK;
}

static bool inputs_ok(const sams_xent *c, int64_t t, const void *h, int64_t h_worker, int64_t h_row, const void *w, int64_t w_row, const int64_t *labels)
{
    const int size = type_size(c->type);
    if (t < 0 || t > c->t_max || !w || !aligned_to(w, size) || w_row < 0 || h_worker < 0 || h_row < 0) return false;
    return t == 0 || (h && labels && aligned_to(h, size) && aligned_to(labels, 8));
}

}  // namespace sams

using namespace sams;

extern "C" {

int sams_xent_create(sams_xent **out, int32_t n, int64_t t_max, int64_t dim, int64_t vocab, int32_t type, int32_t train, void *hip_stream)
{
    if (!out) return SAMS_EINVAL;
    *out = nullptr;
    if (n < 1 || n > kMaxWorkers || t_max < 0 || t_max > SAMS_MAX_TOKENS / n || dim < 1 || dim > SAMS_MAX_DIM || vocab < 1 || vocab > SAMS_MAX_VOCAB || !type_ok(type))
        return SAMS_EINVAL;
    if ((n * t_max / Small::BN + 1) * (vocab / Small::BM + 1) > INT32_MAX) return SAMS_EINVAL;       // tiles are counted in 32 bits
    sams_xent *c = new (std::nothrow) sams_xent();
    if (!c) return SAMS_ENOMEM;
    c->n = n; c->t_max = t_max; c->dim = dim; c->vocab = vocab; c->type = type; c->train = train != 0;
    c->stream = (hipStream_t)hip_stream;
    const int64_t rows = n * t_max, ld = type == SAMS_F32 ? row_words<SPLIT>(dim) : row_words<F16>(dim), row_bytes = type_size(type), whole = dz_words(vocab),
                  worker_bytes = t_max * whole * row_bytes;
    auto take = [&](int64_t most) {                                  // most: of a worker's dz that is not cut into pieces
        c->scratch = Scratch{};
        c->h = c->scratch.reserve(rows * ld * 2);
        c->w = c->scratch.reserve(vocab * ld * 2);
        c->part = c->scratch.reserve(rows * ((vocab + Small::BM - 1) / Small::BM) * 8);
        c->token = c->scratch.reserve(rows * 4);
        c->at_label = c->scratch.reserve(rows * 4);
        c->inv = c->scratch.reserve(n * 4);
        c->amax = c->scratch.reserve(2 * kAmaxBlocks * 4);
        c->exps = c->scratch.reserve(2 * 4);
        if (train) {
            if (worker_bytes <= most && whole <= kMaxRowWords / 2) {
                c->piece = whole;
                c->dz_bytes = worker_bytes * (worker_bytes ? std::min<int64_t>(n, std::max<int64_t>(1, kXentPieceBytes / worker_bytes)) : 0);
            } else {
                c->piece = t_max ? kXentPieceBytes / (t_max * row_bytes) / 256 * 256 : whole;
                c->piece = std::min({std::max<int64_t>(c->piece, 1024), whole, kMaxRowWords / 2});
                c->dz_bytes = t_max * c->piece * row_bytes;
            }
            c->dz = c->scratch.reserve(c->dz_bytes);
            // for fewer tokens there may be more parts, in as much memory
            c->dh = c->scratch.reserve(std::max(rows * dh_pitch(dim) * 4, std::min(kPartBytes, rows * dh_pitch(dim) * 4 * kMaxSplit)));
        }
        return c->scratch.take();
    };
    int rc = take(kXentWorkerBytes);
    if (rc == SAMS_ENOMEM && train && worker_bytes > kXentPieceBytes && worker_bytes <= kXentWorkerBytes) rc = take(kXentPieceBytes);
    if (rc == SAMS_OK) rc = enqueue_fill_u32_on(nullptr, c->stream, c->scratch.at<uint32_t>(c->exps), 2, 0u);
    if (rc != SAMS_OK) {
        if (c->scratch.base) (void)hipFree(c->scratch.base);
        delete c;
        return rc;
    }
    *out = c;
    return SAMS_OK;
}

int sams_xent_destroy(sams_xent *c)
{
    if (!c) return SAMS_OK;
    hipError_t e = hipStreamSynchronize(c->stream);
    if (c->scratch.base) (void)hipFree(c->scratch.base);
    delete c;
    if (e != hipSuccess) { g_last_hip_error = (int)e; return SAMS_EHIP; }
    return SAMS_OK;
}

int64_t sams_xent_scratch_bytes(const sams_xent *c) { return c ? c->scratch.bytes : 0; }

int linear_xent_forward(sams_xent *c, int64_t t, const void *h, int64_t h_worker, int64_t h_row, const void *w, int64_t w_row, const int64_t *labels, float *loss, float *lse)
{
    if (!c || !inputs_ok(c, t, h, h_worker, h_row, w, w_row, labels) || !loss || !aligned_to(loss, 4) || (t > 0 && (!lse || !aligned_to(lse, 4)))) return SAMS_EINVAL;
    SAMS_BY_TYPE(c->type, T, return enqueue_forward<T>(c, t, h, Rows{h_worker, h_row}, w, w_row, labels, loss, lse));
}

int linear_xent_backward(sams_xent *c, int64_t t, const void *h, int64_t h_worker, int64_t h_row, const void *w, int64_t w_row, const int64_t *labels, const float *lse,
                         const float *grad_loss, void *dh, int64_t dh_worker, int64_t dh_row, void *dw, int64_t dw_worker, int64_t dw_row, int32_t dw_type, int32_t accumulate)
{
    if (!c || !c->train || !inputs_ok(c, t, h, h_worker, h_row, w, w_row, labels) || !aligned_to(grad_loss, 4)) return SAMS_EINVAL;
    if (dw_type != c->type && dw_type != SAMS_F32) return SAMS_EINVAL;
    if (!dw || !aligned_to(dw, type_size(dw_type)) || (c->vocab > 1 && dw_row < c->dim) || (c->n > 1 && dw_worker < c->dim)) return SAMS_EINVAL;
    if (t > 0 && (!lse || !aligned_to(lse, 4) || !dh || !aligned_to(dh, type_size(c->type)) || (t > 1 && dh_row < c->dim) || (c->n > 1 && dh_worker < c->dim))) return SAMS_EINVAL;
    SAMS_BY_TYPE(c->type, T, return enqueue_backward<T>(c, t, h, Rows{h_worker, h_row}, w, w_row, labels, lse, grad_loss, dh, Rows{dh_worker, dh_row}, dw,
                                                        Rows{dw_worker, dw_row}, dw_type, accumulate));
}

}  // extern "C"
