// Updates orthogonalised by Newton-Schulz steps, alone or within a momentum update of weight matrices.
//
//   X_0 = G / (|G|_F + eps);   X_{j+1} = p(X_j) = a X + b (X X') X + c (X X')^2 X = (a I + b A + c A^2) X,  A = X X'
//
// p acts on the singular values s of X: s -> a s + b s^3 + c s^5, with X's directions left alone.  A is formed on the shorter side
// (for a tall matrix A = X' X, and X multiplies from the left), so that a step is three products: X X' (or X' X), A A, and P X
// (or X P).  A and P are symmetric: half of their tiles are computed, each written twice.
//
// Numbers.  Every matrix of the iteration has a bound that the coefficients give on the host: |x_ij| <= the largest singular value,
// which p keeps below max |p| over the range before.  So they are held as fixed-point-like words: 16-bit floats (11 bits) after
// scaling by a power of two that puts the bound near the top of their range: pairs of words (22 bits), or single ones for large bfloat16
// matrices (bfloat16's own 8 bits cost the same and would add up to several roundings of the result; nothing here needs their
// range).  G itself is only scaled by the power of two that brings its norm to 2^14 to 2^15, which loses nothing of a 16-bit G's
// numbers above 2^-29 of the norm and up to 2^-39 of the norm of smaller ones; the rest of 1 / (|G| + eps) goes into the first step's products.
//
// Large matrices are bound by the matrix cores: five steps of one 4096 x 8192 in bf16 take 2.36 ms, 1.02 PFLOP/s over everything; 12 of
// 768 x 768 in 32 bits from 8 workers' gradients 565 us (0.19 PFLOP/s of pairs, each product one or two rounds of tiles), 78 of them
// for the gradients' bytes.  Small ones are bound by the steps' chain: 50 of 84 x 120 take 52 us.
#include <math.h>
#include <new>

#include "sams_gemm.h"
#include "sams_train.h"

struct sams_ortho {
    int64_t batch, rows, cols;
    int32_t type;
    hipStream_t stream;
    sams::Scratch scratch;
    int64_t x[2], gram, poly, scale, part, update, sums; // offsets in the scratch
};

namespace sams {

using namespace gemm;

// Words between the products are pairs, but single ones for large bfloat16 matrices: there the roundings of a matrix's many numbers average
// out against its singular directions.  Off the 64-bit result (2-norm; bfloat16's own rounding is 1.7e-3 of it): single words 3.6e-3 at
// 32 x 768, 2.3e-3 at 512 x 8013, 2.0e-3 at 1024 x 1024, 1.9e-3 at 4096 x 8192, where pairs would take about twice the time.
constexpr int64_t kSingleMin = 1024;    // of the shorter side
static bool ortho_pairs(int type, int64_t rows, int64_t cols) { return type != SAMS_BF16 || rows < kSingleMin || cols < kSingleMin; }

constexpr int kNormSlices = 512;        // of a matrix, for the sum of its squares

struct OrthoScale {
    float sigma, sigma2;                // what the words of G still have to be multiplied by, and its square
    int32_t exponent;                   // words of G = G * 2^exponent
};

__device__ __forceinline__ OrthoScale ortho_scale(double norm, float eps)
{
    int e = 0;
    if (norm > 0 && isfinite(norm)) {
        (void)frexp(norm, &e);
        e = 15 - e;                                                  // norm * 2^e in [2^14, 2^15)
    }
    const double sigma = norm > 0 ? ldexp(1.0 / (norm + (double)eps), -e) : (norm == 0 ? 0.0 : norm);
    return OrthoScale{(float)sigma, (float)(sigma * sigma), e};
}

// sums of squares in 64 bits: no norm is too large or too small for its square; a wavefront per row
template <int T>
__global__ void __launch_bounds__(256) k_ortho_squares(const typename TypeOf<T>::type *g, int64_t g_mat, int64_t g_row, int64_t rows, int64_t cols, double *part)
{
    __shared__ double sums[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double s = 0;
    for (int64_t r = blockIdx.x * 4 + wave; r < rows; r += kNormSlices * 4) {
        const typename TypeOf<T>::type *p = g + blockIdx.y * g_mat + r * g_row;
        for (int64_t i = lane * 8; i < cols; i += 512) {
            float v[8];
            load8<T>(p, i, cols, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) s = __builtin_fma((double)v[e], (double)v[e], s);
        }
    }
    s = wave_sum(s);
    if (lane == 0) sums[wave] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.y * kNormSlices + blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// m' = beta m + (1 - beta) mean_i g_i (workers in ascending order); the matrix to orthogonalise is m', or beta m' + (1 - beta) mean g,
// and the sum of its squares is made on the way.  Bound by memory: 8 workers' 12 matrices of 768 x 768 60 us, 5.1 TB/s.
__global__ void __launch_bounds__(256) k_muon_head(const float *g, int64_t g_worker, int64_t g_mat, int32_t n, const float *m, int64_t m_mat, float *m_out, int64_t m_out_mat,
                                                   float beta, int nesterov, float *update, int64_t elems, double *part)
{
    __shared__ double sums[4];
    const float rest = 1.f - beta, workers = (float)n;
    const float *pg = g + blockIdx.y * g_mat;
    double s = 0;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < elems; i += kNormSlices * 1024) {
        float mean[4] = {0.f, 0.f, 0.f, 0.f}, mi[4], u[4];
#pragma unroll 4
        for (int w = 0; w < n; ++w) {
            uint32_t raw[4];
            float v[4];
            load_piece<SAMS_F32>(pg + w * g_worker, i, elems, raw);
            widen<SAMS_F32>(raw, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) mean[e] += v[e];
        }
        uint32_t raw[4];
        load_piece<SAMS_F32>(m + blockIdx.y * m_mat, i, elems, raw);
        widen<SAMS_F32>(raw, mi);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float share = rest * (mean[e] / workers);
            mi[e] = beta * mi[e] + share;
            u[e] = nesterov ? beta * mi[e] + share : mi[e];
            if (i + e < elems) s = __builtin_fma((double)u[e], (double)u[e], s);
        }
        store_piece<SAMS_F32>(m_out + blockIdx.y * m_out_mat, i, elems, mi);
        store_piece<SAMS_F32>(update + blockIdx.y * elems, i, elems, u);
    }
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.y * kNormSlices + blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// the words of X_0, and what they stand for
template <int T, int KIND>
__global__ void __launch_bounds__(256) k_ortho_words(const typename TypeOf<T>::type *g, int64_t g_mat, int64_t g_row, int64_t rows, int64_t cols, float eps,
                                                     const double *part, OrthoScale *scale, uint16_t *x)
{
    __shared__ double norm;
    if (threadIdx.x < 64) {
        double s = 0;
        for (int i = threadIdx.x; i < kNormSlices; i += 64) s += part[blockIdx.y * kNormSlices + i];
        s = wave_sum(s);
        if (threadIdx.x == 0) norm = sqrt(s);
    }
    __syncthreads();
    const OrthoScale by_norm = ortho_scale(norm, eps);
    if (blockIdx.x == 0 && threadIdx.x == 0) scale[blockIdx.y] = by_norm;
    const double by = ldexp(1.0, by_norm.exponent);
    const int64_t width = row_numbers<KIND>(cols), ld = row_words<KIND>(cols);
    for (int64_t r = blockIdx.x * 4 + (threadIdx.x >> 6); r < rows; r += gridDim.x * 4) {
        const typename TypeOf<T>::type *p = g + blockIdx.y * g_mat + r * g_row;
        uint16_t *o = x + (blockIdx.y * rows + r) * ld;
        for (int64_t i = (threadIdx.x & 63) * 8; i < width; i += 512) {
            float v[8];
            load8<T>(p, i, cols, v);
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = (float)((double)v[q] * by);
            put8<KIND>(o, i, v);
        }
    }
}

struct OrthoDims {
    int64_t rows, cols, small;          // of X; small = min(rows, cols)
};

// tile number `run` of the lower triangles, and its matrix
__device__ __forceinline__ void triangle_at(uint32_t run, int64_t tiles, int &i, int &j, int64_t &matrix)
{
    const uint32_t each = (uint32_t)(tiles * (tiles + 1) / 2);
    matrix = run / each;
    const int id = (int)(run % each);
    i = (int)((sqrtf(8.f * (float)id + 1.f) - 1.f) * 0.5f);
    while ((i + 1) * (i + 2) / 2 <= id) ++i;
    while (i * (i + 1) / 2 > id) --i;
    j = id - i * (i + 1) / 2;
}
__device__ __forceinline__ void triangle(int64_t tiles, int &i, int &j, int64_t &matrix)           // a workgroup's
{
    triangle_at(tile_run(blockIdx.x, gridDim.x), tiles, i, j, matrix);
}

// Writes a symmetric matrix's tile and its mirror image, with zeros in what fills the rows up; value(row, col, v) makes eight numbers of them.
template <class S, int KIND, typename F>
__device__ __forceinline__ void put_symmetric(uint16_t *o, int64_t ld, int64_t small, int64_t m0, int64_t n0, const f32x16 (&acc)[S::MI][S::NI], char *lds, F value)
{
    const int64_t width = row_numbers<KIND>(small);
    auto emit = [&](int64_t row, int64_t col, const float (&raw)[8]) {
        if (row >= small || col >= width) return;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = raw[e];
        value(row, col, v);
        if (col + 8 > small) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e >= small) v[e] = 0.f;
        }
        put8<KIND>(o + row * ld, col, v);
    };
    eights<S, false>(acc, lds, [&](int dn, int dm, const float (&raw)[8]) { emit(n0 + dn, m0 + dm, raw); });
    if (m0 != n0) eights<S, true>(acc, lds, [&](int dm, int dn, const float (&raw)[8]) { emit(m0 + dm, n0 + dn, raw); });
}

// A = X X' (X' X where X is tall), times f and, in the first step, sigma^2.  161 us at 4096 x 8192 in single words, 0.85 PFLOP/s of the half
// that is computed: 253 tiles of 192 fill the chip once, where 136 of 256 would take half of it.
template <class S, int KIND, bool TALL>
__global__ void __launch_bounds__(S::THREADS) k_ortho_gram(const uint16_t *x, OrthoDims d, float f, const OrthoScale *scale, uint16_t *gram)
{
    __shared__ __align__(16) char lds[S::LDS_BYTES];
    int ti, tj;
    int64_t matrix;
    triangle((d.small + S::BM - 1) / S::BM, ti, tj, matrix);
    const int64_t m0 = (int64_t)ti * S::BM, n0 = (int64_t)tj * S::BN, ldx = row_words<KIND>(d.cols), ldg = row_words<KIND>(d.small);
    const Operand X{x + matrix * d.rows * ldx, ldx, TALL ? d.cols : d.rows};
    f32x16 acc[S::MI][S::NI];
    clear<S>(acc);
    tile_product<S, KIND, TALL, TALL>(acc, X, m0, X, n0, 0, TALL ? d.rows : d.cols, lds);
    if (scale) f *= scale[matrix].sigma2;
    put_symmetric<S, KIND>(gram + matrix * d.small * ldg, ldg, d.small, m0, n0, acc, lds, [&](int64_t, int64_t, float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= f;
    });
}

// The same where a few tiles' k's are long: the k's in parts, whose sums of 64 x 64 numbers lie one after the other (tiles fastest) and
// are added up in ascending order by k_ortho_gram_join.  Orthogonalised in 32 bits: 8 of 64 x
// 5145 275 us whole, 188 cut; 3 of 320 x 8192 513, 353; one of 256 x 1024 125, 133, and not cut.
constexpr int kGramParts = 32;          // of k, at most, and as many as make a tile for every CU
constexpr int kGramTiles = 256;         // parts of all tiles, at most
template <int KIND, bool TALL>
__global__ void __launch_bounds__(Small::THREADS) k_ortho_gram_part(const uint16_t *x, OrthoDims d, uint32_t tiles, uint32_t parts, float *sums)
{
    typedef Small S;
    __shared__ __align__(16) char lds[S::LDS_BYTES];
    const uint32_t part = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    int ti, tj;
    int64_t matrix;
    triangle_at(tile, (d.small + S::BM - 1) / S::BM, ti, tj, matrix);
    const int64_t m0 = (int64_t)ti * S::BM, n0 = (int64_t)tj * S::BN, ldx = row_words<KIND>(d.cols), k = TALL ? d.rows : d.cols;
    const int64_t steps = (k + tile_k<KIND>() - 1) / tile_k<KIND>();
    const int64_t lo = steps * part / parts * tile_k<KIND>(), hi = steps * (part + 1) / parts * tile_k<KIND>();
    const Operand X{x + matrix * d.rows * ldx, ldx, TALL ? d.cols : d.rows};
    f32x16 acc[S::MI][S::NI];
    clear<S>(acc);
    tile_product<S, KIND, TALL, TALL>(acc, X, m0, X, n0, lo, (hi < k ? hi : k) - lo, lds);
    float *out = sums + (int64_t)blockIdx.x * (S::BM * S::BN);
    eights<S, false>(acc, lds, [&](int dn, int dm, const float (&v)[8]) {
        float4 *o = (float4 *)(out + dn * S::BM + dm);
        o[0] = make_float4(v[0], v[1], v[2], v[3]);
        o[1] = make_float4(v[4], v[5], v[6], v[7]);
    });
}

// a quarter of a tile and of its mirror image (blockIdx.y) by a workgroup
template <int KIND>
__global__ void __launch_bounds__(256) k_ortho_gram_join(const float *sums, uint32_t tiles, uint32_t parts, OrthoDims d, float f, const OrthoScale *scale, uint16_t *gram)
{
    constexpr int B = Small::BM;
    int ti, tj;
    int64_t matrix;
    triangle_at(blockIdx.x, (d.small + B - 1) / B, ti, tj, matrix);
    const bool mirror = threadIdx.x >= 128;
    if (mirror && ti == tj) return;
    const int at = blockIdx.y * 128 + (threadIdx.x & 127), r = at / (B / 8), c = at % (B / 8) * 8;
    const int64_t row = (int64_t)(mirror ? ti : tj) * B + r, col = (int64_t)(mirror ? tj : ti) * B + c;
    if (row >= d.small || col >= row_numbers<KIND>(d.small)) return;
    if (scale) f *= scale[matrix].sigma2;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (uint32_t p = 0; p < parts; ++p) {
        const float *tile = sums + ((int64_t)p * tiles + blockIdx.x) * (B * B);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += mirror ? tile[(c + e) * B + r] : tile[r * B + c + e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = col + e < d.small ? v[e] * f : 0.f;
    const int64_t ld = row_words<KIND>(d.small);
    put8<KIND>(gram + matrix * d.small * ld + row * ld, col, v);
}

// P = a I + b A + c A A: 99 us at 4096, 0.70 PFLOP/s of the half that is computed, 253 tiles of 192 on 256 CUs.
template <class S, int KIND>
__global__ void __launch_bounds__(S::THREADS) k_ortho_poly(const uint16_t *gram, OrthoDims d, float a, float b, float c, uint16_t *poly)
{
    __shared__ __align__(16) char lds[S::LDS_BYTES];
    int ti, tj;
    int64_t matrix;
    triangle((d.small + S::BM - 1) / S::BM, ti, tj, matrix);
    const int64_t m0 = (int64_t)ti * S::BM, n0 = (int64_t)tj * S::BN, ld = row_words<KIND>(d.small);
    const Operand A{gram + matrix * d.small * ld, ld, d.small};
    f32x16 acc[S::MI][S::NI];
    clear<S>(acc);
    tile_product<S, KIND, false, false>(acc, A, m0, A, n0, 0, d.small, lds);
    put_symmetric<S, KIND>(poly + matrix * d.small * ld, ld, d.small, m0, n0, acc, lds, [&](int64_t row, int64_t col, float (&v)[8]) {
        float g[8];
        get8<KIND>(A.p + row * ld, col, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (row == col + e ? a : 0.f) + b * g[e] + c * v[e];
    });
}

// eight parameters from `at` on, of which those from `limit` on do not exist (0): in pieces of 16 bytes where they do (one by one, the last
// step's products of 12 matrices of 768 x 768 take 70 us, so 57)
__device__ __forceinline__ void load_numbers(const float *row, int64_t at, int64_t limit, float (&v)[8])
{
    typedef float anywhere __attribute__((ext_vector_type(4), aligned(4)));
    if (at + 8 <= limit) {
        const anywhere a = *(const anywhere *)(row + at), b = *(const anywhere *)(row + at + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = at + e < limit ? row[at + e] : 0.f;
    }
}

// where the last step's X goes
struct OrthoOut {
    void *out;                          // the caller's tensor
    int64_t out_mat, out_row;
    const float *x;                     // or: parameters, x_out = keep * x - rate * X
    int64_t x_mat;
    float keep, rate;
};

// 233 us at 4096 x 8192 in single words, 1.18 PFLOP/s; 48 us for 12 pairs-of-words 768 x 768, 432 tiles of 128 on 256 CUs.
//
// X' = P X (X P where X is tall), times f and, in the first step, sigma; LAST: to the caller (T: its type; with parameters f32)
template <class S, int KIND, bool TALL, bool LAST, int T>
__global__ void __launch_bounds__(S::THREADS) k_ortho_apply(const uint16_t *poly, const uint16_t *x, OrthoDims d, Launch launch, uint32_t tiles_m, uint32_t tiles_n, float f,
                                                            const OrthoScale *scale, uint16_t *next, OrthoOut o)
{
    __shared__ __align__(16) char lds[S::LDS_BYTES];
    uint32_t mi, ni, batch;
    tile_place(launch, tiles_m, tiles_n, mi, ni, batch);
    const int64_t matrix = batch;
    const int64_t m0 = (int64_t)mi * S::BM, n0 = (int64_t)ni * S::BN;            // m: X's columns, n: its rows
    const int64_t ldx = row_words<KIND>(d.cols), ldp = row_words<KIND>(d.small);
    const Operand X{x + matrix * d.rows * ldx, ldx, TALL ? d.rows : d.cols}, P{poly + matrix * d.small * ldp, ldp, d.small};
    f32x16 acc[S::MI][S::NI];
    clear<S>(acc);
    if constexpr (TALL) tile_product<S, KIND, false, false>(acc, P, m0, X, n0, 0, d.small, lds);
    else tile_product<S, KIND, true, false>(acc, X, m0, P, n0, 0, d.small, lds);
    if (scale) f *= scale[matrix].sigma;
    const int64_t width = row_numbers<KIND>(d.cols);
    eights<S, false>(acc, lds, [&](int dn, int dm, const float (&raw)[8]) {
        const int64_t r = n0 + dn, col = m0 + dm;
        if (r >= d.rows || col >= (LAST ? d.cols : width)) return;
        if constexpr (LAST) {
            typedef typename TypeOf<T>::type E;
            E *out = (E *)o.out + matrix * o.out_mat + r * o.out_row;
            const float *px = o.x ? o.x + matrix * o.x_mat + r * d.cols : nullptr;
            E e8[8];
            float was[8];
            if constexpr (T == SAMS_F32)
                if (px) load_numbers(px, col, d.cols, was);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = raw[e] * f;
                if constexpr (T == SAMS_F32) e8[e] = px ? o.keep * was[e] - o.rate * v : v;
                else e8[e] = (E)v;
            }
            u32x4 w;
            __builtin_memcpy(&w, e8, 16);
            store_numbers(out, col, d.cols, w);
            if constexpr (T == SAMS_F32) {
                __builtin_memcpy(&w, e8 + 4, 16);
                store_numbers(out, col + 4, d.cols, w);
            }
        } else {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = col + e < d.cols ? raw[e] * f : 0.f;
            put8<KIND>(next + matrix * d.rows * ldx + r * ldx, col, v);
        }
    });
}

// ---- matrices that fit one workgroup's LDS: all steps in one launch ----
//
// X and one square matrix (A, then P in its place) stay in LDS as planes of 16-bit floats (the pairs' first parts, then the second
// ones), rows 16 bytes longer than whole fragments, so that rows next to each other start on other banks.  Sixteen wavefronts
// share out 32 x 32 tiles, hold their results until all have read what these replace, and write them over it.  50 matrices of 84 x 120,
// five steps: 45 us (the whole update 52, by launches of their own 80), a chain of reads from LDS, 3 x 8 dependent matrix instructions and a barrier for each of
// a step's three products; most CUs have nothing to do.
constexpr int kSmallWaves = 16, kSmallTiles = 3;                    // tiles a wavefront can hold
constexpr int kSmallLds = 163840 - 1024;

struct SmallLayout {
    int rows32, cols32, small32, pitch_x, pitch_s;                  // in numbers: padded extents, words from row to row
    int plane_x, plane_s;                                           // words of a plane
};
static inline __host__ __device__ SmallLayout small_layout(int64_t rows, int64_t cols)
{
    SmallLayout l;
    l.rows32 = (int)(rows + 31) / 32 * 32;
    l.cols32 = (int)(cols + 31) / 32 * 32;
    l.small32 = l.rows32 < l.cols32 ? l.rows32 : l.cols32;
    l.pitch_x = l.cols32 + 8;
    l.pitch_s = l.small32 + 8;
    l.plane_x = l.rows32 * l.pitch_x;
    l.plane_s = l.small32 * l.pitch_s;
    return l;
}
static bool small_fits(int64_t rows, int64_t cols)
{
    if (rows > 4096 || cols > 4096) return false;
    const SmallLayout l = small_layout(rows, cols);
    return (int64_t)(l.plane_x + l.plane_s) * 4 <= kSmallLds && l.rows32 / 32 * (l.cols32 / 32) <= kSmallWaves * kSmallTiles &&
           l.small32 / 32 * (l.small32 / 32) <= kSmallWaves * kSmallTiles;
}

// what the host knows of a step: the polynomial, and the powers of two between the words
struct SmallStep { float f_gram, a, b, c, f_apply; };
struct SmallSteps { int count; SmallStep step[SAMS_MAX_ORTHO_STEPS]; };

// a lane's 8 k's (from k0 + 8 * (lane / 32) on) of row r0 + lane % 32, or, where rows are k's, of column r0 + lane % 32
__device__ __forceinline__ u32x4 small_fragment(const uint16_t *m, int pitch, int r0, int k0, int lane) { return *(const u32x4 *)(m + (r0 + (lane & 31)) * pitch + k0 + 8 * (lane >> 5)); }
__device__ __forceinline__ u32x4 small_fragment_k(const uint16_t *m, int pitch, int r0, int k0, int lane)
{
    const int g = lane >> 4, q = lane & 15;
    typedef __attribute__((address_space(3))) short4v *lds_ptr;
    const uint16_t *at = m + (k0 + 8 * (g >> 1) + (q >> 2)) * pitch + r0 + (g & 1) * 16 + (q & 3) * 4;
    const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * pitch));
    const words2 a = __builtin_bit_cast(words2, lo), b = __builtin_bit_cast(words2, hi);
    return u32x4{a[0], a[1], b[0], b[1]};
}

// acc[t] = the product of tile (m, n) number wave + kSmallWaves t, n fastest, over k (a multiple of 32); A_K, B_K: rows are k's
template <bool A_K, bool B_K>
__device__ __forceinline__ void small_product(f32x16 (&acc)[kSmallTiles], const uint16_t *a, int pitch_a, int plane_a, const uint16_t *b, int pitch_b, int plane_b, int tiles,
                                              int tiles_n, int k, int lane, int wave)
{
#pragma unroll
    for (int t = 0; t < kSmallTiles; ++t) {
        const int id = wave + t * kSmallWaves;
        if (id >= tiles) break;
        asm volatile("" : "+v"(lane));                               // addresses made here, not kept for every tile over all steps
        const int m0 = id / tiles_n * 32, n0 = id % tiles_n * 32;
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[t][q] = 0.f;
        for (int k0 = 0; k0 < k; k0 += 32) {
            u32x4 fa[2][2], fb[2][2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int at = k0 + 16 * u;
                    fa[u][h] = A_K ? small_fragment_k(a + h * plane_a, pitch_a, m0, at, lane) : small_fragment(a + h * plane_a, pitch_a, m0, at, lane);
                    fb[u][h] = B_K ? small_fragment_k(b + h * plane_b, pitch_b, n0, at, lane) : small_fragment(b + h * plane_b, pitch_b, n0, at, lane);
                }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                acc[t] = mfma<F16>(fa[u][0], fb[u][0], acc[t]);
                acc[t] = mfma<F16>(fa[u][0], fb[u][1], acc[t]);
                acc[t] = mfma<F16>(fa[u][1], fb[u][0], acc[t]);
            }
        }
    }
}

// f(row, column, numbers) for the fours of a wavefront's tiles: n are rows, m columns
template <typename F>
__device__ __forceinline__ void small_fours(const f32x16 (&acc)[kSmallTiles], int tiles, int tiles_n, int lane, int wave, F f)
{
#pragma unroll
    for (int t = 0; t < kSmallTiles; ++t) {
        const int id = wave + t * kSmallWaves;
        if (id >= tiles) break;
        asm volatile("" : "+v"(lane));
        const int m0 = id / tiles_n * 32, n0 = id % tiles_n * 32;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float v[4] = {acc[t][4 * q], acc[t][4 * q + 1], acc[t][4 * q + 2], acc[t][4 * q + 3]};
            f(n0 + (lane & 31), m0 + 8 * q + 4 * (lane >> 5), v);
        }
    }
}

__device__ __forceinline__ void small_put(uint16_t *at, int plane, const float (&v)[4])
{
    const u32x4 w = pack_words<SPLIT>(v);
    *(words2 *)at = words2{w[0], w[1]};
    *(words2 *)(at + plane) = words2{w[2], w[3]};
}

__device__ __forceinline__ void small_get(const uint16_t *at, int plane, float (&v)[4])
{
    typedef _Float16 half4 __attribute__((ext_vector_type(4)));
    const half4 a = *(const half4 *)at, b = *(const half4 *)(at + plane);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)a[e] + (float)b[e];
}

// part: the sums of squares where they are made already (part_count of them a matrix), else null
template <int T, bool TALL>
__global__ void __launch_bounds__(64 * kSmallWaves) k_ortho_small(const typename TypeOf<T>::type *g, int64_t g_mat, int64_t g_row, int rows, int cols, float eps, const double *part,
                                                                  SmallSteps steps, OrthoOut o)
{
    typedef typename TypeOf<T>::type E;
    __shared__ __align__(16) uint16_t lds[kSmallLds / 2];
    __shared__ double sums[kSmallWaves];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int lane = tid & 63;
    const SmallLayout l = small_layout(rows, cols);
    uint16_t *x = lds, *sq = lds + l.plane_x * 2;
    const E *pg = g + blockIdx.x * g_mat;
    const int fours = l.cols32 / 4, small = rows < cols ? rows : cols;
    auto load4 = [&](int r, int c, float (&v)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = r < rows && c + e < cols ? (float)pg[r * g_row + c + e] : 0.f;
    };
    double s = 0;
    if (part) {
        for (int i = tid; i < kNormSlices; i += 64 * kSmallWaves) s += part[blockIdx.x * kNormSlices + i];
    } else {
        for (int i = tid; i < rows * fours; i += 64 * kSmallWaves) {
            float v[4];
            load4(i / fours, i % fours * 4, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_fma((double)v[e], (double)v[e], s);
        }
    }
    s = wave_sum(s);
    if (lane == 0) sums[wave] = s;
    __syncthreads();
    double norm = 0;
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) norm += sums[w];
    norm = sqrt(norm);
    const OrthoScale scale = ortho_scale(norm, eps);
    const double by = ldexp(1.0, scale.exponent);
    for (int i = tid; i < l.rows32 * fours; i += 64 * kSmallWaves) {
        const int r = i / fours, c = i % fours * 4;
        float v[4];
        load4(r, c, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)((double)v[e] * by);
        small_put(x + r * l.pitch_x + c, l.plane_x, v);
    }
    __syncthreads();
    f32x16 acc[kSmallTiles];
    const int ts = l.small32 / 32, square = ts * ts, tr = l.rows32 / 32, tiles = tr * (l.cols32 / 32), large32 = TALL ? l.rows32 : l.cols32;
    for (int step = 0; step < steps.count; ++step) {
        const SmallStep p = steps.step[step];
        const float fg = step ? p.f_gram : p.f_gram * scale.sigma2, fa = step ? p.f_apply : p.f_apply * scale.sigma;
        small_product<TALL, TALL>(acc, x, l.pitch_x, l.plane_x, x, l.pitch_x, l.plane_x, square, ts, large32, lane, wave);
        small_fours(acc, square, ts, lane, wave, [&](int r, int c, const float (&v)[4]) {
            const float w[4] = {v[0] * fg, v[1] * fg, v[2] * fg, v[3] * fg};
            small_put(sq + r * l.pitch_s + c, l.plane_s, w);
        });
        __syncthreads();
        small_product<false, false>(acc, sq, l.pitch_s, l.plane_s, sq, l.pitch_s, l.plane_s, square, ts, l.small32, lane, wave);
#pragma unroll
        for (int t = 0; t < kSmallTiles; ++t) {                      // P, still in registers: A is read by the others
            const int id = wave + t * kSmallWaves;
            if (id >= square) break;
            asm volatile("" : "+v"(lane));
            const int m0 = id / ts * 32, n0 = id % ts * 32;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = n0 + (lane & 31), c = m0 + 8 * q + 4 * (lane >> 5);
                float w[4];
                small_get(sq + r * l.pitch_s + c, l.plane_s, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t][4 * q + e] = r < small && c + e < small ? (r == c + e ? p.a : 0.f) + p.b * w[e] + p.c * acc[t][4 * q + e] : 0.f;
            }
        }
        __syncthreads();
        small_fours(acc, square, ts, lane, wave, [&](int r, int c, const float (&v)[4]) { small_put(sq + r * l.pitch_s + c, l.plane_s, v); });
        __syncthreads();
        if constexpr (TALL) small_product<false, false>(acc, sq, l.pitch_s, l.plane_s, x, l.pitch_x, l.plane_x, tiles, tr, l.small32, lane, wave);
        else small_product<true, false>(acc, x, l.pitch_x, l.plane_x, sq, l.pitch_s, l.plane_s, tiles, tr, l.small32, lane, wave);
        if (step + 1 < steps.count) {
            __syncthreads();
            small_fours(acc, tiles, tr, lane, wave, [&](int r, int c, const float (&v)[4]) {
                const float w[4] = {v[0] * fa, v[1] * fa, v[2] * fa, v[3] * fa};
                small_put(x + r * l.pitch_x + c, l.plane_x, w);
            });
            __syncthreads();
        } else {
            small_fours(acc, tiles, tr, lane, wave, [&](int r, int c, const float (&v)[4]) {
                if (r >= rows) return;
                E *out = (E *)o.out + blockIdx.x * o.out_mat + r * o.out_row;
                const float *px = o.x ? o.x + blockIdx.x * o.x_mat + (int64_t)r * cols : nullptr;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < cols) out[c + e] = (E)(px ? o.keep * px[c + e] - o.rate * (v[e] * fa) : v[e] * fa);
            });
        }
    }
}

// the largest of |a + b u + c u^2| * u^(odd ? 1/2 : 0) for 0 <= u <= u_max
static double poly_bound(double a, double b, double c, double u_max, bool odd)
{
    auto f = [&](double u) { return fabs(a + b * u + c * u * u) * (odd ? sqrt(u) : 1.0); };
    double best = fmax(f(0.0), f(u_max));
    auto at = [&](double u) { if (u > 0 && u < u_max) best = fmax(best, f(u)); };
    if (!odd) {
        if (c != 0) at(-b / (2 * c));
    } else if (c != 0) {                                             // d/ds (a s + b s^3 + c s^5) = a + 3 b u + 5 c u^2
        const double disc = 9 * b * b - 20 * a * c;
        if (disc >= 0) { at((-3 * b + sqrt(disc)) / (10 * c)); at((-3 * b - sqrt(disc)) / (10 * c)); }
    } else if (b != 0) {
        at(-a / (3 * b));
    }
    return best;
}

// power of two that takes a bound to about 2^14, a quarter of what a 16-bit float holds
static int word_exponent(double bound)
{
    if (!(bound > 0) || !isfinite(bound)) return 0;
    int e;
    (void)frexp(bound, &e);
    e = 14 - e;
    return e > 60 ? 60 : e < -60 ? -60 : e;
}

// the steps' factors, from bounds of X's singular values: words of X = X * 2^ex (the first: X = words * sigma), A's and P's likewise
static void plan_steps(int steps, const float *coef, SmallSteps *plan)
{
    const double a = coef[0], b = coef[1], c = coef[2];
    double bound = 1.0;
    int ex = 0;
    plan->count = steps;
    for (int s = 0; s < steps; ++s) {
        const double u = bound * bound, after = poly_bound(a, b, c, u, true);
        const int ea = word_exponent(u), ep = word_exponent(poly_bound(a, b, c, u, false)), en = s + 1 == steps ? 0 : word_exponent(after);
        plan->step[s] = SmallStep{(float)ldexp(1.0, ea - 2 * ex), (float)ldexp(a, ep), (float)ldexp(b, ep - ea), (float)ldexp(c, ep - 2 * ea), (float)ldexp(1.0, en - ep - ex)};
        ex = en;
        bound = after;
    }
}

// tiles of 64 x 64 on and under the diagonals
static int64_t gram_tiles(int64_t batch, int64_t small)
{
    const int64_t a = (small + Small::BM - 1) / Small::BM;
    return batch * (a * (a + 1) / 2);
}

// The parts that the k's of A's tiles are cut into (pairs): where a tile for every CU by parts, and a launch more to join them (6.5 us), is
// estimated to be the faster way.
static uint32_t gram_parts(int64_t batch, int64_t small, int64_t large, int shape)
{
    const int64_t tiles = gram_tiles(batch, small), parts = std::min<int64_t>(std::min<int64_t>(kGramParts, kGramTiles / tiles), large / 128);
    if (parts < 2) return 1;
    const int64_t size = kTileCosts[shape].size, a = (small + size - 1) / size;
    const double whole = tile_estimate(shape, true, (double)(batch * (a * (a + 1) / 2)), (double)large, 1), cut = tile_estimate(3, true, (double)tiles, (double)large, (int)parts) + 6500.0;
    return cut < whole ? (uint32_t)parts : 1;
}

template <int KIND, int T>
static int enqueue_steps(sams_ortho *c, int64_t batch, const SmallSteps &plan, const OrthoOut &o)
{
    const OrthoDims d{c->rows, c->cols, c->rows < c->cols ? c->rows : c->cols};
    const bool tall = c->rows > c->cols;
    uint16_t *gram = c->scratch.at<uint16_t>(c->gram), *poly = c->scratch.at<uint16_t>(c->poly);
    const OrthoScale *scale = c->scratch.at<OrthoScale>(c->scale);
    const int64_t large = d.rows + d.cols - d.small;
    const int of_gram = choose_tiles(KIND == SPLIT, batch, d.small, d.small, true, large, 1, 0).shape, of_poly = choose_tiles(KIND == SPLIT, batch, d.small, d.small, true, d.small, 1, 0).shape,
              of_apply = choose_tiles(KIND == SPLIT, batch, d.cols, d.rows, false, d.small, 1, 0).shape;
    const uint32_t parts = KIND == SPLIT ? gram_parts(batch, d.small, large, of_gram) : 1, tiles = (uint32_t)gram_tiles(batch, d.small);
    for (int s = 0; s < plan.count; ++s) {
        const uint16_t *x = c->scratch.at<uint16_t>(c->x[s & 1]);
        uint16_t *next = c->scratch.at<uint16_t>(c->x[(s + 1) & 1]);
        const SmallStep &p = plan.step[s];
        const OrthoScale *first = s == 0 ? scale : nullptr;
        auto square = [&](auto shape) {
            const int64_t ts = (d.small + decltype(shape)::BM - 1) / decltype(shape)::BM;
            return dim3((unsigned)(ts * (ts + 1) / 2 * batch));
        };
        if (parts > 1) {
            if constexpr (KIND == SPLIT) {                           // (a bfloat16 matrix of single words has tiles enough)
                float *sums = c->scratch.at<float>(c->sums);
                auto cut = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(tiles * parts), dim3(Small::THREADS), 0, c->stream, x, d, tiles, parts, sums); };
                if (tall) cut(k_ortho_gram_part<KIND, true>);
                else cut(k_ortho_gram_part<KIND, false>);
                hipLaunchKernelGGL((k_ortho_gram_join<KIND>), dim3(tiles, 4), dim3(256), 0, c->stream, sums, tiles, parts, d, p.f_gram, first, gram);
            }
        } else with_tile<KIND>(of_gram, [&](auto shape) {
            typedef decltype(shape) S;
            if (tall) hipLaunchKernelGGL((k_ortho_gram<S, KIND, true>), square(shape), dim3(S::THREADS), 0, c->stream, x, d, p.f_gram, first, gram);
            else hipLaunchKernelGGL((k_ortho_gram<S, KIND, false>), square(shape), dim3(S::THREADS), 0, c->stream, x, d, p.f_gram, first, gram);
        });
        with_tile<KIND>(of_poly, [&](auto shape) {
            typedef decltype(shape) S;
            hipLaunchKernelGGL((k_ortho_poly<S, KIND>), square(shape), dim3(S::THREADS), 0, c->stream, gram, d, p.a, p.b, p.c, poly);
        });
        const bool last = s + 1 == plan.count;
        with_tile<KIND>(of_apply, [&](auto shape) {
            typedef decltype(shape) S;
            const uint32_t tm = (uint32_t)((d.cols + S::BM - 1) / S::BM), tn = (uint32_t)((d.rows + S::BN - 1) / S::BN);
            auto apply = [&](auto kernel) {
                in_launches((int64_t)tm * tn * batch, S::THREADS, [&](dim3 grid, Launch l) {
                    hipLaunchKernelGGL(kernel, grid, dim3(S::THREADS), 0, c->stream, poly, x, d, l, tm, tn, p.f_apply, first, next, o);
                });
            };
            if (tall && last) apply(k_ortho_apply<S, KIND, true, true, T>);
            else if (tall) apply(k_ortho_apply<S, KIND, true, false, T>);
            else if (last) apply(k_ortho_apply<S, KIND, false, true, T>);
            else apply(k_ortho_apply<S, KIND, false, false, T>);
        });
        SAMS_HIP(hipGetLastError());
    }
    return SAMS_OK;
}

// from a matrix in memory to the last step; squares_made: the sums of its squares are in the scratch
template <int T>
static int enqueue_ortho(sams_ortho *c, int64_t batch, const void *g, int64_t g_mat, int64_t g_row, bool squares_made, int steps, const float *coef, float eps, const OrthoOut &o)
{
    typedef typename TypeOf<T>::type E;
    double *part = c->scratch.at<double>(c->part);
    SmallSteps plan;
    plan_steps(steps, coef, &plan);
    if (small_fits(c->rows, c->cols)) {
        auto all = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)batch), dim3(64 * kSmallWaves), 0, c->stream, (const E *)g, g_mat, g_row, (int)c->rows, (int)c->cols, eps,
                               squares_made ? part : nullptr, plan, o);
        };
        if (c->rows > c->cols) all(k_ortho_small<T, true>);
        else all(k_ortho_small<T, false>);
        SAMS_HIP(hipGetLastError());
        return SAMS_OK;
    }
    if (!squares_made)
        hipLaunchKernelGGL(k_ortho_squares<T>, dim3(kNormSlices, (unsigned)batch), dim3(256), 0, c->stream, (const E *)g, g_mat, g_row, c->rows, c->cols, part);
    auto large = [&](auto kind) {
        constexpr int KIND = decltype(kind)::value;
        hipLaunchKernelGGL((k_ortho_words<T, KIND>), dim3((unsigned)grid_for(c->rows, 4, 1024), (unsigned)batch), dim3(256), 0, c->stream, (const E *)g, g_mat, g_row, c->rows, c->cols,
                           eps, part, c->scratch.at<OrthoScale>(c->scale), c->scratch.at<uint16_t>(c->x[0]));
        SAMS_HIP(hipGetLastError());
        return enqueue_steps<KIND, T>(c, batch, plan, o);
    };
    if constexpr (T == SAMS_BF16)
        if (!ortho_pairs(T, c->rows, c->cols)) return large(std::integral_constant<int, F16>());
    return large(std::integral_constant<int, SPLIT>());
}

static bool coef_ok(const float *coef)
{
    return coef && isfinite(coef[0]) && isfinite(coef[1]) && isfinite(coef[2]);
}

}  // namespace sams

using namespace sams;

extern "C" {

int sams_ortho_create(sams_ortho **out, int64_t batch, int64_t rows, int64_t cols, int32_t type, void *hip_stream)
{
    if (!out) return SAMS_EINVAL;
    *out = nullptr;
    if (batch < 1 || batch > SAMS_MAX_BATCH || rows < 1 || rows > SAMS_MAX_DIM || cols < 1 || cols > SAMS_MAX_DIM || !type_ok(type)) return SAMS_EINVAL;
    sams_ortho *c = new (std::nothrow) sams_ortho();
    if (!c) return SAMS_ENOMEM;
    c->batch = batch; c->rows = rows; c->cols = cols; c->type = type;
    c->stream = (hipStream_t)hip_stream;
    const int64_t small = rows < cols ? rows : cols;
    const bool pairs = ortho_pairs(type, rows, cols);
    const int64_t ldx = pairs ? row_words<SPLIT>(cols) : row_words<F16>(cols), ldp = pairs ? row_words<SPLIT>(small) : row_words<F16>(small);
    for (int q = 0; q < 2; ++q) c->x[q] = c->scratch.reserve(batch * rows * ldx * 2);
    c->gram = c->scratch.reserve(batch * small * ldp * 2);
    c->poly = c->scratch.reserve(batch * small * ldp * 2);
    c->scale = c->scratch.reserve(batch * (int64_t)sizeof(OrthoScale));
    c->part = c->scratch.reserve(batch * kNormSlices * 8);
    c->sums = pairs && gram_tiles(1, small) < kGramTiles ? c->scratch.reserve((int64_t)kGramTiles * Small::BM * Small::BN * 4) : -1;
    c->update = type == SAMS_F32 ? c->scratch.reserve(batch * rows * cols * 4) : -1;
    const int rc = c->scratch.take();
    if (rc != SAMS_OK) { delete c; return rc; }
    *out = c;
    return SAMS_OK;
}

int sams_ortho_destroy(sams_ortho *c)
{
    if (!c) return SAMS_OK;
    hipError_t e = hipStreamSynchronize(c->stream);
    if (c->scratch.base) (void)hipFree(c->scratch.base);
    delete c;
    if (e != hipSuccess) { g_last_hip_error = (int)e; return SAMS_EHIP; }
    return SAMS_OK;
}

int64_t sams_ortho_scratch_bytes(const sams_ortho *c) { return c ? c->scratch.bytes : 0; }

int orthogonalize(sams_ortho *c, int64_t batch, const void *g, int64_t g_mat, int64_t g_row, int32_t steps, const float *coef_host, float eps,
                  void *out, int64_t out_mat, int64_t out_row)
{
    if (!c || batch < 0 || batch > c->batch || steps < 1 || steps > SAMS_MAX_ORTHO_STEPS || !coef_ok(coef_host) || !(eps >= 0.f)) return SAMS_EINVAL;
    if (batch == 0) return SAMS_OK;
    const int size = type_size(c->type);
    if (!g || !out || !aligned_to(g, size) || !aligned_to(out, size) || g_mat < 0 || g_row < 0 || (c->rows > 1 && out_row < c->cols) || (batch > 1 && out_mat < c->cols)) return SAMS_EINVAL;
    const OrthoOut o{out, out_mat, out_row, nullptr, 0, 0.f, 0.f};
    SAMS_BY_TYPE(c->type, T, return enqueue_ortho<T>(c, batch, g, g_mat, g_row, false, steps, coef_host, eps, o));
}

int muon_update(sams_ortho *c, int32_t n, int64_t batch, const float *g, int64_t g_worker, int64_t g_mat, const float *m, int64_t m_mat, const float *x,
                int64_t x_mat, float *m_out, int64_t m_out_mat, float *x_out, int64_t x_out_mat, float beta, int32_t nesterov, float lr, float scale,
                float weight_decay, int32_t steps, const float *coef_host, float eps)
{
    if (!c || c->type != SAMS_F32 || n < 1 || n > kMaxWorkers || batch < 0 || batch > c->batch || steps < 1 || steps > SAMS_MAX_ORTHO_STEPS ||
        !coef_ok(coef_host) || !(eps >= 0.f)) return SAMS_EINVAL;
    if (batch == 0) return SAMS_OK;
    if (!g || !m || !x || !m_out || !x_out || !aligned_to(g, 4) || !aligned_to(m, 4) || !aligned_to(x, 4) || !aligned_to(m_out, 4) || !aligned_to(x_out, 4)) return SAMS_EINVAL;
    const int64_t elems = c->rows * c->cols;
    if (g_worker < 0 || g_mat < 0 || m_mat < 0 || x_mat < 0 || (batch > 1 && (m_out_mat < elems || x_out_mat < elems))) return SAMS_EINVAL;
    float *update = c->scratch.at<float>(c->update);
    hipLaunchKernelGGL(k_muon_head, dim3(kNormSlices, (unsigned)batch), dim3(256), 0, c->stream, g, g_worker, g_mat, n, m, m_mat, m_out, m_out_mat, beta, nesterov, update, elems,
                       c->scratch.at<double>(c->part));
    SAMS_HIP(hipGetLastError());
    const OrthoOut o{x_out, x_out_mat, c->cols, x, x_mat, 1.f - lr * weight_decay, lr * scale};
    return enqueue_ortho<SAMS_F32>(c, batch, update, elems, c->cols, true, steps, coef_host, eps, o);
}

}  // extern "C"
