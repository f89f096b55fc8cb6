// Layer norm over the last axis, forward and backward, for n workers' rows at once.
//
//   forward   mu = mean(x), s = 1 / sqrt(mean((x - mu)^2) + eps), y = (x - mu) s w + b
//   backward  with z = (x - mu) s and a = dy w:  dx = s (a - mean(a) - z mean(a z)),
//             dw = sum over a worker's rows of dy z, db = sum over them of dy
#include <new>
#include <type_traits>

#include "sams_train.h"

struct sams_norm {
    int32_t n, type;
    int64_t t_max, dim;
    hipStream_t stream;
    sams::Scratch scratch;
    int64_t part;            // [n][parts][2][dim] sums over parts of a worker's rows
};

namespace sams {

constexpr int64_t kNormForwardThreads = 1024 * 256;      // of the forward pass: half of what the chip holds
constexpr int kNormBlocks = 512;        // workgroups of the backward pass that leave sums (all workers'): two for every CU

template <int TPR> constexpr int kNormBlock = TPR == 64 ? 256 : TPR;        // threads of a workgroup: a row's, or four rows' wavefronts
template <int TPR> constexpr int kNormBackBlock = TPR < 512 ? 512 : TPR;    // of the backward pass: several rows', whose sums are joined in LDS

template <int N>
__device__ __forceinline__ void load_floats(const float *p, int64_t at, int64_t dim, float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        uint32_t raw[4] = {0, 0, 0, 0};
        if (p && at + i < dim) load_piece<SAMS_F32>(p, at + i, dim, raw);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i + e] = __builtin_bit_cast(float, raw[e]);
    }
}

// Sum of a and b over the threads of a row: within the wavefront, and where a row has several, through LDS (two buffers that take
// turns, so that one barrier is enough).
template <int TPR>
__device__ __forceinline__ float2 row_sum(float a, float b, float2 (&buf)[2][16], int &turn)
{
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (TPR > 64) {
        const int wave = threadIdx.x >> 6, first = wave & ~(TPR / 64 - 1);
        if ((threadIdx.x & 63) == 0) buf[turn][wave] = make_float2(a, b);
        __syncthreads();
        a = b = 0.f;
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) { a += buf[turn][first + w].x; b += buf[turn][first + w].y; }
        turn ^= 1;
    }
    return make_float2(a, b);
}

// TPR threads per row, each with CH pieces of 16 bytes in registers: a row is read once, though mean and variance are sums of their own (no
// cancellation).  Workgroups go from row to row, with the weights in registers and the next row under way.  Bound by memory:
// 16,384 rows of 8,192 bf16 122 us, 4.4 TB/s (a copy: 4.7); 8,192 rows of 768 bf16 10.0 us, 2.5 TB/s, of which some 4 are the
// launch and a row's way; 4 rows of 512 2.6 us.
template <int T, int TPR, int CH>
__global__ void __launch_bounds__(kNormBlock<TPR>) k_norm_forward(const typename TypeOf<T>::type *x, Rows xs, const float *w, const float *b, float eps,
                                                                        typename TypeOf<T>::type *y, Rows ys, float *mean, float *rstd, uint32_t t, uint32_t rows, int64_t dim)
{
    constexpr int N = kPiece<T>, GROUPS = kNormBlock<TPR> / TPR;
    __shared__ float2 buf[2][16];
    int turn = 0;
    const int lane = threadIdx.x % TPR;
    float wv[CH][N], bv[CH][N];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        load_floats(w, (int64_t)(c * TPR + lane) * N, dim, wv[c]);
        load_floats(b, (int64_t)(c * TPR + lane) * N, dim, bv[c]);
    }
    const float over = 1.f / (float)dim;
    uint32_t row = blockIdx.x * GROUPS + threadIdx.x / TPR;
    const uint32_t stride = gridDim.x * GROUPS;
    uint32_t raw[CH][4];
    auto fetch = [&](uint32_t r) {
        const uint32_t worker = r / t;
        const typename TypeOf<T>::type *p = x + worker * xs.worker + (r - worker * t) * xs.row;
#pragma unroll
        for (int c = 0; c < CH; ++c) load_piece<T>(p, (int64_t)(c * TPR + lane) * N, dim, raw[c]);
    };
    if (row < rows) fetch(row);
    for (; row < rows; row += stride) {
        float v[CH][N];
#pragma unroll
        for (int c = 0; c < CH; ++c) widen<T>(raw[c], v[c]);
        const uint32_t worker = row / t;
        typename TypeOf<T>::type *o = y + worker * ys.worker + (row - worker * t) * ys.row;
        if (row + stride < rows) fetch(row + stride);
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < N; ++i) sum += v[c][i];
        const float mu = row_sum<TPR>(sum, 0.f, buf, turn).x * over;
        float sq = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[c][i] = (c * TPR + lane) * N + i < dim ? v[c][i] - mu : 0.f;
                sq = __builtin_fmaf(v[c][i], v[c][i], sq);
            }
        const float s = 1.f / sqrtf(row_sum<TPR>(sq, 0.f, buf, turn).x * over + eps);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t at = (int64_t)(c * TPR + lane) * N;
            if (at >= dim) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) v[c][i] = __builtin_fmaf(v[c][i] * s, wv[c][i], bv[c][i]);
            store_piece<T>(o, at, dim, v[c]);
        }
        if (lane == 0) { mean[row] = mu; rstd[row] = s; }
    }
}

// The same for the backward pass.  A workgroup has rows of one worker (part blockIdx.x of gridDim.x, worker blockIdx.y), and a thread
// its columns of all of them, so that dw and db are added up in registers beside dx; a workgroup's sums are left in `part`.  Every number
// is read once; the rows, the weights and the sums fill the registers, so that little else is under way while a row's sums meet.
// 16,384 rows of 8,192 bf16 222 us, 3.6 TB/s; 8,192 rows of 768 bf16 16.0 us, 2.4 TB/s, and 4 us to join their 512 parts.
template <int T, int TPR, int CH>
__global__ void __launch_bounds__(kNormBackBlock<TPR>, 4) k_norm_backward(const typename TypeOf<T>::type *dy, Rows dys, const typename TypeOf<T>::type *x, Rows xs, const float *w,
                                                                         const float *mean, const float *rstd, typename TypeOf<T>::type *dx, Rows dxs, float *part, uint32_t t,
                                                                         int64_t dim)
{
    constexpr int N = kPiece<T>, GROUPS = kNormBackBlock<TPR> / TPR;
    __shared__ float2 buf[2][16];
    extern __shared__ float joined[];                                // GROUPS > 1: [GROUPS / 2][2][dim]
    int turn = 0;
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const uint32_t worker = blockIdx.y;
    const uint32_t lo = (uint32_t)((uint64_t)t * blockIdx.x / gridDim.x), hi = (uint32_t)((uint64_t)t * (blockIdx.x + 1) / gridDim.x);
    float wv[CH][N], sw[CH][N], sb[CH][N];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        load_floats(w, (int64_t)(c * TPR + lane) * N, dim, wv[c]);
#pragma unroll
        for (int i = 0; i < N; ++i) sw[c][i] = sb[c][i] = 0.f;
    }
    const float over = 1.f / (float)dim;
    uint32_t rx[CH][4], rd[CH][4];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) rx[c][i] = rd[c][i] = 0;
    float mu = 0.f, s = 0.f;
    auto fetch = [&](uint32_t r) {
        const typename TypeOf<T>::type *px = x + worker * xs.worker + r * xs.row, *pd = dy + worker * dys.worker + r * dys.row;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            load_piece<T>(px, (int64_t)(c * TPR + lane) * N, dim, rx[c]);
            load_piece<T>(pd, (int64_t)(c * TPR + lane) * N, dim, rd[c]);
        }
        mu = mean[(int64_t)worker * t + r];
        s = rstd[(int64_t)worker * t + r];
    };
    if (lo + group < hi) fetch(lo + group);
    for (uint32_t first = lo; first < hi; first += GROUPS) {         // as often for every row's threads: they meet in row_sum
        const uint32_t r = first + group;
        float z[CH][N], d[CH][N];
        const float scale = s, shift = mu;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            widen<T>(rx[c], z[c]);
            widen<T>(rd[c], d[c]);
            if (GROUPS > 1 && r >= hi)
#pragma unroll
                for (int i = 0; i < N; ++i) z[c][i] = d[c][i] = 0.f;
        }
        if (r + GROUPS < hi) fetch(r + GROUPS);
        float sa = 0.f, saz = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < N; ++i) {                            // past the row's end d and w are 0
                z[c][i] = (z[c][i] - shift) * scale;
                sw[c][i] = __builtin_fmaf(d[c][i], z[c][i], sw[c][i]);
                sb[c][i] += d[c][i];
                d[c][i] *= wv[c][i];
                sa += d[c][i];
                saz = __builtin_fmaf(d[c][i], z[c][i], saz);
            }
        const float2 sums = row_sum<TPR>(sa, saz, buf, turn);
        if (GROUPS > 1 && r >= hi) continue;
        const float ma = sums.x * over, maz = sums.y * over;
        typename TypeOf<T>::type *o = dx + worker * dxs.worker + r * dxs.row;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t at = (int64_t)(c * TPR + lane) * N;
            if (at >= dim) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) d[c][i] = scale * (d[c][i] - ma - z[c][i] * maz);
            store_piece<T>(o, at, dim, d[c]);
        }
    }
#pragma unroll
    for (int half = GROUPS / 2; half; half /= 2) {                   // the upper half's sums are added to the lower half's
        if (group >= half && group < 2 * half)
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int64_t at = (int64_t)(c * TPR + lane) * N + i;
                    if (at < dim) {
                        joined[((group - half) * 2) * dim + at] = sw[c][i];
                        joined[((group - half) * 2 + 1) * dim + at] = sb[c][i];
                    }
                }
        __syncthreads();
        if (group < half)
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int64_t at = (int64_t)(c * TPR + lane) * N + i;
                    if (at < dim) {
                        sw[c][i] += joined[(group * 2) * dim + at];
                        sb[c][i] += joined[(group * 2 + 1) * dim + at];
                    }
                }
        __syncthreads();
    }
    if (group) return;
    float *o = part + ((int64_t)worker * gridDim.x + blockIdx.x) * 2 * dim;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t at = (int64_t)(c * TPR + lane) * N + i;
            if (at < dim) { o[at] = sw[c][i]; o[dim + at] = sb[c][i]; }
        }
}

// ---- rows too long for the registers of 1024 threads: read again for every pass over them ----

// A wavefront per row.  The variance is that of the differences from the mean, in a pass of its own: no cancellation.
template <int T>
__global__ void __launch_bounds__(256) k_norm_forward_long(const typename TypeOf<T>::type *x, Rows xs, const float *w, const float *b, float eps,
                                                           typename TypeOf<T>::type *y, Rows ys, float *mean, float *rstd, int64_t t, int64_t rows, int64_t dim)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = blockIdx.x * (int64_t)4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const int64_t worker = row / t, token = row - worker * t;
    const typename TypeOf<T>::type *px = x + worker * xs.worker + token * xs.row;
    float sum = 0.f;
    for (int64_t i = lane; i < dim; i += 64) sum += (float)px[i];
    const float mu = wave_sum(sum) / (float)dim;
    float sq = 0.f;
    for (int64_t i = lane; i < dim; i += 64) {
        const float c = (float)px[i] - mu;
        sq += c * c;
    }
    const float s = 1.f / sqrtf(wave_sum(sq) / (float)dim + eps);
    typename TypeOf<T>::type *py = y + worker * ys.worker + token * ys.row;
    for (int64_t i = lane; i < dim; i += 64) {
        float v = ((float)px[i] - mu) * s * w[i];
        if (b) v += b[i];
        py[i] = (typename TypeOf<T>::type)v;
    }
    if (lane == 0) { mean[row] = mu; rstd[row] = s; }
}

template <int T>
__global__ void __launch_bounds__(256) k_norm_backward_long(const typename TypeOf<T>::type *dy, Rows dys, const typename TypeOf<T>::type *x, Rows xs, const float *w,
                                                       const float *mean, const float *rstd, typename TypeOf<T>::type *dx, Rows dxs, int64_t t, int64_t rows, int64_t dim)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = blockIdx.x * (int64_t)4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const int64_t worker = row / t, token = row - worker * t;
    const typename TypeOf<T>::type *px = x + worker * xs.worker + token * xs.row;
    const typename TypeOf<T>::type *pd = dy + worker * dys.worker + token * dys.row;
    const float mu = mean[row], s = rstd[row];
    float sa = 0.f, saz = 0.f;
    for (int64_t i = lane; i < dim; i += 64) {
        const float a = (float)pd[i] * w[i], z = ((float)px[i] - mu) * s;
        sa += a;
        saz += a * z;
    }
    sa = wave_sum(sa) / (float)dim;
    saz = wave_sum(saz) / (float)dim;
    typename TypeOf<T>::type *po = dx + worker * dxs.worker + token * dxs.row;
    for (int64_t i = lane; i < dim; i += 64) {
        const float a = (float)pd[i] * w[i], z = ((float)px[i] - mu) * s;
        po[i] = (typename TypeOf<T>::type)(s * (a - sa - z * saz));
    }
}

// Sums over one part of a worker's rows; a thread per column.
template <int T>
__global__ void __launch_bounds__(256) k_norm_columns(const typename TypeOf<T>::type *dy, Rows dys, const typename TypeOf<T>::type *x, Rows xs, const float *mean,
                                                      const float *rstd, float *part, int64_t t, int64_t dim)
{
    const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x, worker = blockIdx.z;
    if (i >= dim) return;
    const int64_t lo = t * blockIdx.y / gridDim.y, hi = t * (blockIdx.y + 1) / gridDim.y;
    float sw = 0.f, sb = 0.f;
    for (int64_t r = lo; r < hi; ++r) {
        const float d = (float)dy[worker * dys.worker + r * dys.row + i];
        const float z = ((float)x[worker * xs.worker + r * xs.row + i] - mean[worker * t + r]) * rstd[worker * t + r];
        sw += d * z;
        sb += d;
    }
    float *o = part + ((worker * gridDim.y + blockIdx.y) * 2) * dim + i;
    o[0] = sw;
    o[dim] = sb;
}

// Adds up the parts of every column: four threads a column, each a quarter of the parts in ascending order.
__global__ void __launch_bounds__(256) k_norm_join(const float *part, int parts, float *dw, int64_t dw_worker, float *db, int64_t db_worker, int accumulate, int64_t dim)
{
    __shared__ float sums[4][2][64];
    const int q = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t i = blockIdx.x * (int64_t)64 + lane, worker = blockIdx.y;
    float sw = 0.f, sb = 0.f;
    if (i < dim) {
        const int lo = parts * q / 4, hi = parts * (q + 1) / 4;
        const float *o = part + (worker * parts + lo) * 2 * dim + i;
#pragma unroll 8
        for (int p = lo; p < hi; ++p, o += 2 * dim) {
            sw += o[0];
            sb += o[dim];
        }
    }
    sums[q][0][lane] = sw;
    sums[q][1][lane] = sb;
    __syncthreads();
    if (q || i >= dim) return;
    sw = (sums[0][0][lane] + sums[1][0][lane]) + (sums[2][0][lane] + sums[3][0][lane]);
    sb = (sums[0][1][lane] + sums[1][1][lane]) + (sums[2][1][lane] + sums[3][1][lane]);
    float *ow = dw + worker * dw_worker + i;
    *ow = accumulate ? *ow + sw : sw;
    if (db) {
        float *ob = db + worker * db_worker + i;
        *ob = accumulate ? *ob + sb : sb;
    }
}

// How many threads a row gets, and how many pieces each holds: the fewest threads that hold it in MOST pieces each (a wavefront alone
// needs no barrier).  The backward pass takes about 40 registers a piece of 4 numbers and 75 a piece of 8, the forward pass half of
// that.  false: the row is too long.
template <int T, int MOST, typename F>
static bool by_row(int64_t dim, F f)
{
    const int64_t pieces = (dim + kPiece<T> - 1) / kPiece<T>;
#define SAMS_ROW(TPR, CH) \
    if constexpr (CH <= MOST) \
        if (pieces <= TPR * CH) { f(std::integral_constant<int, TPR>(), std::integral_constant<int, CH>()); return true; }
    SAMS_ROW(64, 1) SAMS_ROW(64, 2) SAMS_ROW(128, 1) SAMS_ROW(128, 2) SAMS_ROW(256, 1) SAMS_ROW(256, 2) SAMS_ROW(512, 1) SAMS_ROW(512, 2) SAMS_ROW(1024, 1) SAMS_ROW(1024, 2)
#undef SAMS_ROW
    return false;
}

// parts that the rows of a worker are split into, in the backward pass
static int norm_parts(int32_t n, int64_t t, bool wide)
{
    const int64_t blocks = wide ? kNormBlocks / 2 : kNormBlocks, most = n < blocks ? blocks / n : 1, some = (t + 3) / 4;        // no workgroup left for a second round
    return (int)(some < 1 ? 1 : some < most ? some : most);
}

}  // namespace sams

using namespace sams;

extern "C" {

int sams_norm_create(sams_norm **out, int32_t n, int64_t t_max, int64_t dim, int32_t type, void *hip_stream)
{
    if (!out) return SAMS_EINVAL;
    *out = nullptr;
    if (n < 1 || n > kMaxWorkers || t_max < 0 || t_max > SAMS_MAX_TOKENS / n || dim < 1 || dim > SAMS_MAX_DIM || !type_ok(type)) return SAMS_EINVAL;
    sams_norm *c = new (std::nothrow) sams_norm();
    if (!c) return SAMS_ENOMEM;
    c->n = n; c->t_max = t_max; c->dim = dim; c->type = type;
    c->stream = (hipStream_t)hip_stream;
    c->part = c->scratch.reserve((int64_t)n * norm_parts(n, t_max, false) * 2 * dim * 4);
    const int rc = c->scratch.take();
    if (rc != SAMS_OK) { delete c; return rc; }
    *out = c;
    return SAMS_OK;
}

int sams_norm_destroy(sams_norm *c)
{
    if (!c) return SAMS_OK;
    hipError_t e = hipStreamSynchronize(c->stream);
    if (c->scratch.base) (void)hipFree(c->scratch.base);
    delete c;
    if (e != hipSuccess) { g_last_hip_error = (int)e; return SAMS_EHIP; }
    return SAMS_OK;
}

int64_t sams_norm_scratch_bytes(const sams_norm *c) { return c ? c->scratch.bytes : 0; }

int layer_norm_forward(sams_norm *c, int64_t t, const void *x, int64_t x_worker, int64_t x_row, const float *weight, const float *bias,
                       float eps, void *y, int64_t y_worker, int64_t y_row, float *mean, float *rstd)
{
    if (!c || t < 0 || t > c->t_max || !(eps >= 0.f) || !weight || !aligned_to(weight, 4) || !aligned_to(bias, 4)) return SAMS_EINVAL;
    if (t == 0) return SAMS_OK;
    const int size = type_size(c->type);
    if (!x || !y || !mean || !rstd || !aligned_to(x, size) || !aligned_to(y, size) || !aligned_to(mean, 4) || !aligned_to(rstd, 4)) return SAMS_EINVAL;
    if (x_row < 0 || x_worker < 0 || (t > 1 && y_row < c->dim) || (c->n > 1 && y_worker < c->dim)) return SAMS_EINVAL;
    const int64_t rows = c->n * t;
    SAMS_BY_TYPE(c->type, T, {
        typedef TypeOf<T>::type E;
        if (!by_row<T, 2>(c->dim, [&](auto tpr, auto ch) {
                constexpr int TPR = decltype(tpr)::value, CH = decltype(ch)::value, BLOCK = kNormBlock<TPR>, GROUPS = BLOCK / TPR;
                hipLaunchKernelGGL((k_norm_forward<T, TPR, CH>), dim3((unsigned)grid_for(rows, GROUPS, kNormForwardThreads / BLOCK)), dim3(BLOCK), 0,
                                   c->stream, (const E *)x, Rows{x_worker, x_row}, weight, bias, eps, (E *)y, Rows{y_worker, y_row}, mean, rstd, (uint32_t)t, (uint32_t)rows, c->dim);
            }))
            hipLaunchKernelGGL(k_norm_forward_long<T>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, c->stream, (const E *)x, Rows{x_worker, x_row}, weight, bias, eps, (E *)y,
                               Rows{y_worker, y_row}, mean, rstd, t, rows, c->dim);
    });
    SAMS_HIP(hipGetLastError());
    return SAMS_OK;
}

int layer_norm_backward(sams_norm *c, int64_t t, const void *dy, int64_t dy_worker, int64_t dy_row, const void *x, int64_t x_worker,
                        int64_t x_row, const float *weight, const float *mean, const float *rstd, void *dx, int64_t dx_worker,
                        int64_t dx_row, float *dweight, int64_t dweight_worker, float *dbias, int64_t dbias_worker, int32_t accumulate)
{
    if (!c || t < 0 || t > c->t_max || !weight || !dweight || !aligned_to(weight, 4) || !aligned_to(dweight, 4) || !aligned_to(dbias, 4)) return SAMS_EINVAL;
    if (c->n > 1 && (dweight_worker < c->dim || (dbias && dbias_worker < c->dim))) return SAMS_EINVAL;
    const int size = type_size(c->type);
    if (t > 0) {
        if (!dy || !x || !mean || !rstd || !dx || !aligned_to(dy, size) || !aligned_to(x, size) || !aligned_to(dx, size) ||
            !aligned_to(mean, 4) || !aligned_to(rstd, 4)) return SAMS_EINVAL;
        if (dy_row < 0 || dy_worker < 0 || x_row < 0 || x_worker < 0 || (t > 1 && dx_row < c->dim) || (c->n > 1 && dx_worker < c->dim)) return SAMS_EINVAL;
    }
    const int64_t rows = c->n * t;
    float *part = c->scratch.at<float>(c->part);
    int parts = norm_parts(c->n, t, false);
    SAMS_BY_TYPE(c->type, T, {
        typedef TypeOf<T>::type E;
        if (!by_row<T, T == SAMS_F32 ? 2 : 1>(c->dim, [&](auto tpr, auto ch) {
                constexpr int TPR = decltype(tpr)::value, CH = decltype(ch)::value, BLOCK = kNormBackBlock<TPR>, GROUPS = BLOCK / TPR;
                parts = norm_parts(c->n, t, BLOCK > 512);
                hipLaunchKernelGGL((k_norm_backward<T, TPR, CH>), dim3((unsigned)parts, (unsigned)c->n), dim3(BLOCK), (unsigned)(GROUPS / 2 * 2 * c->dim * 4), c->stream,
                                   (const E *)dy, Rows{dy_worker, dy_row}, (const E *)x, Rows{x_worker, x_row}, weight, mean, rstd, (E *)dx, Rows{dx_worker, dx_row}, part, (uint32_t)t,
                                   c->dim);
            })) {
            hipLaunchKernelGGL(k_norm_columns<T>, dim3((unsigned)((c->dim + 255) / 256), (unsigned)parts, (unsigned)c->n), dim3(256), 0, c->stream, (const E *)dy, Rows{dy_worker, dy_row},
                               (const E *)x, Rows{x_worker, x_row}, mean, rstd, part, t, c->dim);
            if (rows)                                                // last: dx may lie over x or dy
                hipLaunchKernelGGL(k_norm_backward_long<T>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, c->stream, (const E *)dy, Rows{dy_worker, dy_row}, (const E *)x,
                                   Rows{x_worker, x_row}, weight, mean, rstd, (E *)dx, Rows{dx_worker, dx_row}, t, rows, c->dim);
        }
    });
    hipLaunchKernelGGL(k_norm_join, dim3((unsigned)((c->dim + 63) / 64), (unsigned)c->n), dim3(256), 0, c->stream, part, parts, dweight, dweight_worker, dbias, dbias_worker, accumulate, c->dim);
    SAMS_HIP(hipGetLastError());
    return SAMS_OK;
}

}  // extern "C"
