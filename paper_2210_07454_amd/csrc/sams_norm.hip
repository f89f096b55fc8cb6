// Layer norm over the last axis, forward and backward, for n workers' rows at once.
//
//   forward   mu = mean(x), s = 1 / sqrt(mean((x - mu)^2) + eps), y = (x - mu) s w + b
//   backward  with z = (x - mu) s and a = dy w:  dx = s (a - mean(a) - z mean(a z)),
//             dw = sum over a worker's rows of dy z, db = sum over them of dy
#include <new>

#include "sams_train.h"

struct sams_norm {
    int32_t n, type;
    int64_t t_max, dim;
    hipStream_t stream;
    sams::Scratch scratch;
    int64_t part;            // [n][kNormParts][2][dim] sums over parts of a worker's rows
};

namespace sams {

constexpr int kNormParts = 32;          // parts of a worker's rows that the sums of dw and db are made in

// A wavefront per row.  The variance is that of the differences from the mean, in a pass of its own: no cancellation.
template <int T>
__global__ void __launch_bounds__(256) k_norm_forward(const typename TypeOf<T>::type *x, Rows xs, const float *w, const float *b, float eps,
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
__global__ void __launch_bounds__(256) k_norm_backward(const typename TypeOf<T>::type *dy, Rows dys, const typename TypeOf<T>::type *x, Rows xs, const float *w,
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
    const int64_t lo = t * blockIdx.y / kNormParts, hi = t * (blockIdx.y + 1) / kNormParts;
    float sw = 0.f, sb = 0.f;
    for (int64_t r = lo; r < hi; ++r) {
        const float d = (float)dy[worker * dys.worker + r * dys.row + i];
        const float z = ((float)x[worker * xs.worker + r * xs.row + i] - mean[worker * t + r]) * rstd[worker * t + r];
        sw += d * z;
        sb += d;
    }
    float *o = part + ((worker * kNormParts + blockIdx.y) * 2) * dim + i;
    o[0] = sw;
    o[dim] = sb;
}

__global__ void __launch_bounds__(256) k_norm_join(const float *part, float *dw, int64_t dw_worker, float *db, int64_t db_worker, int accumulate, int64_t dim)
{
    const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x, worker = blockIdx.y;
    if (i >= dim) return;
    float sw = 0.f, sb = 0.f;
    for (int p = 0; p < kNormParts; ++p) {
        const float *o = part + ((worker * kNormParts + p) * 2) * dim + i;
        sw += o[0];
        sb += o[dim];
    }
    float *ow = dw + worker * dw_worker + i;
    *ow = accumulate ? *ow + sw : sw;
    if (db) {
        float *ob = db + worker * db_worker + i;
        *ob = accumulate ? *ob + sb : sb;
    }
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
    c->part = c->scratch.reserve((int64_t)n * kNormParts * 2 * dim * 4);
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
    SAMS_BY_TYPE(c->type, T, hipLaunchKernelGGL(k_norm_forward<T>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, c->stream,
        (const TypeOf<T>::type *)x, Rows{x_worker, x_row}, weight, bias, eps, (TypeOf<T>::type *)y, Rows{y_worker, y_row}, mean, rstd, t, rows, c->dim));
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
    const unsigned cols = (unsigned)((c->dim + 255) / 256);
    SAMS_BY_TYPE(c->type, T, {
        typedef TypeOf<T>::type E;
        hipLaunchKernelGGL(k_norm_columns<T>, dim3(cols, kNormParts, (unsigned)c->n), dim3(256), 0, c->stream, (const E *)dy, Rows{dy_worker, dy_row},
                           (const E *)x, Rows{x_worker, x_row}, mean, rstd, part, t, c->dim);
        if (rows)                                                    // last: dx may lie over x or dy
            hipLaunchKernelGGL(k_norm_backward<T>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, c->stream, (const E *)dy, Rows{dy_worker, dy_row},
                               (const E *)x, Rows{x_worker, x_row}, weight, mean, rstd, (E *)dx, Rows{dx_worker, dx_row}, t, rows, c->dim);
    });
    hipLaunchKernelGGL(k_norm_join, dim3(cols, (unsigned)c->n), dim3(256), 0, c->stream, part, dweight, dweight_worker, dbias, dbias_worker, accumulate, c->dim);
    SAMS_HIP(hipGetLastError());
    return SAMS_OK;
}

}  // extern "C"
