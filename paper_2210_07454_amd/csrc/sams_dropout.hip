// Dropout of hidden states, with the residual stream added where there is one:
//
//   forward   y = r + m x / (1 - p)        backward   dx = m dy / (1 - p)   (dr = dy)
//
// m is made again from the generator in either pass.
#include <new>

#include "sams_gemm.h"
#include "sams_random.h"

struct sams_dropout {
    int32_t n, type;
    int64_t t_max, dim;
    hipStream_t stream;
};

namespace sams {

constexpr int kDropBlock = 256;

// A workgroup has kDropBlock pieces of 8 columns that follow each other, row after row, a thread one: one call of the generator, whose instructions take
// a third of the time that its memory does.  Bound by memory: 16,384 rows of 8,192 bf16 with a residual 160 us, 5.0 TB/s, without 88 us, 6.1 (a
// copy: 4.7); 8,192 rows of 768 8.9 and 7.2 us.  (Two pieces a thread, both loads under way at once: 4,593 rows of 1,283 in 32 bits
// 12.8 us instead of 11.6; four: wide rows 133 us instead of 124.)
template <int T>
__global__ void __launch_bounds__(kDropBlock) k_dropout(const typename TypeOf<T>::type *x, Rows xs, const typename TypeOf<T>::type *r, Rows rs, const int64_t *rng, Keep keep,
                                                       typename TypeOf<T>::type *y, Rows ys, uint32_t t, uint32_t rows, int64_t dim, uint32_t pieces, uint32_t first)
{
    const uint32_t id = first + blockIdx.x, in = id % pieces * kDropBlock;      // below 2^22
    const uint32_t off = in % pieces + threadIdx.x, down = off / pieces, piece = off - down * pieces;
    const uint32_t row = id / pieces * kDropBlock + in / pieces + down;
    if (row >= rows) return;
    const uint32_t worker = row / t, at = row - worker * t;
    const int64_t column = (int64_t)piece * 8;
    float v[8], res[8];
    load8<T>(x + worker * xs.worker + at * xs.row, column, dim, v);
    if (r) load8<T>(r + worker * rs.worker + at * rs.row, column, dim, res);
    if (keep.least) {
        uint32_t numbers[4];
        philox(read_seed(rng), piece, at, worker, numbers);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = kept(numbers, e, keep.least) ? v[e] * keep.scale : 0.f;
    }
    if (r) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += res[e];
    }
    typename TypeOf<T>::type *to = y + worker * ys.worker + at * ys.row;
#pragma unroll
    for (int e = 0; e < 8; e += kPiece<T>) {
        float part[kPiece<T>];
#pragma unroll
        for (int i = 0; i < kPiece<T>; ++i) part[i] = v[e + i];
        if (column + e < dim) store_piece<T>(to, column + e, dim, part);
    }
}

static int dropout(sams_dropout *c, int64_t t, const void *x, Rows xs, const void *r, Rows rs, const int64_t *rng, double p, void *y, Rows ys)
{
    Keep keep;
    if (!c || t < 0 || t > c->t_max || !keep_of(p, keep)) return SAMS_EINVAL;
    if (t == 0) return SAMS_OK;
    const int size = type_size(c->type);
    if (!x || !y || !aligned_to(x, size) || !aligned_to(r, size) || !aligned_to(y, size) || (keep.least && !rng) || !aligned_to(rng, 8)) return SAMS_EINVAL;
    if (xs.row < 0 || xs.worker < 0 || (r && (rs.row < 0 || rs.worker < 0)) || (t > 1 && ys.row < c->dim) || (c->n > 1 && ys.worker < c->dim)) return SAMS_EINVAL;
    const int64_t rows = c->n * t, pieces = (c->dim + 7) / 8, blocks = (rows * pieces + kDropBlock - 1) / kDropBlock;
    SAMS_BY_TYPE(c->type, T, {
        typedef TypeOf<T>::type E;
        gemm::in_launches(blocks, kDropBlock, [&](dim3 grid, gemm::Launch l) {
            hipLaunchKernelGGL(k_dropout<T>, grid, dim3(kDropBlock), 0, c->stream, (const E *)x, xs, (const E *)r, rs, rng, keep, (E *)y, ys, (uint32_t)t, (uint32_t)rows, c->dim,
                               (uint32_t)pieces, l.first);
        });
    });
    SAMS_HIP(hipGetLastError());
    return SAMS_OK;
}

}  // namespace sams

using namespace sams;

extern "C" {

int sams_dropout_create(sams_dropout **out, int32_t n, int64_t t_max, int64_t dim, int32_t type, void *hip_stream)
{
    if (!out) return SAMS_EINVAL;
    *out = nullptr;
    if (n < 1 || n > kMaxWorkers || t_max < 0 || t_max > SAMS_MAX_TOKENS / n || dim < 1 || dim > SAMS_MAX_DIM || !type_ok(type)) return SAMS_EINVAL;
    sams_dropout *c = new (std::nothrow) sams_dropout();
    if (!c) return SAMS_ENOMEM;
    c->n = n; c->t_max = t_max; c->dim = dim; c->type = type;
    c->stream = (hipStream_t)hip_stream;
    *out = c;
    return SAMS_OK;
}

int sams_dropout_destroy(sams_dropout *c)
{
    delete c;
    return SAMS_OK;
}

int64_t sams_dropout_scratch_bytes(const sams_dropout *) { return 0; }

int dropout_forward(sams_dropout *c, int64_t t, const void *x, int64_t x_worker, int64_t x_row, const void *residual, int64_t residual_worker,
                    int64_t residual_row, const int64_t *rng, double p, void *y, int64_t y_worker, int64_t y_row)
{
    return dropout(c, t, x, Rows{x_worker, x_row}, residual, Rows{residual_worker, residual_row}, rng, p, y, Rows{y_worker, y_row});
}

int dropout_backward(sams_dropout *c, int64_t t, const void *dy, int64_t dy_worker, int64_t dy_row, const int64_t *rng, double p, void *dx,
                     int64_t dx_worker, int64_t dx_row)
{
    return dropout(c, t, dy, Rows{dy_worker, dy_row}, nullptr, Rows{}, rng, p, dx, Rows{dx_worker, dx_row});
}

}  // extern "C"
