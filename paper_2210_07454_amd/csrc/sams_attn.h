// What the passes of the attention with a bias by relative position have in common: their arguments, the tiles' way through LDS to the
// matrix cores, and what a distance between two tokens means.
#pragma once
#include "sams_gemm.h"
#include "sams_random.h"

namespace sams {
namespace attn {

using gemm::f32x16;
using gemm::u32x4;

constexpr int kThreads = 256, kWaves = 4, kRows = 128;      // a workgroup's rows: 32 for each wavefront, which keeps them in registers
constexpr float kLog2e = 1.44269504088896340736f;

struct Args {
    const void *q, *k, *v, *o, *dout;
    Rows qs, ks, vs, os, douts;
    void *out, *dq, *dk, *dv;
    Rows outs, dqs, dks, dvs;
    const float *bias;              // [heads][buckets], or none
    const int32_t *starts;          // [buckets]
    const int32_t *lengths;         // [n][seqs], or none
    const int64_t *rng;
    float *row_max, *row_sum;       // [n][heads][t]: a row's largest logit (times log2 e) and its sum of exponentials
    float *delta;                   // [n][heads][t]: sums of dP P
    float *part;                    // [n][heads][seqs * tiles][buckets]: the bias's gradient
    int64_t t;
    uint32_t n, seqs, len, heads, kv_heads, dim, buckets, tiles;
    uint32_t seq_first, seq_count;  // sequences that a launch deals with, of every worker
    float scale, scale2;            // the logits' factor, and the same times log2 e
    Keep keep;
    int32_t causal;
};

// ---- fragments: eight numbers of a row a lane, as one matrix instruction of 16-bit words takes them, or eight of 32-bit numbers ----
template <int T> struct Fragment { typedef u32x4 type; };
template <> struct Fragment<SAMS_F32> { typedef float type __attribute__((ext_vector_type(8))); };

// c += a' b over 16 k's.  A lane brings the k's 8 (lane / 32) .. + 7 of column lane % 32 of either; 32-bit numbers go in pairs of k and
// k + 8, so that their fragments hold the same k's.  c: column lane % 32, rows 8 (i / 4) + 4 (lane / 32) + i % 4.
template <int T>
__device__ __forceinline__ f32x16 product(const typename Fragment<T>::type &a, const typename Fragment<T>::type &b, f32x16 c)
{
    if constexpr (T == SAMS_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
        return c;
    } else {
        return gemm::mfma<T == SAMS_BF16 ? gemm::BF16 : gemm::F16>(a, b, c);
    }
}

// numbers 8 half .. + 7 of an accumulator as a fragment: the k's 16 half + 4 (lane / 32) + {0 .. 3, 8 .. 11} of its rows
template <int T>
__device__ __forceinline__ typename Fragment<T>::type words_of(const f32x16 &v, int half)
{
    typename Fragment<T>::type f;
    if constexpr (T == SAMS_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = v[8 * half + i];
    } else {
        typedef typename TypeOf<T>::type E;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = gemm::pair_of<E>(v[8 * half + 2 * i], v[8 * half + 2 * i + 1]);
    }
    return f;
}

// ---- tiles in LDS: rows of D numbers, and some bytes that put the rows on different banks ----
template <int T, int D> struct Tile {
    typedef typename TypeOf<T>::type E;
    typedef typename Fragment<T>::type Frag;
    static constexpr int ROWS = T == SAMS_F32 ? 32 : 64;                        // that a workgroup takes at a time
    static constexpr int LD = D * (int)sizeof(E) + (T != SAMS_F32 && D == 128 ? 80 : 16);     // bytes from row to row
    static constexpr int BYTES = ROWS * LD;
    static constexpr int PIECES = D * (int)sizeof(E) / 16, N = ROWS * PIECES / kThreads;      // of 16 bytes: a row's, a thread's
    static_assert(ROWS * PIECES % kThreads == 0, "every thread brings as many");

    // numbers 16 s + 8 (lane / 32) .. + 7 of row row0 + lane % 32
    __device__ __forceinline__ static Frag along(const char *tile, int row0, int s, int lane)
    {
        const char *at = tile + (row0 + (lane & 31)) * LD + (16 * s + 8 * (lane >> 5)) * (int)sizeof(E);
        if constexpr (T == SAMS_F32) {
            typedef float f4 __attribute__((ext_vector_type(4)));
            const f4 a = *(const f4 *)at, b = *(const f4 *)(at + 16);
            return Frag{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        } else {
            return *(const u32x4 *)at;
        }
    }
    // column col0 + lane % 32 of the rows row0 + 4 (lane / 32) + {0 .. 3, 8 .. 11}.  16-bit words through the transposing load: of every
    // 16 lanes four give the address of one row's 16 columns, and each gets one column's four rows.
    __device__ __forceinline__ static Frag across(const char *tile, int row0, int col0, int lane)
    {
        if constexpr (T == SAMS_F32) {
            Frag f;
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = *(const float *)(tile + (row0 + 4 * (lane >> 5) + (i & 3) + 8 * (i >> 2)) * LD + (col0 + (lane & 31)) * 4);
            return f;
        } else {
            const int g = lane >> 4, q = lane & 15;
            const char *at = tile + (row0 + 4 * (g >> 1) + (q >> 2)) * LD + (col0 + (g & 1) * 16 + (q & 3) * 4) * 2;
            typedef __attribute__((address_space(3))) gemm::short4v *lds_ptr;
            const gemm::words2 a = __builtin_bit_cast(gemm::words2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at)));
            const gemm::words2 b = __builtin_bit_cast(gemm::words2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 8 * LD)));
            return Frag{a[0], a[1], b[0], b[1]};
        }
    }
};

// A tile on its way to LDS: rows from `first` on, those from `limit` on and columns from dim on as zeros.
template <int T, int D>
struct Bring {
    typedef Tile<T, D> Ti;
    typedef typename TypeOf<T>::type E;
    uint32_t raw[Ti::N][4];

    __device__ __forceinline__ void load(const E *p, int64_t row, uint32_t first, uint32_t limit, uint32_t dim)
    {
        p += (int64_t)first * row;
#pragma unroll
        for (int i = 0; i < Ti::N; ++i) {
            const uint32_t r = (i * kThreads + threadIdx.x) / Ti::PIECES, at = (i * kThreads + threadIdx.x) % Ti::PIECES * kPiece<T>;
#pragma unroll
            for (int e = 0; e < 4; ++e) raw[i][e] = 0;
            if (first + r < limit && at < dim) load_piece<T>(p + r * row, at, dim, raw[i]);
        }
    }
    __device__ __forceinline__ void store(char *tile) const
    {
#pragma unroll
        for (int i = 0; i < Ti::N; ++i) {
            const int r = (i * kThreads + threadIdx.x) / Ti::PIECES, c = (i * kThreads + threadIdx.x) % Ti::PIECES;
            *(u32x4 *)(tile + r * Ti::LD + c * 16) = u32x4{raw[i][0], raw[i][1], raw[i][2], raw[i][3]};
        }
    }
};

// a lane's fragments of a row that stays in registers: all zeros where it does not exist
template <int T, int D>
__device__ __forceinline__ void row_fragments(const typename TypeOf<T>::type *p, bool there, uint32_t dim, int lane, typename Fragment<T>::type (&f)[D / 16])
{
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
        const uint32_t at = 16 * s + 8 * (lane >> 5);
#pragma unroll
        for (int h = 0; h < 8; h += kPiece<T>) {
            uint32_t raw[4] = {0, 0, 0, 0};
            if (there && at + h < dim) load_piece<T>(p, at + h, dim, raw);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (T == SAMS_F32) f[s][h + e] = __builtin_bit_cast(float, raw[e]);
                else f[s][e] = raw[e];
            }
        }
    }
}

// what the other half of the wavefront has for the same column
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// ---- a wavefront's 32 columns of D numbers, of which a lane has four next to each other at a time, stored as rows ----
template <int T, int D>
__device__ __forceinline__ void store_columns(typename TypeOf<T>::type *row, bool there, uint32_t dim, const f32x16 (&acc)[D / 32], float scale, int lane)
{
    typedef typename TypeOf<T>::type E;
    if (!there) return;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const uint32_t at = 32 * d + 8 * a + 4 * (lane >> 5);
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = acc[d][4 * a + i] * scale;
            if (at + 4 <= dim) {
                const auto w = gemm::pack_numbers<E>(v);
                typedef uint32_t anywhere __attribute__((ext_vector_type(sizeof(E)), aligned(2)));
                *(anywhere *)(row + at) = __builtin_bit_cast(anywhere, w);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (at + i < dim) row[at + i] = (E)v[i];
            }
        }
}

// ---- the bias ----
// Bucket b is the distances (key minus query) from starts[b] on to starts[b + 1] - 1; what lies before starts[1] is bucket 0.  A workgroup
// has the starts in LDS; a tile whose distances all lie in one bucket adds one number, any other one looks its numbers up by distance in a
// window that the workgroup has filled for it.
__device__ __forceinline__ float bias_of(float v)
{
    // numbers stay numbers, however large: rows of nothing but the type's lowest value have equal weights
    return __builtin_isfinite(v) ? fminf(fmaxf(v * kLog2e, -1.7e38f), 1.7e38f) : v;
}

struct Starts {
    const int *at;          // [buckets] in LDS
    uint32_t buckets;

    // of a tile's distances from lo to hi: the bucket of lo, and whether it is that of hi too.  Every wavefront finds out for itself.
    __device__ __forceinline__ bool one_bucket(int lo, int hi, uint32_t &bucket) const
    {
        uint32_t below = 0, above = 0;
        for (uint32_t b = 0; b < buckets; b += 64) {
            const uint32_t i = b + (threadIdx.x & 63);
            const bool there = i > 0 && i < buckets;
            const int start = there ? at[i] : 0;
            below += __builtin_popcountll(__ballot(there && start <= lo));
            above += __builtin_popcountll(__ballot(there && start <= hi));
        }
        bucket = below;
        return below == above;
    }
    __device__ __forceinline__ uint32_t of(int distance) const
    {
        uint32_t lo = 0, n = buckets;               // the answer is one of lo .. lo + n - 1
        while (n > 1) {
            const uint32_t half = n >> 1;
            const bool up = at[lo + half] <= distance;
            lo = up ? lo + half : lo;
            n = up ? n - half : half;
        }
        return lo;
    }
};

// What a tile of `cols` streamed rows against a workgroup's kRows needs to know of its distances, in LDS, two of them in turn.
struct Window {
    float value[64 + kRows];
    uint16_t bucket[64 + kRows];
};
// the same in registers: one bucket, or the window
struct Band {
    bool one;
    uint32_t bucket;
    float value;
};
__device__ __forceinline__ Band band_of(const Starts &starts, const float *bias, int lo, int count, Window &w)
{
    Band b = {true, 0, 0.f};
    if (starts.buckets == 0) return b;
    b.one = starts.one_bucket(lo, lo + count - 1, b.bucket);
    if (b.one) {
        b.value = bias_of(bias[b.bucket]);
    } else if ((int)threadIdx.x < count) {
        const uint32_t k = starts.of(lo + (int)threadIdx.x);
        w.value[threadIdx.x] = bias_of(bias[k]);
        w.bucket[threadIdx.x] = (uint16_t)k;
    }
    return b;
}

// 4 (i / 4) + ... : row i of a lane in an accumulator
__device__ __forceinline__ int row_of(int i, int lane) { return 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3); }

// A tile's place: worker, sequence, head, and its first row
struct Place {
    uint32_t worker, seq, head, first, length;
};
__device__ __forceinline__ Place place_of(const Args &a, gemm::Launch l, uint32_t heads, bool last_first)
{
    Place p;
    uint32_t id = gemm::tile_run(l.first + blockIdx.x, l.total);
    const uint32_t unit = id / a.tiles;
    id -= unit * a.tiles;
    p.first = (last_first ? a.tiles - 1 - id : id) * kRows;
    p.head = unit % heads;
    p.seq = a.seq_first + unit / heads % a.seq_count;
    p.worker = unit / heads / a.seq_count;
    int64_t length = a.len;
    if (a.lengths) {
        const int32_t given = a.lengths[p.worker * a.seqs + p.seq];
        length = given < 0 ? 0 : given < length ? given : length;
    }
    p.length = (uint32_t)length;
    return p;
}

template <int T>
__device__ __forceinline__ const typename TypeOf<T>::type *rows_of(const void *p, Rows r, const Args &a, const Place &at, uint32_t head)
{
    return (const typename TypeOf<T>::type *)p + at.worker * r.worker + (int64_t)at.seq * a.len * r.row + (int64_t)head * a.dim;
}
template <int T>
__device__ __forceinline__ typename TypeOf<T>::type *rows_of(void *p, Rows r, const Args &a, const Place &at, uint32_t head)
{
    return (typename TypeOf<T>::type *)p + at.worker * r.worker + (int64_t)at.seq * a.len * r.row + (int64_t)head * a.dim;
}
__device__ __forceinline__ int64_t stats_of(const Args &a, const Place &at, uint32_t head)
{
    return ((int64_t)at.worker * a.heads + head) * a.t + (int64_t)at.seq * a.len;
}

// runs body with the head's width, rounded up, as a compile-time constant
#define SAMS_BY_WIDTH(dim, D, ...)                                 \
    do {                                                           \
        if ((dim) <= 32) { constexpr int D = 32; __VA_ARGS__; }    \
        else if ((dim) <= 64) { constexpr int D = 64; __VA_ARGS__; } \
        else if ((dim) <= 96) { constexpr int D = 96; __VA_ARGS__; } \
        else { constexpr int D = 128; __VA_ARGS__; }               \
    } while (0)

constexpr int kLdsBytes = 160 * 1024;
hipError_t prepare_forward(int type, uint32_t dim);
hipError_t prepare_backward(int type, uint32_t dim);
void launch_forward(const Args &a, int type, hipStream_t stream);
void launch_backward(const Args &a, int type, int64_t parts, float *dbias, int64_t dbias_worker, int accumulate, hipStream_t stream);

}  // namespace attn
}  // namespace sams
