// What the passes of the attention with a bias by relative position have in common: their arguments, the tiles' way through LDS to the
// matrix cores, and what a distance between two tokens means.
#pragma once
#include "sams_gemm.h"
#include "sams_random.h"

namespace sams {
namespace attn {

using gemm::f32x16;
using gemm::u32x4;

// A workgroup's rows: 32 for each wavefront, which keeps them in registers; or, with SPLIT 2, for each two of them, which take half of the
// rows that are streamed each and add up their results at the end.
constexpr int kThreads = 256, kWaves = 4, kRows = 128;
template <int SPLIT> constexpr int kOwn = kRows / SPLIT;
constexpr float kLog2e = 1.44269504088896340736f;
// A bias, or a row's largest logit, of this size or more leaves a logit (in units of ln 2) four bits behind the point at most, so that the order in which
// numbers are added to it moves P by more than a word of 16 bits shows, and from 2^25 on by powers of two.  From here on logits are rounded as sums first, the same in
// all kernels, before the largest is taken off.
constexpr float kLarge = 1e6f;

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
    float *part;                    // [n][heads][seqs * tiles][buckets]: the bias's gradient, in parts
    float *dbias;                   // [n][heads][buckets], where there is one part
    int64_t dbias_worker;
    float dbias_scale;
    int32_t accumulate;
    int64_t t;
    uint32_t n, seqs, len, heads, kv_heads, dim, buckets, tiles;
    uint32_t seq_first, seq_count;  // sequences that a launch deals with, of every worker
    int32_t edge_lo, edge_hi;       // the second bucket's start, and the last one's
    int32_t table_first;            // distances that are looked up in a table: the first one, and how many; 0: none are
    uint32_t table_count;
    const uint16_t *table_buckets;  // [table_count]
    uint32_t head_pieces, query_pieces;     // that the rows of a key's sums are cut into, of a group's heads and of a head's queries
    float *dk_parts, *dv_parts;     // [pieces][n][t][kv_heads * dim], if there are several
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

// ---- tiles in LDS ----
// Rows of D numbers have room for a power of two of pieces of 16 bytes; piece c of row r lies at c ^ turn(r).  So the pieces that sixteen lanes read at a time lie on
// different banks, whether they are one piece of sixteen rows, or four of each of four rows (counters show no bank conflict in any kernel).  The
// turn of a row is that of its bits one by one: a lane's part of an address is made once, and what the instruction adds to it comes by exclusive or.
template <int PIECES>
__host__ __device__ constexpr uint32_t turn(uint32_t r)
{
    return PIECES == 4 ? (r >> 2) & 3 : PIECES == 8 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3);
}
constexpr int power_of_two(int n) { return n <= 4 ? 4 : 2 * power_of_two((n + 1) / 2); }

typedef __attribute__((address_space(3))) char *lds_at;
__device__ __forceinline__ lds_at in_lds(uint32_t at) { return (lds_at)(uintptr_t)at; }
__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(lds_at)p; }

template <int T, int D> struct Tile {
    typedef typename TypeOf<T>::type E;
    typedef typename Fragment<T>::type Frag;
    static constexpr int SIZE = sizeof(E);
    static constexpr int ROWS = T == SAMS_F32 && D > 64 ? 32 : 64;              // that a workgroup takes at a time
    static constexpr int PIECES = D * SIZE / 16, ROOM = power_of_two(PIECES);   // a row's, and what it has room for
    static constexpr int LD = ROOM * 16, BYTES = ROWS * LD;
    static constexpr int N = ROWS * PIECES / kThreads;                          // pieces that a thread brings
    static_assert(ROWS * PIECES % kThreads == 0, "every thread brings as many");

    // A lane's addresses, of the first of two tiles that follow each other; the other one's are BYTES further, which is an exclusive or too.  They stay
    // in registers: reading a fragment takes the one instruction.
    struct Along {                  // numbers 16 s + 8 (lane / 32) .. + 7 of row row0 + lane % 32
        uint32_t at[D / 16];
        __device__ __forceinline__ void init(uint32_t tile, int lane)
        {
            const uint32_t r = lane & 31, c = (lane >> 5) * (SIZE / 2), from = tile + r * LD + ((c ^ turn<ROOM>(r)) << 4);
#pragma unroll
            for (int s = 0; s < D / 16; ++s) at[s] = from ^ (s * 16 * SIZE);
        }
        __device__ __forceinline__ void move(uint32_t bits)        // to the other tile (BYTES), or to its other 32 rows (32 LD)
        {
#pragma unroll
            for (int s = 0; s < D / 16; ++s) at[s] ^= bits;
        }
        // of the tile `further` bytes behind
        __device__ __forceinline__ Frag read(int further, int row0, int s) const
        {
            if constexpr (T == SAMS_F32) {
                typedef float f4 __attribute__((ext_vector_type(4)));
                typedef __attribute__((address_space(3))) const f4 *f4_at;
                const f4 a = *(f4_at)in_lds(at[s] + row0 * LD + further), b = *(f4_at)in_lds((at[s] ^ 16) + row0 * LD + further);
                return Frag{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            } else {
                return *(__attribute__((address_space(3))) const u32x4 *)in_lds(at[s] + row0 * LD + further);
            }
        }
    };
    // Column col0 + lane % 32 of the rows row0 + 4 (lane / 32) + {0 .. 3, 8 .. 11}.  16-bit words through the transposing load: of every 16
    // lanes four give the address of one row's 16 columns, and each gets one column's four rows.
    struct Across {
        static constexpr int OWN = T == SAMS_F32 ? 1 : 2 * (D / 32);
        uint32_t at[OWN];
        __device__ __forceinline__ void init(uint32_t tile, int lane)
        {
            if constexpr (T == SAMS_F32) {
                const uint32_t r = 4 * (lane >> 5), c = (lane & 31) >> 2;
                at[0] = tile + r * LD + ((c ^ turn<ROOM>(r)) << 4) + (lane & 3) * 4;
            } else {
                const uint32_t g = lane >> 4, q = lane & 15, r = 4 * (g >> 1) + (q >> 2), c = (g & 1) * 2 + ((q & 3) >> 1);
                const uint32_t from = tile + r * LD + ((c ^ turn<ROOM>(r)) << 4) + (q & 1) * 8;
#pragma unroll
                for (int i = 0; i < OWN; ++i) at[i] = from ^ ((i >> 1) * 64) ^ ((i & 1) * (turn<ROOM>(8) << 4));
            }
        }
        __device__ __forceinline__ void move(uint32_t bits)
        {
#pragma unroll
            for (int i = 0; i < OWN; ++i) at[i] ^= bits;
        }
        __device__ __forceinline__ Frag read(int further, int row0, int d) const           // col0 = 32 d
        {
            if constexpr (T == SAMS_F32) {
                Frag f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t r = (i & 3) + 8 * (i >> 2);
                    f[i] = *(__attribute__((address_space(3))) const float *)in_lds((at[0] ^ ((turn<ROOM>(r) << 4) ^ (d * 128))) + (row0 + r) * LD + further);
                }
                return f;
            } else {
                typedef __attribute__((address_space(3))) gemm::short4v *words_at;
                const gemm::words2 a = __builtin_bit_cast(gemm::words2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((words_at)in_lds(at[2 * d] + row0 * LD + further)));
                const gemm::words2 b = __builtin_bit_cast(gemm::words2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((words_at)in_lds(at[2 * d + 1] + (row0 + 8) * LD + further)));
                return Frag{a[0], a[1], b[0], b[1]};
            }
        }
    };
};

// The order of READS reads of LDS and MFMAS matrix instructions that stand before it: AHEAD reads are under way when the first matrix instruction
// begins, and behind each come some more.  (Left to itself, the compiler reads a fragment, waits for it and uses it: dk and dv of 8,192 tokens of 128 columns
// 1.36 ms instead of 1.13, where a SIMD has one wavefront.)
template <int READS, int MFMAS, int AHEAD>
__device__ __forceinline__ void in_order()
{
    constexpr int EACH = (READS + MFMAS - 1) / MFMAS;
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < MFMAS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (AHEAD + i * EACH < READS) __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
    }
}

// What was read before this is under way before any of it is used.  (The compiler would wait for each number in turn: dk and dv of 14 padded sequences'
// 10 heads of 72 79 us instead of 63, of 8 workers' 12 heads of 1024 107 instead of 100.)
__device__ __forceinline__ void all_under_way() { __builtin_amdgcn_sched_barrier(0); }

// ---- rows in memory ----
// A piece of 16 bytes of a row of dim numbers is read where all of it exists: one that reaches past the row's end, or starts there, in its place
// the row's last 16 bytes, of which `ended` makes what was meant.  (dim >= 8; rows start anywhere.)
template <int T> __device__ __forceinline__ uint32_t piece_start(uint32_t at, uint32_t dim) { return at + kPiece<T> <= dim ? at : dim - kPiece<T>; }

template <int T>
__device__ __forceinline__ void read_piece(const char *p, uint32_t (&raw)[4])
{
    const piece_t v = *(const piece_t *)p;
    raw[0] = v[0]; raw[1] = v[1]; raw[2] = v[2]; raw[3] = v[3];
}
template <int T>
__device__ __forceinline__ void ended(uint32_t (&raw)[4], bool there, uint32_t at, uint32_t dim)
{
    constexpr uint32_t N = kPiece<T>;
    if (const uint32_t rest = dim % N) {                            // the same for all threads
        uint64_t lo = raw[0] | (uint64_t)raw[1] << 32, hi = raw[2] | (uint64_t)raw[3] << 32;
        const uint32_t bits = (N - rest) * (128 / N);               // that lie before the piece
        if (bits < 64) {
            lo = lo >> bits | hi << (64 - bits);
            hi >>= bits;
        } else {
            lo = hi >> (bits - 64);
            hi = 0;
        }
        const bool part = at + N > dim;
        raw[0] = part ? (uint32_t)lo : raw[0];
        raw[1] = part ? (uint32_t)(lo >> 32) : raw[1];
        raw[2] = part ? (uint32_t)hi : raw[2];
        raw[3] = part ? (uint32_t)(hi >> 32) : raw[3];
    }
    there = there && at < dim;
#pragma unroll
    for (int e = 0; e < 4; ++e) raw[e] = there ? raw[e] : 0;
}

// A tile on its way to LDS: rows from `first` on, those from `limit` on and columns from dim on as zeros.
template <int T, int D>
struct Bring {
    typedef Tile<T, D> Ti;
    typedef typename TypeOf<T>::type E;
    uint32_t raw[Ti::N][4];

    __device__ __forceinline__ static uint32_t row_of(int i) { return (i * kThreads + threadIdx.x) / Ti::PIECES; }
    __device__ __forceinline__ static uint32_t column_of(int i) { return (i * kThreads + threadIdx.x) % Ti::PIECES * kPiece<T>; }

    // limit > first
    __device__ __forceinline__ void load(const E *p, int64_t row, uint32_t first, uint32_t limit, uint32_t dim)
    {
        const char *base = (const char *)(p + (int64_t)first * row);
        const int64_t bytes = row * Ti::SIZE;
        const uint32_t last = limit - first - 1;
#pragma unroll
        for (int i = 0; i < Ti::N; ++i) {
            const uint32_t r = row_of(i) < last ? row_of(i) : last;
            read_piece<T>(base + r * bytes + piece_start<T>(column_of(i), dim) * Ti::SIZE, raw[i]);
        }
    }
    // first, limit, dim: as they were loaded
    __device__ __forceinline__ void store(char *tile, uint32_t first, uint32_t limit, uint32_t dim)
    {
        if (first + Ti::ROWS > limit || dim != D) {
#pragma unroll
            for (int i = 0; i < Ti::N; ++i) ended<T>(raw[i], first + row_of(i) < limit, column_of(i), dim);
        }
#pragma unroll
        for (int i = 0; i < Ti::N; ++i) {
            const uint32_t r = row_of(i), c = (i * kThreads + threadIdx.x) % Ti::PIECES;
            *(u32x4 *)(tile + r * Ti::LD + ((c ^ turn<Ti::ROOM>(r)) << 4)) = u32x4{raw[i][0], raw[i][1], raw[i][2], raw[i][3]};
        }
    }
};

// A lane's fragments of row `row` of those from p on, which stay in registers: all zeros from row `limit` on (limit > 0).
template <int T, int D>
__device__ __forceinline__ void row_fragments(const typename TypeOf<T>::type *p, int64_t stride, uint32_t row, uint32_t limit, uint32_t dim, int lane,
                                              typename Fragment<T>::type (&f)[D / 16])
{
    p += (int64_t)(row < limit ? row : limit - 1) * stride;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
        for (int h = 0; h < 8; h += kPiece<T>) {
            const uint32_t at = 16 * s + 8 * (lane >> 5) + h;
            uint32_t raw[4];
            read_piece<T>((const char *)(p + piece_start<T>(at, dim)), raw);
            ended<T>(raw, row < limit, at, dim);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (T == SAMS_F32) f[s][h + e] = __builtin_bit_cast(float, raw[e]);
                else f[s][e] = raw[e];
            }
        }
}

// what both halves of the wavefront have for a column, added up, and the larger of both
__device__ __forceinline__ void halves(float v, float &a, float &b)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    a = __builtin_bit_cast(float, (uint32_t)r[0]);
    b = __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float sum_halves(float v)
{
    float a, b;
    halves(v, a, b);
    return a + b;
}
__device__ __forceinline__ float max_halves(float v)
{
    float a, b;
    halves(v, a, b);
    return fmaxf(a, b);
}

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
            if (dim % 4 == 0) {                                     // the same for all threads
                typedef uint32_t anywhere __attribute__((ext_vector_type(sizeof(E)), aligned(2)));
                if (at < dim) *(anywhere *)(row + at) = __builtin_bit_cast(anywhere, gemm::pack_numbers<E>(v));
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (at + i < dim) row[at + i] = (E)v[i];
            }
        }
}

// ---- the bias ----
// Bucket b is the distances (key minus query) from starts[b] on to starts[b + 1] - 1; what lies before starts[1] is bucket 0.  A wavefront's
// tile whose distances all lie before starts[1], or all from the last start on, adds one number.  For others the workgroup has the biases
// of the distances in between by distance in LDS, and kReach more on both sides, so that such a tile's all are there; where
// these are too many ("wide"), a tile is looked at for a start within its distances, and where there is one, the wavefront makes a table
// of its own for it.
constexpr int kReach = 96, kMaxTable = 4096;     // 16 KB of LDS, 24 where the bias's gradient is made

__device__ __forceinline__ float bias_of(float v)
{
    // numbers stay numbers, however large: rows of nothing but the type's lowest value have equal weights
    return __builtin_isfinite(v) ? fminf(fmaxf(v * kLog2e, -1.7e38f), 1.7e38f) : v;
}

struct Bias {
    float *table;           // in LDS: [table_count], or, where that is 0, [kWaves][kReach] of the wavefronts' present tiles
    uint16_t *which;        // in LDS: [table_count] the buckets that the table's biases are of, for who wants them
    const int *starts;      // in LDS: [buckets], where there is no table
    const float *row;       // [buckets], the head's
    float before, behind;   // the first and the last bucket's

    // where they lie in LDS, and how much they take
    __device__ __forceinline__ void place(const Args &a, char *lds)
    {
        table = (float *)lds;
        which = (uint16_t *)(table + a.table_count);
        starts = (const int *)(table + kWaves * kReach);
    }
    static int bytes(const Args &a, bool buckets_too = false)
    {
        return a.table_count ? (int)a.table_count * (buckets_too ? 6 : 4) : (kWaves * kReach + (int)a.buckets) * 4;
    }
    // the workgroup's starts, or the table's buckets; a barrier follows
    __device__ __forceinline__ void bring_starts(const Args &a, bool buckets_too = false) const
    {
        if (a.table_count) {
            if (buckets_too)
                for (uint32_t i = threadIdx.x; i < a.table_count; i += kThreads) which[i] = a.table_buckets[i];
        } else {
            for (uint32_t b = threadIdx.x; b < a.buckets; b += kThreads) ((int *)starts)[b] = a.starts[b];
        }
    }
    // a head's biases; a barrier follows
    __device__ __forceinline__ void bring(const Args &a, uint32_t head)
    {
        before = behind = 0.f;
        if (a.buckets == 0) return;
        row = a.bias + (int64_t)head * a.buckets;
        before = bias_of(row[0]);
        behind = bias_of(row[a.buckets - 1]);
        for (uint32_t i = threadIdx.x; i < a.table_count; i += kThreads) table[i] = bias_of(row[a.table_buckets[i]]);
    }
    __device__ __forceinline__ uint32_t bucket(const Args &a, int distance) const
    {
        if (a.table_count) return which[distance - a.table_first];
        uint32_t lo = 0, n = a.buckets;             // the answer is one of lo .. lo + n - 1
        while (n > 1) {
            const uint32_t half = n >> 1;
            const bool up = starts[lo + half] <= distance;
            lo = up ? lo + half : lo;
            n = up ? n - half : half;
        }
        return lo;
    }
    // whether the distances from lo to hi (kReach apart at most) share a bucket, which one, and its bias
    __device__ __forceinline__ bool one(const Args &a, int lo, int hi, uint32_t &bucket, float &value) const
    {
        bucket = 0;
        value = before;
        if (a.buckets < 2 || hi < a.edge_lo) return true;
        bucket = a.buckets - 1;
        value = behind;
        if (lo >= a.edge_hi) return true;
        if (a.table_count) return false;
        uint32_t below = 0, above = 0;
        for (uint32_t b = 0; b < a.buckets; b += 64) {
            const uint32_t i = b + (threadIdx.x & 63);
            const bool there = i > 0 && i < a.buckets;
            const int start = there ? starts[i] : 0;
            below += __builtin_popcountll(__ballot(there && start <= lo));
            above += __builtin_popcountll(__ballot(there && start <= hi));
        }
        bucket = below;
        value = bias_of(row[below]);
        return below == above;
    }
    // where the bias of `distance`, one of those from lo to lo + kReach - 1, lies, and of those around it
    __device__ __forceinline__ const float *at(const Args &a, int wave, int lo, int distance) const
    {
        if (a.table_count) return table + (distance - a.table_first);
        float *mine = table + wave * kReach;
        const int lane = threadIdx.x & 63;
        __builtin_amdgcn_wave_barrier();
        for (int i = lane; i < kReach; i += 64) mine[i] = bias_of(row[bucket(a, lo + i)]);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        return mine + (distance - lo);
    }
};

// 4 (i / 4) + ... : row i of a lane in an accumulator
__device__ __forceinline__ int row_of(int i, int lane) { return 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3); }

__device__ __forceinline__ int uniform_wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// Wavefronts that a SIMD is to hold, as registers for them go: 256 for each of two, which cover each other's waits.  What the 96 columns' kernels keep in
// memory for that costs less than one wavefront does (14 padded sequences' 10 heads of 72: dk and dv 85 us, alone 107; dq 40 and 52); at 128 columns it
// costs more (8,192 tokens: dk and dv 1.12 ms alone, 2.4 as two).
template <int T, int D> constexpr int kWavesPerSimd = (T == SAMS_F32 ? 2 : 1) * D <= 96 ? 2 : 1;

template <int T, int D>
__device__ __forceinline__ void flip(typename Fragment<T>::type (&f)[D / 16])
{
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
        if constexpr (T == SAMS_F32) f[s] = -f[s];
        else f[s] ^= 0x80008000u;
    }
}

// s = times s + bias of every pair, of a lane's query and the keys of its accumulators; from: where the bias of the first key lies, where
// they differ
template <int NB>
__device__ __forceinline__ void add_bias(const float *from, bool one, float by, float times, int lane, f32x16 (&s)[NB])
{
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        if (one) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[j][i] = __builtin_fmaf(s[j][i], times, by);
        } else {
            float b[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) b[i] = from[32 * j + row_of(i, lane)];
            all_under_way();
#pragma unroll
            for (int i = 0; i < 16; ++i) s[j][i] = __builtin_fmaf(s[j][i], times, b[i]);
        }
    }
}

// A tile's place: worker, sequence, head, and its first row
struct Place {
    uint32_t worker, seq, head, first, length;
};
template <int OWN>
__device__ __forceinline__ Place place_of(const Args &a, gemm::Launch l, uint32_t heads, bool last_first)
{
    Place p;
    // Workgroups go round the eight XCDs one by one.  Each XCD gets the tiles of some heads, so that they find keys and values in its L2; of those
    // the heads' longest tiles come first, so that short ones are left for the end (8 workers' 12 heads of 1024: 71 -> 51 us forward, 89 -> 67 for dq,
    // 176 -> 128 for dk and dv).
    uint32_t id, unit;
    const uint32_t units = l.total / a.tiles;
    if (units % 8 == 0 && gridDim.x == l.total) {
        const uint32_t each = units / 8, i = blockIdx.x >> 3;
        id = i / each;
        unit = (blockIdx.x & 7) * each + (i - id * each);
    } else {
        id = gemm::tile_run(l.first + blockIdx.x, l.total);
        unit = id / a.tiles;
        id -= unit * a.tiles;
    }
    p.first = (last_first ? a.tiles - 1 - id : id) * OWN;
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

// Whether workgroups have two wavefronts for every 32 rows: where 128 rows each would make few of them, or half of a workgroup's wavefronts had
// none.  4 workers' 12 heads of 511 in 32 bits (192 workgroups): forward 54 -> 41 us, dq 73 -> 50, dk and dv 119 -> 79; 48 heads of 1024 (384): forward 27 -> 23; but 14 padded sequences' 10 heads of 333 (420) 25 -> 31,
// and 8 workers' 12 heads of 1024 (768) 46 -> 48.  64 sequences of 50, 16 heads of 64 over 4: forward 15 -> 13.5, backward 55 -> 48; of 40 in 32 bits, 12 heads: 30 -> 20, 104 -> 83.  The limit lies between the 384 and 420 measured, of two widths, and is
// one for all kernels and widths.
constexpr int64_t kFewBlocks = 400;
static inline bool in_halves(int64_t heads_in_all, uint32_t len) { return len <= kRows / 2 || heads_in_all * ((len + kRows - 1) / kRows) < kFewBlocks; }
template <int SPLIT> static inline uint32_t tiles_of(uint32_t len) { return (len + kOwn<SPLIT> - 1) / kOwn<SPLIT>; }
// f(SPLIT), as a compile-time constant; tiles of 32 streamed rows are not split
template <int ROWS, typename F>
static void by_split(bool halves, F f)
{
    if constexpr (ROWS == 64) {
        if (halves) return f(std::integral_constant<int, 2>());
    }
    f(std::integral_constant<int, 1>());
}

// N numbers of every lane of a wavefront for another one of the same rows, through LDS
template <int N>
__device__ __forceinline__ void give(float *lds, const float (&v)[N], int lane)
{
#pragma unroll
    for (int i = 0; i < N; ++i) lds[i * 64 + lane] = v[i];
}
hipError_t prepare_forward(int type, uint32_t dim);
hipError_t prepare_backward(int type, uint32_t dim);
void launch_forward(const Args &a, int type, hipStream_t stream);
// numbers that the scratch holds of dk's parts, and of dv's
int64_t sums_room(int32_t n, int64_t t_max, int32_t heads, int32_t kv_heads, int32_t dim);
void launch_backward(const Args &a, int type, int64_t parts, int64_t sums, float *dbias, int64_t dbias_worker, int accumulate, hipStream_t stream);

}  // namespace attn
}  // namespace sams
