// Products of 16-bit matrices on the matrix cores: C[m][n] = sum_k A(m, k) B(n, k) for one tile of C per workgroup, with
// 32-bit accumulators that stay in registers for whatever the kernel does with its tile.
#pragma once
#include <math.h>
#include <algorithm>
#include <type_traits>

#include "sams_ctx.h"

namespace sams {
namespace gemm {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// What the words of the operands are.  SPLIT: a 32-bit number as the sum of two 16-bit floats, the first rounded to nearest,
// the second what that left: 22 bits of mantissa.  A row of such numbers lies in blocks of 32: 32 first parts, then 32 second
// parts; a product of two numbers takes three of words (the fourth, of both second parts, is below the 22 bits).
enum Kind { BF16 = 0, F16 = 1, SPLIT = 2 };

// One operand.  K_ROWS false: row m (or n) has its k's next to each other; true: a row holds one k of all m (or n).
struct Operand {
    const uint16_t *p;
    int64_t ld;         // words from row to row, a multiple of 8, at most kMaxRowWords
    int64_t size;       // extent along m (or n), in numbers
};

template <int BM_, int BN_, int WAVES_M_, int WAVES_N_, int STAGES_, bool SPREAD16_ = false, bool SPREAD_PAIRS_ = false>
struct Shape {
    static constexpr bool SPREAD16 = SPREAD16_, SPREAD_PAIRS = SPREAD_PAIRS_;      // loads spread over two groups (see tile_product)
    static constexpr int BM = BM_, BN = BN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, STAGES = STAGES_;
    static constexpr int THREADS = 64 * WAVES_M * WAVES_N;
    static constexpr int MI = BM / WAVES_M / 32, NI = BN / WAVES_N / 32;
    static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128;
    static constexpr int LDS_BYTES = STAGES * (A_BYTES + B_BYTES);
};

template <int KIND>
__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (KIND == BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

// Where a 16-byte piece of a tile lies in LDS.  A tile whose rows are 128 bytes: piece c of row r at c ^ swizzle(r), so that the
// fragments of 8 or 16 rows next to each other fall on different banks.  A tile whose rows are k's: piece c of row k at
// c ^ swizzle_k(k), so that the four k's of a transposing read do.
__device__ __forceinline__ int swizzle(int row) { return ((row ^ (row >> 3)) & 1) | (row & 6); }
__device__ __forceinline__ int swizzle_k(int k) { return ((k & 3) << 2) | (k & 2); }
// the part of it that stays within a row of so many pieces
template <int PIECES> constexpr int kPieceMask = (PIECES & -PIECES) - 1;

template <int KIND> __host__ __device__ constexpr int tile_k() { return KIND == SPLIT ? 32 : 64; }      // numbers of k in a stage

// Loads of one operand's tile straight into LDS, 64 words of k (32 numbers of k where they are split) a stage.  They are buffer loads: an
// address that all threads share and moves on, each thread's distances from it, and zeros for a distance past kTileSpan, which rows and
// k's that do not exist are given.
constexpr uint32_t kTileSpan = 0x80000000u;
constexpr int64_t kMaxRowWords = 1 << 22;                           // a tile (256 rows, or 64 k's) spans less than that

// a number that all lanes share, as the instructions that want it in a scalar register need it
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// 16 bytes a lane from a buffer, to LDS from address `at` on, lane by lane.  No register is written, so nothing can be overwritten while
// it is under way.  Written out because the compiler waits for every such load of its own before it lets a transposing read go
// ahead (also of the stage that landed long ago): those who read the stage wait for it, in wait_and_meet.  The buffer's scalar registers
// may come from a readfirstlane right before: what the vector unit writes may be read by a load of it five wait states later, which the
// compiler does not add to instructions it has not made itself; the move to m0 is one, the s_nop four.  (m0 belongs to no value of the compiler's: it is a reserved register, written anew where it is used.)
__device__ __forceinline__ void load_to_lds(u32x4 buffer, uint32_t off, uint32_t at)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(buffer), "s"(at) : "memory");
}

template <int ROWS, int THREADS, int KIND, bool K_ROWS>
struct Loader {
    static constexpr int N = ROWS * 8 / THREADS;                    // 16-byte pieces a thread brings
    static constexpr int PIECES = K_ROWS ? (KIND == SPLIT ? ROWS / 4 : ROWS / 8) : 8;       // of a row of the tile
    const char *base;
    uint32_t off[N];
    int64_t step;

    __device__ __forceinline__ static int row_of(int i, int tid) { return (i * THREADS + tid) / PIECES; }
    __device__ __forceinline__ static int piece_of(int i, int tid)
    {
        const int row = row_of(i, tid), c = (i * THREADS + tid) % PIECES;
        return K_ROWS ? c ^ (swizzle_k(row) & kPieceMask<PIECES>) : c ^ swizzle(row);
    }
    // where a piece starts, in k
    __device__ __forceinline__ static int k_of(int i, int tid) { return K_ROWS ? row_of(i, tid) : (KIND == SPLIT ? piece_of(i, tid) & 3 : piece_of(i, tid)) * 8; }

    __device__ __forceinline__ void init(const Operand &op, int64_t first, int64_t k_first, int tid)
    {
        const int64_t wide = KIND == SPLIT ? 2 : 1;
        if constexpr (K_ROWS) base = (const char *)(op.p + k_first * op.ld + first * wide);
        else base = (const char *)(op.p + first * op.ld + k_first * wide);
        const int64_t words = (KIND == SPLIT ? (op.size + 31) / 32 * 64 : (op.size + 7) / 8 * 8) - first * wide;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = row_of(i, tid), c = piece_of(i, tid);
            const bool there = K_ROWS ? c * 8 < words : row < op.size - first;
            off[i] = there ? (uint32_t)(row * (uint32_t)op.ld * 2 + c * 16) : kTileSpan;
        }
        step = K_ROWS ? tile_k<KIND>() * op.ld * 2 : 128;
    }

    // before a stage's pieces are loaded.  left: k's from its start on
    __device__ __forceinline__ void begin(int tid, int left)
    {
        if (left < tile_k<KIND>()) {                                 // the last stage
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (k_of(i, tid) >= left) off[i] = kTileSpan;
        }
    }
    __device__ __forceinline__ void load(char *lds, int wave, int i)
    {
        const u32x4 buffer = {uniform((uint32_t)(uintptr_t)base), uniform((uint32_t)((uintptr_t)base >> 32) & 0xffff), kTileSpan, 0x00020000};
        const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wave * 1024;
        load_to_lds(buffer, off[i], uniform(at + i * THREADS * 16));
    }
    __device__ __forceinline__ void next() { base += step; }
};

// A lane's 8 k's of its row (lane % 32) for one matrix instruction: k = kbase + 8 * (lane / 32) .. + 7, of part `half` where split.
// Rows that are k's are read through the transposing load: of every 16 lanes, four give the address of one k's 16 columns, and each
// gets one column's four k's.
template <int ROWS, int KIND, bool K_ROWS>
__device__ __forceinline__ u32x4 fragment(const char *tile, int row0, int kbase, int half, int lane)
{
    if constexpr (K_ROWS) {
        constexpr int PIECES = KIND == SPLIT ? ROWS / 4 : ROWS / 8;
        const int g = lane >> 4, q = lane & 15;
        const int k = kbase + 8 * (g >> 1) + (q >> 2);
        const int w = (KIND == SPLIT ? row0 * 2 + half * 32 : row0) + (g & 1) * 16 + (q & 3) * 4;
        const char *at = tile + k * (PIECES * 16) + (((w >> 3) ^ (swizzle_k(k) & kPieceMask<PIECES>)) << 4) + (w & 7) * 2;
        typedef __attribute__((address_space(3))) short4v *lds_ptr;
        const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at));
        const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * (PIECES * 16)));
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
        return u32x4{a[0], a[1], b[0], b[1]};
    } else {
        const int row = row0 + (lane & 31), c = (kbase >> 3) + half * 4 + (lane >> 5);
        return *(const u32x4 *)(tile + row * 128 + ((c ^ swizzle(row)) << 4));
    }
}

// All but the N youngest loads of this thread have landed, its reads of LDS are done, and so are those of the workgroup's others.
template <int N>
__device__ __forceinline__ void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// acc += the tile's product over k numbers from k_first on.  `lds`: S::LDS_BYTES, 16-byte aligned; every thread of the workgroup
// calls it, and LDS is free again when it returns.
//
// A wavefront has the fragments of the next 16 k's on their way while the matrix instructions of these run, across stages too: the
// one barrier of a stage stands before its last fragments are used, when they are in registers and the next stage has
// landed; behind it the stage just read is filled anew.  The order of instructions is written out: after each matrix instruction a
// share of the reads of fragments.  Large tiles of 16-bit numbers have the loads spread over the two groups behind the barrier too
// (issued at once they hold a wavefront back for as long as a group takes: 4096^3 121 us, spread 112); the others need them early more
// (pairs in Middle, one tile a CU, k = 1536: 31 us at once, 40 spread).
// In two steps for those who have something else to do while the first stages are on their way: start() begins to load them, into all
// stages of LDS but the last, which is the caller's until finish().
template <class S, int KIND, bool A_K_ROWS, bool B_K_ROWS>
struct Product {
    typedef Loader<S::BM, S::THREADS, KIND, A_K_ROWS> LA;
    typedef Loader<S::BN, S::THREADS, KIND, B_K_ROWS> LB;
    static constexpr int BK = tile_k<KIND>(), STAGE = S::A_BYTES + S::B_BYTES, LOADS = LA::N + LB::N;
    LA la;
    LB lb;
    int left;

    __device__ __forceinline__ void load(char *to, int wave, int i)
    {
        if (i < LA::N) la.load(to, wave, i);
        else lb.load(to + S::A_BYTES, wave, i - LA::N);
    }
    __device__ __forceinline__ void begin()
    {
        la.begin(threadIdx.x, left);
        lb.begin(threadIdx.x, left);
        left -= BK;
    }
    __device__ __forceinline__ void next()
    {
        la.next();
        lb.next();
    }
    __device__ __forceinline__ void start(const Operand &A, int64_t m0, const Operand &B, int64_t n0, int64_t k_first, int64_t k, char *lds)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        la.init(A, m0, k_first, threadIdx.x);
        lb.init(B, n0, k_first, threadIdx.x);
        left = (int)k;
        if (k <= 0) return;
#pragma unroll
        for (int s = 0; s + 1 < S::STAGES; ++s) {                    // past k: zeros, here and below, so that the count of loads holds
            begin();
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load(lds + s * STAGE, wave, i);
            next();
        }
    }
    __device__ __forceinline__ void finish(f32x16 (&acc)[S::MI][S::NI], int64_t k, char *lds)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wm = wave / S::WAVES_N * S::MI * 32, wn = wave % S::WAVES_N * S::NI * 32;
        constexpr int HALVES = KIND == SPLIT ? 2 : 1, GROUPS = BK / 16, PRODUCTS = S::MI * S::NI * (KIND == SPLIT ? 3 : 1), FRAGMENTS = HALVES * (S::MI + S::NI);
        if (k <= 0) return;
        u32x4 fa[2][HALVES][S::MI], fb[2][HALVES][S::NI];
        auto read = [&](const char *stage, int group, int into, int f) {     // first parts first
            const int h = f / (S::MI + S::NI), e = f % (S::MI + S::NI);
            if (e < S::MI) fa[into][h][e] = fragment<S::BM, KIND, A_K_ROWS>(stage, wm + e * 32, group * 16, h, lane);
            else fb[into][h][e - S::MI] = fragment<S::BN, KIND, B_K_ROWS>(stage + S::A_BYTES, wn + (e - S::MI) * 32, group * 16, h, lane);
        };
        constexpr int BEHIND = (KIND == SPLIT ? S::SPREAD_PAIRS : S::SPREAD16) ? LOADS / 2 : LOADS;        // loads of a stage that the group behind the barrier begins
        // one group: its matrix instructions, the reads of another one, loads from `first` to `last` of a stage
        auto work = [&](int from, const char *stage, int group, int into, char *to, int first, int last) {
#pragma unroll
            for (int p = 0; p < PRODUCTS; ++p) {
                const int q = p / (S::MI * S::NI), i = p / S::NI % S::MI, j = p % S::NI;
                acc[i][j] = mfma<KIND>(fa[from][q == 2 ? HALVES - 1 : 0][i], fb[from][q == 1 ? HALVES - 1 : 0][j], acc[i][j]);
#pragma unroll
                for (int f = FRAGMENTS * p / PRODUCTS; f < FRAGMENTS * (p + 1) / PRODUCTS; ++f) read(stage, group, into, f);
                if (first < last)
#pragma unroll
                    for (int l = first + (last - first) * p / PRODUCTS; l < first + (last - first) * (p + 1) / PRODUCTS; ++l) load(to, wave, l);
                if constexpr (BEHIND < LOADS) __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (BEHIND == LOADS) {                             // the same order, without the compiler's hands tied in each place
                constexpr int READS = HALVES * (S::MI * (A_K_ROWS ? 2 : 1) + S::NI * (B_K_ROWS ? 2 : 1));
#pragma unroll
                for (int p = 0; p < PRODUCTS; ++p) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, (READS + PRODUCTS - 1) / PRODUCTS, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        constexpr int AHEAD = (S::STAGES - 2) * LOADS;                   // loads that may be under way when the next stage is read
        char *cur = lds, *nxt = lds + STAGE, *const end = lds + S::STAGES * STAGE, *fill = end - STAGE;
        begin();
#pragma unroll
        for (int i = 0; i < BEHIND; ++i) load(fill, wave, i);
        wait_and_meet<AHEAD + BEHIND>();
#pragma unroll
        for (int f = 0; f < FRAGMENTS; ++f) read(cur, 0, 0, f);
        for (int todo = (int)k; todo > 0; todo -= BK) {
            work(0, cur, 1, 1, fill, BEHIND, LOADS);                     // the second half of what the last group began to load
            next();
#pragma unroll
            for (int g = 1; g + 1 < GROUPS; ++g) work(g & 1, cur, g + 1, (g + 1) & 1, nullptr, 0, 0);
            wait_and_meet<AHEAD>();
            begin();
            if constexpr (BEHIND == LOADS) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) load(cur, wave, i);
                work((GROUPS - 1) & 1, nxt, 0, 0, nullptr, 0, 0);
            } else {
                work((GROUPS - 1) & 1, nxt, 0, 0, cur, 0, BEHIND);
            }                                                            // (reads after the last stage: what nobody uses)
            fill = cur;
            cur = nxt;
            nxt = nxt + STAGE == end ? lds : nxt + STAGE;
        }
        wait_and_meet<0>();
    }
};

template <class S, int KIND, bool A_K_ROWS, bool B_K_ROWS>
__device__ __forceinline__ void tile_product(f32x16 (&acc)[S::MI][S::NI], const Operand &A, int64_t m0, const Operand &B, int64_t n0, int64_t k_first,
                                             int64_t k, char *lds)
{
    Product<S, KIND, A_K_ROWS, B_K_ROWS> product;
    product.start(A, m0, B, n0, k_first, k, lds);
    product.finish(acc, k, lds);
}

template <class S>
__device__ __forceinline__ void clear(f32x16 (&acc)[S::MI][S::NI])
{
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NI; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
}

// A number as it stands in 32 bits.  The two parts of a pair are made from it; without this the compiler may round the first part
// straight from the factors of the product that the number is, once for the pair and once, otherwise, for what is left of it.
__device__ __forceinline__ float settled(float v)
{
    asm("" : "+v"(v));
    return v;
}

// Between a wavefront's writes to LDS and its other lanes' reads of them (which LDS serves in order): the compiler keeps the order too.
__device__ __forceinline__ void same_wave_lds() { asm volatile("" ::: "memory"); __builtin_amdgcn_wave_barrier(); }

// Hands the tile over row by row: C[n][m], n the row, m along it.  A lane holds four m's next to each other of one n, and 32 lanes 32
// rows, so that stores from the registers would touch 32 lines at once; each wavefront turns its 32 rows round in LDS and stores them in
// pieces of 16 bytes, a row's pieces in lanes next to each other.
//   row(n)            what the numbers of row n need (n counted from the tile's corner), computed once a lane and 32 rows
//   pack(r, m, v)     four numbers from m on: 8 bytes (BYTES 2), 16 bytes (BYTES 4), or for pairs the first parts, then the second
//   store(n, at, w)   16 bytes of row n, `at` bytes from the tile's corner
template <class S, int BYTES, bool PAIRS, typename Row, typename Pack, typename Store>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[S::MI][S::NI], char *lds, Row row, Pack pack, Store store)
{
    constexpr int ROW = S::MI * 32 * BYTES, PIECES = ROW / 16;
    static_assert(32 * ROW * S::WAVES_M * S::WAVES_N <= S::LDS_BYTES, "a wavefront's rows have to fit");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31;
    const int wm = wave / S::WAVES_N * S::MI * 32, wn = wave % S::WAVES_N * S::NI * 32;
    char *mine = lds + wave * 32 * ROW, *mine_row = mine + r * ROW;
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int j = 0; j < S::NI; ++j) {
        const auto what = row(wn + j * 32 + r);
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int m = i * 32 + q * 8 + (lane >> 5) * 4;
                const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                const auto w = pack(what, wm + m, v);
                if constexpr (PAIRS) {
                    const int at = i * 128 + (m & 31) * 2;
                    *(u32x2 *)(mine_row + (((at >> 4) ^ (r & kPieceMask<PIECES>)) << 4) + (at & 15)) = u32x2{w[0], w[1]};
                    *(u32x2 *)(mine_row + ((((at + 64) >> 4) ^ (r & kPieceMask<PIECES>)) << 4) + (at & 15)) = u32x2{w[2], w[3]};
                } else {
                    const int at = m * BYTES;
                    *(decltype(pack(what, 0, v)) *)(mine_row + (((at >> 4) ^ (r & kPieceMask<PIECES>)) << 4) + (at & 15)) = w;
                }
            }
        same_wave_lds();
#pragma unroll
        for (int it = 0; it < PIECES / 2; ++it) {
            const int slot = it * 64 + lane, n = slot / PIECES, c = slot % PIECES;
            store(wn + j * 32 + n, wm * BYTES + c * 16, *(const u32x4 *)(mine + n * ROW + ((c ^ (n & kPieceMask<PIECES>)) << 4)));
        }
        same_wave_lds();
    }
}

// The same with the numbers themselves in LDS: emit(n, m, v) gets eight numbers of row n from m on, so that what it reads beside them
// comes in pieces of 16 bytes too.  MIRROR: of the transposed tile, C[m][n]; emit(m, n, v).  A wavefront has the same bytes of LDS in either
// order, whichever side of its part of the tile is longer: one may be through with the tile and at its mirror image while another still
// reads the tile, and nothing but a wavefront's own order keeps the two apart.
template <class S, bool MIRROR, typename Emit>
__device__ __forceinline__ void eights(const f32x16 (&acc)[S::MI][S::NI], char *lds, Emit emit)
{
    constexpr int ALONG = (MIRROR ? S::NI : S::MI) * 32, ROW = ALONG * 4, PIECES = ROW / 16, EIGHTS = ALONG / 8;
    constexpr int MINE = 32 * 32 * 4 * (S::MI > S::NI ? S::MI : S::NI);
    static_assert(32 * ROW <= MINE && MINE * S::WAVES_M * S::WAVES_N <= S::LDS_BYTES, "a wavefront's rows have to fit");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 31, h = lane >> 5;
    const int wm = wave / S::WAVES_N * S::MI * 32, wn = wave % S::WAVES_N * S::NI * 32;
    char *mine = lds + wave * MINE;
    typedef float f32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int outer = 0; outer < (MIRROR ? S::MI : S::NI); ++outer) {
#pragma unroll
        for (int inner = 0; inner < (MIRROR ? S::NI : S::MI); ++inner)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x16 &a = MIRROR ? acc[outer][inner] : acc[inner][outer];
                if constexpr (MIRROR) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int r = 8 * q + 4 * h + e, at = (inner * 32 + l) * 4;
                        *(float *)(mine + r * ROW + (((at >> 4) ^ (r & kPieceMask<PIECES>)) << 4) + (at & 15)) = a[4 * q + e];
                    }
                } else {
                    const int c = (inner * 32 + 8 * q + 4 * h) >> 2;
                    *(f32x4 *)(mine + l * ROW + ((c ^ (l & kPieceMask<PIECES>)) << 4)) = f32x4{a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
                }
            }
        same_wave_lds();
#pragma unroll
        for (int it = 0; it < EIGHTS / 2; ++it) {
            const int slot = it * 64 + lane, r = slot / EIGHTS, c = slot % EIGHTS * 2;
            const f32x4 lo = *(const f32x4 *)(mine + r * ROW + ((c ^ (r & kPieceMask<PIECES>)) << 4)), hi = *(const f32x4 *)(mine + r * ROW + (((c + 1) ^ (r & kPieceMask<PIECES>)) << 4));
            const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            if constexpr (MIRROR) emit(wm + outer * 32 + r, wn + c * 4, v);
            else emit(wn + outer * 32 + r, wm + c * 4, v);
        }
        same_wave_lds();
    }
}

// eight numbers as words of an operand, whose row's number i (a multiple of 8) they start at; and back
template <int KIND>
__device__ __forceinline__ void put8(uint16_t *row, int64_t i, const float (&v)[8])
{
    if constexpr (KIND == BF16) {
        bf16x8 w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = (__bf16)v[e];
        *(bf16x8 *)(row + i) = w;
    } else {
        half8 w;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = KIND == SPLIT ? settled(v[e]) : v[e];
            w[e] = (_Float16)x[e];
        }
        if constexpr (KIND == SPLIT) {
            half8 rest;
#pragma unroll
            for (int e = 0; e < 8; ++e) rest[e] = (_Float16)(x[e] - (float)w[e]);
            uint16_t *p = row + (i >> 5) * 64 + (i & 31);
            *(half8 *)p = w;
            *(half8 *)(p + 32) = rest;
        } else {
            *(half8 *)(row + i) = w;
        }
    }
}

template <int KIND>
__device__ __forceinline__ void get8(const uint16_t *row, int64_t i, float (&v)[8])
{
    const uint16_t *p = KIND == SPLIT ? row + (i >> 5) * 64 + (i & 31) : row + i;
    const half8 w = *(const half8 *)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)w[e];
    if constexpr (KIND == SPLIT) {
        const half8 rest = *(const half8 *)(p + 32);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += (float)rest[e];
    }
}

template <typename E>
__device__ __forceinline__ uint32_t pair_of(float a, float b)
{
    typedef E e2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, e2{(E)a, (E)b});
}

typedef uint32_t words2 __attribute__((ext_vector_type(2)));

// four numbers as words of an operand, for store_rows
template <int KIND>
__device__ __forceinline__ auto pack_words(const float (&v)[4])
{
    if constexpr (KIND == SPLIT) {
        typedef _Float16 half2v __attribute__((ext_vector_type(2)));
        _Float16 first[4];
        float rest[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = settled(v[i]);
            first[i] = (_Float16)x;
            rest[i] = x - (float)first[i];
        }
        return u32x4{__builtin_bit_cast(uint32_t, half2v{first[0], first[1]}), __builtin_bit_cast(uint32_t, half2v{first[2], first[3]}), pair_of<_Float16>(rest[0], rest[1]),
                     pair_of<_Float16>(rest[2], rest[3])};
    } else if constexpr (KIND == F16) {
        return words2{pair_of<_Float16>(v[0], v[1]), pair_of<_Float16>(v[2], v[3])};
    } else {
        return words2{pair_of<__bf16>(v[0], v[1]), pair_of<__bf16>(v[2], v[3])};
    }
}

// four numbers as a caller's type, for store_rows
template <typename E>
__device__ __forceinline__ auto pack_numbers(const float (&v)[4])
{
    if constexpr (sizeof(E) == 4) return u32x4{__builtin_bit_cast(uint32_t, v[0]), __builtin_bit_cast(uint32_t, v[1]), __builtin_bit_cast(uint32_t, v[2]), __builtin_bit_cast(uint32_t, v[3])};
    else return words2{pair_of<E>(v[0], v[1]), pair_of<E>(v[2], v[3])};
}

// 16 bytes of a caller's row, of which numbers from `limit` on do not exist; rows start anywhere
template <typename E>
__device__ __forceinline__ void store_numbers(E *row, int64_t at, int64_t limit, u32x4 w)
{
    constexpr int N = 16 / sizeof(E);
    typedef uint32_t anywhere __attribute__((ext_vector_type(4), aligned(2)));
    if (at + N <= limit) {
        *(anywhere *)(row + at) = w;
    } else {
        E e[N];
        __builtin_memcpy(e, &w, 16);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (at + i < limit) row[at + i] = e[i];
    }
}

// A workgroup's place in `batch` grids of tiles.  Workgroups go round the eight XCDs one by one; each XCD gets a contiguous run of tiles,
// so that the tiles of a product meet their operands in few XCDs' L2 (12 products of 768^3 spread over all eight read them from the
// memory side at 11 TB/s), and a run goes over `kTileGroup` columns of tiles at a time.
constexpr int kTileGroup = 8;
__device__ __forceinline__ uint32_t tile_run(uint32_t id, uint32_t total)
{
    const uint32_t xcd = id & 7, each = total >> 3, over = total & 7;
    return xcd * each + (xcd < over ? xcd : over) + (id >> 3);
}
__device__ __forceinline__ void tile_place(uint32_t at, uint32_t total, uint32_t tiles_m, uint32_t tiles_n, uint32_t &mi, uint32_t &ni, uint32_t &batch)
{
    uint32_t id = tile_run(at, total);
    batch = id / (tiles_m * tiles_n);
    id -= batch * tiles_m * tiles_n;
    const uint32_t group = id / (kTileGroup * tiles_n), first = group * kTileGroup;
    const uint32_t wide = tiles_m - first < kTileGroup ? tiles_m - first : kTileGroup;
    const uint32_t in = id - first * tiles_n;
    mi = first + in % wide;
    ni = in / wide;
}
// A launch's share of the tiles: a grid may have fewer than 2^32 threads, which thin matrices' tiles can exceed.
struct Launch { uint32_t first, total; };
__device__ __forceinline__ void tile_place(Launch l, uint32_t tiles_m, uint32_t tiles_n, uint32_t &mi, uint32_t &ni, uint32_t &batch)
{
    tile_place(l.first + blockIdx.x, l.total, tiles_m, tiles_n, mi, ni, batch);
}
// f(workgroups, share) for as many launches as the tiles take; a first one that is a multiple of 8 leaves the XCDs' runs as they are
template <typename F>
static void in_launches(int64_t tiles, int threads, F f)
{
    const int64_t most = ((int64_t)1 << 31) / threads;
    for (int64_t first = 0; first < tiles; first += most) f(dim3((unsigned)std::min(most, tiles - first)), Launch{(uint32_t)first, (uint32_t)tiles});
}

// The tiles in use.  At 8192^3 (16 bits; pairs), Large reaches 1.27 PFLOP/s (0.45), 83 % of the library's 1.54 in 16 bits and three times
// its 0.15 in 32, the card's clock down to 1.85 GHz (1.55) by then; Wide 1.05 (0.36), there for products that make a CU's worth of its tiles
// but few of Large's; Middle 1.1, two workgroups on a CU; MiddlePairs (0.39), one; Small 0.65 (0.29).  Small's four
// stages cover a load's way where a CU has one workgroup: 640 x 640 x 12800 takes it 56 us (92), with two stages 95 (186), Middle 134 and, for
// pairs, with its two stages 267, MiddlePairs 150.
typedef Shape<256, 256, 2, 4, 2, true> Large;
typedef Shape<192, 192, 2, 2, 2> Wide;
typedef Shape<128, 128, 2, 2, 2> Middle;
typedef Shape<128, 128, 2, 2, 3, false, true> MiddlePairs;
typedef Shape<64, 64, 2, 2, 4> Small;

// What a product of m x n x k numbers, `batch` times, is estimated to take in tiles of a size (Large, Wide, Middle, Small), its k cut into
// `parts`, in ns: a CU's workgroups one after the other, each at the pace it has beside others or, alone on its CU, by itself
// (measured as above), and what a tile costs before and after its k's.
struct TileCost { int size; double pace16, alone16, pace_pairs, alone_pairs, fixed; };
constexpr TileCost kTileCosts[4] = {{256, 26, 26, 75, 75, 5000}, {192, 17, 17, 47.4, 47.4, 3500}, {128, 7.5, 10.5, 22, 17, 3000}, {64, 3.0, 4.4, 6.9, 7.2, 1200}};

static inline double tile_estimate(int shape, bool pairs, double tiles, double k, int parts)
{
    const TileCost &c = kTileCosts[shape];
    const double rounds = ceil(tiles * parts / 256), each = k / parts;
    return (rounds > 1 ? rounds * (pairs ? c.pace_pairs : c.pace16) : pairs ? c.alone_pairs : c.alone16) * each + rounds * c.fixed;
}

struct TileChoice { int shape, parts; };

// part_ns: what another part costs (its sums are written and read once more); triangular: tiles on and under the diagonal only
static inline TileChoice choose_tiles(bool pairs, int64_t batch, int64_t m, int64_t n, bool triangular, int64_t k, int most_parts, double part_ns)
{
    TileChoice best{2, 1};
    double least = 1e30;
    for (int shape = 0; shape < 4; ++shape) {
        const int64_t size = kTileCosts[shape].size, a = (m + size - 1) / size, b = (n + size - 1) / size;
        const double tiles = (double)batch * (triangular ? a * (a + 1) / 2 : a * b);
        for (int parts = 1; parts <= most_parts; ++parts) {
            const double ns = tile_estimate(shape, pairs, tiles, (double)k, parts) + (most_parts > 1 ? parts * part_ns : 0.0);
            if (ns < least) { least = ns; best = TileChoice{shape, parts}; }
        }
    }
    return best;
}

// workgroups of a kernel that goes from tile to tile: as many as the chip holds at once
template <class S> static uint32_t at_once(uint32_t tiles) { return std::min<uint32_t>(tiles, 256 * (163840 / S::LDS_BYTES)); }

template <int KIND, typename F>
static void with_tile(int shape, F f)
{
    if (shape == 0) f(Large());
    else if (shape == 1) f(Wide());
    else if (shape == 2) f(typename std::conditional<KIND == SPLIT, MiddlePairs, Middle>::type());
    else f(Small());
}

// words of a row of `numbers` numbers: whole 128-byte lines
template <int KIND> __host__ __device__ constexpr int64_t row_words(int64_t numbers)
{
    return KIND == SPLIT ? (numbers + 31) / 32 * 64 : (numbers + 63) / 64 * 64;
}
// numbers of such a row, with those that only fill it up
template <int KIND> __host__ __device__ constexpr int64_t row_numbers(int64_t numbers)
{
    return KIND == SPLIT ? (numbers + 31) / 32 * 32 : (numbers + 63) / 64 * 64;
}

}  // namespace gemm
}  // namespace sams
