// The attention's backward pass, from the forward pass's output and row statistics:
//
//   P_ij = exp(s_ij - max_i) / sum_i,   dP_ij = m_ij / (1 - p) do_i . v_j,   delta_i = do_i . o_i = sum_j P_ij dP_ij,   dS = P (dP - delta)
//   dv_j = sum_i m_ij / (1 - p) P_ij do_i,   dq_i = scale sum_j dS_ij k_j,   dk_j = scale sum_i dS_ij q_i
//   dbias[bucket] = sum of dS over the pairs whose distance lies in the bucket
//
// in two kernels, each of which makes S and dP again: one has the queries in registers and goes over the keys (delta, dq), one has
// the keys and goes over the queries of every head that shares them (dk, dv, dbias).  So every sum has one place and a fixed order, without
// atomics; seven products of a pair where one kernel would take five.
#include "sams_attn.h"

namespace sams {
namespace attn {

constexpr int kAhead = 4;       // fragments under way before the matrix instructions begin (8: 1 % either way)

// 16-bit floats have few digits below 2^-14, and dS may be all below that: a column of dS (a lane's, and that of the lane 32 from it) is
// multiplied by a power of two that brings its largest number so far to 2^14, and the column's sums with it.
template <int T, int D> struct ColumnScale {
    float by = 1.f;
    __device__ __forceinline__ void start() { if constexpr (T == SAMS_F16) by = 0x1p40f; }
    __device__ __forceinline__ void fit(f32x16 &v, f32x16 (&acc)[D / 32])
    {
        if constexpr (T == SAMS_F16) {
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(v[i]));
            most = max_halves(most);
            if (__any(most * by > 32768.f)) {
                const uint32_t power = __builtin_bit_cast(uint32_t, most) >> 23;            // 127 + its exponent
                const float next = most * by > 32768.f ? __builtin_bit_cast(float, (127 + 14 + 127 - power) << 23) : by;
                const float less = next / by;
                by = next;
#pragma unroll
                for (int d = 0; d < D / 32; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[d][i] *= less;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] *= by;
        }
    }
};

// Sums of dS by bucket, of a wavefront.  A tile of one bucket adds to a lane's own number, which is joined when the bucket changes.  In others the 32 x 32 numbers
// of a block are first added up along their diagonals: rotated by their row, a lane's numbers all belong to one of two distances, and those of a bucket follow
// each other.  (Adding each number to its bucket's in LDS takes twice the kernel's time: LDS adds 32-bit floats at a third of one a cycle.)
struct BucketSums {
    float *to;              // [buckets] in LDS, of this wavefront alone
    float own;
    uint32_t bucket;

    __device__ __forceinline__ void flush(int lane)
    {
        const float total = wave_sum(own);
        if (lane == 0) to[bucket] += total;
        own = 0.f;
    }
    __device__ __forceinline__ void one(uint32_t b, const f32x16 &ds, int lane)
    {
        if (b != bucket) {
            flush(lane);
            bucket = b;
        }
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = ds[i] + ds[i + 8];
        own += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    }
    // corner: the block's first key less its first query
    __device__ __forceinline__ void many(const Args &a, const Bias &bias, int corner, const f32x16 &ds, int lane)
    {
        float up = 0.f, down = 0.f;             // distances lane % 32 and lane % 32 - 32
        const int half = lane & 32;
        const int mine = (int)bias.bucket(a, corner + (lane ? lane : 1) - 32);
        float rotated[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) rotated[i] = __shfl(ds[i], ((row_of(i, lane) + lane) & 31) | half);
        all_under_way();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if ((lane & 31) + row_of(i, lane) < 32) up += rotated[i];
            else down += rotated[i];
        }
        up = sum_halves(up);
        down = sum_halves(down);
        float v = half ? up : down;             // the distance lane - 32
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {      // sums over the lanes of a bucket, which follow each other
            const float below = __shfl_up(v, o);
            const int theirs = __shfl_up(mine, o);
            if (lane >= o && theirs == mine) v += below;
        }
        const int next = __shfl_down(mine, 1);
        if (lane == 63 || next != mine) to[mine] += v;
        __builtin_amdgcn_wave_barrier();
    }
};

// dq and delta; laid out as the forward pass.  o has been rounded to 16 bits: what do . o is off by is small beside dP, but not beside the
// 32 bits that dbias is held to.  So delta is also added up as it is defined, sum P dP, for the other kernel, and dq, which needs it before that
// sum is done, is put right at the end: dq = scale (sum P (dP - d) k + (d - delta) sum P k), with d = do . o.  (Without: dbias off by 2.6e-3, dq by 2.6e-3
// instead of 2.4e-3; sum P k takes a quarter of the products.)  Bound as the forward pass: 8 workers' 12 heads of 1024 x 64 bf16 65 us, 400 TFLOP/s with sum P k and
// 300 without it, vector instructions in 56 % of a SIMD's time, the matrix core in 23 %; 8,192 tokens' 16 heads of 128 columns 677 us, 810 TFLOP/s (610), 35
// and 36 %, one wavefront a SIMD with 380 registers, which waits in 32 % of its time.
template <int T, int D, bool DROP, int SPLIT>
__global__ void __launch_bounds__(kThreads, (kWavesPerSimd<T, D>)) k_attn_dq(Args a, gemm::Launch launch)
{
    typedef Tile<T, D> Ti;
    typedef typename TypeOf<T>::type E;
    constexpr int BN = Ti::ROWS, NB = BN / 32 / SPLIT, OWN = kOwn<SPLIT>;
    constexpr float SHIFT = T == SAMS_F16 ? 14.f : 0.f;             // P in 16-bit floats: times 2^14
    constexpr bool ROUNDED = T != SAMS_F32;
    extern __shared__ __align__(16) char lds[];
    char *tile_k = lds, *tile_v = lds + 2 * Ti::BYTES;
    Bias bias;
    bias.place(a, lds + 4 * Ti::BYTES);

    const int lane = threadIdx.x & 63, wave = uniform_wave();
    const int half_of = wave % SPLIT;                              // which of a tile's keys
    const Place at = place_of<OWN>(a, launch, a.heads, a.causal);
    const uint32_t q0 = at.first + wave / SPLIT * 32, query = q0 + (lane & 31);
    const bool row_there = query < a.len, live = query < at.length;
    const int64_t stat = stats_of(a, at, at.head) + query;

    f32x16 acc[D / 32], pk[ROUNDED ? D / 32 : 1];
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = pk[ROUNDED ? d : 0][i] = 0.f;
    float over = 0.f;

    if (at.first < at.length) {
        const uint32_t kv = at.head / (a.heads / a.kv_heads);
        const E *k = rows_of<T>(a.k, a.ks, a, at, kv), *v = rows_of<T>(a.v, a.vs, a, at, kv);
        const uint32_t end = a.causal && at.first + OWN < at.length ? at.first + OWN : at.length;
        Seed seed = {};
        if constexpr (DROP) seed = read_seed(a.rng);
        const uint32_t stream = (at.worker * a.seqs + at.seq) * a.heads + at.head;

        Bring<T, D> bk, bv;
        bk.load(k, a.ks.row, 0, at.length, a.dim);
        bv.load(v, a.vs.row, 0, at.length, a.dim);
        typename Ti::Frag qf[D / 16], df[D / 16];
        row_fragments<T, D>(rows_of<T>(a.q, a.qs, a, at, at.head), a.qs.row, query, at.length, a.dim, lane, qf);
        // as in the forward pass: the matrix cores' sums of 16-bit words' products are not always negated with the words (those of 32-bit numbers are)
        const float scale = ROUNDED ? fabsf(a.scale2) : a.scale2;
        if (ROUNDED && a.scale2 < 0.f) flip<T, D>(qf);
        row_fragments<T, D>(rows_of<T>(a.dout, a.douts, a, at, at.head), a.douts.row, query, at.length, a.dim, lane, df);
        // do . o, less the factor 1 / (1 - p) that dP is made without
        float d = 0.f, exact = 0.f;
        {
            typename Ti::Frag of[D / 16];
            row_fragments<T, D>(rows_of<T>(a.o, a.os, a, at, at.head), a.os.row, query, at.length, a.dim, lane, of);
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                E x[8], y[8];
                __builtin_memcpy(x, &of[s], sizeof(x));
                __builtin_memcpy(y, &df[s], sizeof(y));
#pragma unroll
                for (int i = 0; i < 8; ++i) d = __builtin_fmaf((float)x[i], (float)y[i], d);
            }
            d = sum_halves(d) / a.keep.scale;
        }
        const float top = live ? a.row_max[stat] : 0.f, total = live ? a.row_sum[stat] : 0.f;
        const bool large = __any(fabsf(top) >= kLarge);
        over = total == 0.f ? 0.f : 1.f / total;
        ColumnScale<T, D> fit;
        fit.start();

        bias.bring_starts(a);
        bias.bring(a, at.head);
        bk.store(tile_k, 0, at.length, a.dim);
        bv.store(tile_v, 0, at.length, a.dim);
        typename Ti::Along rows;
        typename Ti::Across columns;
        rows.init(lds_address(lds) + half_of * (32 * Ti::LD), lane);
        columns.init(lds_address(lds) + half_of * (32 * Ti::LD), lane);
        __syncthreads();
        int turn = 0;
        for (uint32_t key0 = 0; key0 < end; key0 += BN, turn ^= 1) {
            const bool more = key0 + BN < end;
            if (more) {
                bk.load(k, a.ks.row, key0 + BN, at.length, a.dim);
                bv.load(v, a.vs.row, key0 + BN, at.length, a.dim);
            }
            const uint32_t mine = key0 + half_of * 32;              // the wavefront's first key
            const int lo = (int)mine - (int)(q0 + 31);
            uint32_t bucket;
            float by;
            const bool one = bias.one(a, lo, lo + NB * 32 - 1 + 31, bucket, by);
            if (q0 < at.length && mine < at.length && (!a.causal || mine <= q0 + 31) && !(one && by == -__builtin_inff())) {
                const bool edge = mine + NB * 32 > at.length || q0 + 32 > at.length || (a.causal && mine + NB * 32 - 1 > q0);
                const bool plain = one && !edge && fabsf(by) < kLarge && !large;    // as in the forward pass
                const float *biases = one ? nullptr : bias.at(a, wave, lo, lo + 31 - (lane & 31));
                const int limit = (live ? (int)(a.causal ? query + 1 : at.length) : 0) - (int)mine;
#pragma unroll 1
                for (int j = 0; j < NB; ++j) {
                    f32x16 s[1], dp;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[0][i] = dp[i] = 0.f;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) s[0] = product<T>(rows.read(0, 0, c), qf[c], s[0]);
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) dp = product<T>(rows.read(2 * Ti::BYTES, 0, c), df[c], dp);
                    if constexpr (T != SAMS_F32) in_order<D / 8, D / 8, kAhead>();
                    float times = scale, from = by - top + SHIFT;
                    if (!plain) {
                        add_bias<1>(biases + 32 * j, one, by, scale, lane, s);
                        times = 1.f;
                        from = SHIFT - top;
                        if (T == SAMS_F16 && large) {               // as in the forward pass
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[0][i] -= top;
                            from = SHIFT;
                        }
                        if (edge) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[0][i] = 32 * j + row_of(i, lane) < limit ? s[0][i] : -__builtin_inff();
                        }
                    }
                    // P, times the row's sum: that is divided out of the row's results at the end
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[0][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][i], times, from));
                    typename Ti::Frag wp[2];
                    if constexpr (ROUNDED) {
                        wp[0] = words_of<T>(s[0], 0);
                        wp[1] = words_of<T>(s[0], 1);
                    }
                    // dS = m P dP - P d
                    if constexpr (DROP) {
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            uint32_t numbers[4];
                            philox(seed, ((mine + 32 * j + 16 * half) >> 4) * 2 + (lane >> 5), query, stream, numbers);
#pragma unroll
                            for (int e = 0; e < 8; ++e) dp[8 * half + e] = kept(numbers, e, a.keep.least) ? dp[8 * half + e] : 0.f;
                        }
                    }
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        part[i & 3] = __builtin_fmaf(s[0][i], dp[i], part[i & 3]);
                        s[0][i] *= dp[i] - d;
                    }
                    exact += (part[0] + part[1]) + (part[2] + part[3]);
                    fit.fit(s[0], acc);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const typename Ti::Frag w = words_of<T>(s[0], half);
#pragma unroll
                        for (int d = 0; d < D / 32; ++d) {
                            const typename Ti::Frag k = columns.read(0, 16 * half, d);
                            acc[d] = product<T>(k, w, acc[d]);
                            if constexpr (ROUNDED) pk[d] = product<T>(k, wp[half], pk[d]);
                        }
                    }
                    if constexpr (T != SAMS_F32) in_order<D / 8, D / 8, kAhead>();
                    if constexpr (NB == 2) {
                        rows.move(32 * Ti::LD);
                        columns.move(32 * Ti::LD);
                    }
                }
            }
            if (more) {
                bk.store(tile_k + (turn ^ 1) * Ti::BYTES, key0 + BN, at.length, a.dim);
                bv.store(tile_v + (turn ^ 1) * Ti::BYTES, key0 + BN, at.length, a.dim);
            }
            rows.move(Ti::BYTES);
            columns.move(Ti::BYTES);
            __syncthreads();
        }
        over *= T == SAMS_F16 ? 0x1p-14f : 1.f;
        exact = sum_halves(exact) * over;
        if constexpr (SPLIT == 2) {
            // the odd wavefronts' results, which their neighbours add to their own; tiles are done with
            constexpr int N = (ROUNDED ? D : D / 2) + 1;
            float *there = (float *)lds + wave / 2 * (N * 64);
            if (half_of) {
                float v[N];
#pragma unroll
                for (int i = 0; i < D / 2; ++i) v[i] = acc[i / 16][i % 16] * (1.f / fit.by);
                if constexpr (ROUNDED)
#pragma unroll
                    for (int i = 0; i < D / 2; ++i) v[D / 2 + i] = pk[i / 16][i % 16];
                v[N - 1] = exact;
                give<N>(there, v, lane);
            }
            __syncthreads();
            if (half_of) return;
#pragma unroll
            for (int i = 0; i < D / 2; ++i) acc[i / 16][i % 16] = __builtin_fmaf(acc[i / 16][i % 16], 1.f / fit.by, there[i * 64 + lane]);
            if constexpr (ROUNDED)
#pragma unroll
                for (int i = 0; i < D / 2; ++i) pk[i / 16][i % 16] += there[(D / 2 + i) * 64 + lane];
            exact += there[(N - 1) * 64 + lane];
            fit.by = 1.f;
        }
        if (live && lane < 32) a.delta[stat] = exact;
        if constexpr (ROUNDED) {
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][e] = __builtin_fmaf(acc[i][e], 1.f / fit.by, (d - exact) * pk[i][e]);
        }
    }
    if (SPLIT == 2 && half_of) return;
    store_columns<T, D>(rows_of<T>(a.dq, a.dqs, a, at, at.head) + (int64_t)query * a.dqs.row, row_there, a.dim, acc, a.scale * a.keep.scale * over, lane);
}

// dk, dv and dbias.  A workgroup has 128 keys, a lane (and the lane 32 from it) one; queries and the output's gradients come by tiles.  The
// products are S = Q K' and dP = dO V', whose accumulators become the second operands of dV' = dO' P and dK' = Q' dS as they are.  Where there are few keys
// and heads of keys, a group's heads and a head's queries are shared out to several workgroups, whose sums another kernel joins.  The most of the three
// kernels' work for every pair: four products, two of them with both sides through LDS, and what the bias's gradient takes (16 of 148 us of a backward pass of 8 workers' 12 heads of 1024
// with 32 buckets).  103 us there, 250 TFLOP/s: vector instructions in 46 % of a SIMD's time, the matrix core busy in 13 %, a wavefront waiting in 48 % of its own; 8,192 tokens' 16
// heads of 128 columns, two heads of keys, 1.05 ms, 520 TFLOP/s, one wavefront a SIMD: 29, 23 and 43 %.
template <int T, int D, bool DROP, int SPLIT>
__global__ void __launch_bounds__(kThreads, (kWavesPerSimd<T, D>)) k_attn_dkv(Args a, gemm::Launch launch, int64_t parts)
{
    typedef Tile<T, D> Ti;
    constexpr int BQ = Ti::ROWS, NB = BQ / 32 / SPLIT, OWN = kOwn<SPLIT>;
    constexpr float SHIFT = T == SAMS_F16 ? 0x1p14f : 1.f;          // P in 16-bit floats
    constexpr int NUMBERS = 80;                                     // bytes of a query's numbers: 32 of 16 bits, and 16 that put the queries on different banks
    extern __shared__ __align__(16) char lds[];
    char *tile_q = lds, *tile_d = lds + 2 * Ti::BYTES;
    float *stats = (float *)(lds + 4 * Ti::BYTES);                  // [2][3][BQ]
    char *numbers_lds = (char *)(stats + 2 * 3 * BQ);               // [kWaves][32] queries' numbers
    float *sums_lds = (float *)(numbers_lds + (DROP ? kWaves * 32 * NUMBERS : 0));      // [kWaves][buckets]
    Bias bias;
    bias.place(a, (char *)(sums_lds + kWaves * a.buckets));

    const int lane = threadIdx.x & 63, wave = uniform_wave();
    const uint32_t pieces = a.head_pieces * a.query_pieces;
    const int half_of = wave % SPLIT;                              // which of a tile's queries
    Place at = place_of<OWN>(a, launch, a.kv_heads * pieces, false);
    const uint32_t piece = at.head % pieces, head_piece = piece / a.query_pieces, query_piece = piece % a.query_pieces;
    at.head /= pieces;
    const uint32_t k0 = at.first + wave / SPLIT * 32, key = k0 + (lane & 31);
    const bool row_there = key < a.len, live = key < at.length;

    f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.f;
    ColumnScale<T, D> fit;
    fit.start();
    const uint32_t group = a.heads / a.kv_heads / a.head_pieces, head0 = at.head * (a.heads / a.kv_heads) + head_piece * group;
    // this piece's tiles of queries; OWN is a multiple of BQ, so that the first key's tile is the first one where earlier queries see none
    const uint32_t tile0 = a.causal ? at.first / BQ : 0, tiles = (at.length + BQ - 1) / BQ;
    uint32_t begin = 0, end = 0;
    if (at.first < at.length) {
        begin = (tile0 + (tiles - tile0) * query_piece / a.query_pieces) * BQ;
        end = (tile0 + (tiles - tile0) * (query_piece + 1) / a.query_pieces) * BQ;
    }
    BucketSums sums = {sums_lds + wave * a.buckets, 0.f, 0};
    const bool summed = a.part || a.dbias;
    // a head's sums of the workgroup; between barriers
    auto leave = [&](uint32_t head, bool some) {
        float *part = a.part + (((int64_t)at.worker * a.heads + head) * parts + ((int64_t)(at.seq - a.seq_first) * a.tiles + at.first / OWN) * a.query_pieces + query_piece) * a.buckets;
        float *all = a.dbias + at.worker * a.dbias_worker + (int64_t)head * a.buckets;
        for (uint32_t b = threadIdx.x; b < a.buckets; b += kThreads) {
            const float v = some ? (sums_lds[b] + sums_lds[a.buckets + b]) + (sums_lds[2 * a.buckets + b] + sums_lds[3 * a.buckets + b]) : 0.f;
            if (a.dbias) all[b] = a.accumulate ? __builtin_fmaf(v, a.dbias_scale, all[b]) : v * a.dbias_scale;
            else part[b] = v;
        }
    };
    auto clear = [&]() {
        for (uint32_t i = threadIdx.x; i < kWaves * a.buckets; i += kThreads) sums_lds[i] = 0.f;
    };
    if (begin >= end) {
        for (uint32_t h = 0; summed && h < group; ++h) leave(head0 + h, false);
    } else {
        bias.bring_starts(a, summed);
        clear();
        Seed seed = {};
        if constexpr (DROP) seed = read_seed(a.rng);
        Bring<T, D> bq, bd;
        float stat[3] = {0.f, 0.f, 0.f};
        auto load = [&](uint32_t head, uint32_t query0) {
            bq.load(rows_of<T>(a.q, a.qs, a, at, head), a.qs.row, query0, at.length, a.dim);
            bd.load(rows_of<T>(a.dout, a.douts, a, at, head), a.douts.row, query0, at.length, a.dim);
            if (threadIdx.x < BQ) {
                const uint32_t query = query0 + threadIdx.x;
                const int64_t from = stats_of(a, at, head) + query;
                const bool there = query < at.length;
                const float total = there ? a.row_sum[from] : 0.f;
                stat[0] = there ? a.row_max[from] : 0.f;
                stat[1] = total == 0.f ? 0.f : SHIFT / total;
                stat[2] = there ? a.delta[from] : 0.f;
            }
        };
        auto store = [&](uint32_t query0, int turn) {
            bq.store(tile_q + turn * Ti::BYTES, query0, at.length, a.dim);
            bd.store(tile_d + turn * Ti::BYTES, query0, at.length, a.dim);
            if (threadIdx.x < BQ)
#pragma unroll
                for (int i = 0; i < 3; ++i) stats[(turn * 3 + i) * BQ + threadIdx.x] = stat[i];
        };
        uint32_t head = head0, query0 = begin;
        const uint32_t last = head + group - 1;
        load(head, query0);
        typename Ti::Frag kf[D / 16], vf[D / 16];
        row_fragments<T, D>(rows_of<T>(a.k, a.ks, a, at, at.head), a.ks.row, key, at.length, a.dim, lane, kf);
        row_fragments<T, D>(rows_of<T>(a.v, a.vs, a, at, at.head), a.vs.row, key, at.length, a.dim, lane, vf);
        const float scale = T == SAMS_F32 ? a.scale2 : fabsf(a.scale2);
        if (T != SAMS_F32 && a.scale2 < 0.f) flip<T, D>(kf);        // products as the other kernels make them
        bias.bring(a, head);
        store(query0, 0);
        typename Ti::Along rows;
        typename Ti::Across columns;
        rows.init(lds_address(lds) + half_of * (32 * Ti::LD), lane);
        columns.init(lds_address(lds) + half_of * (32 * Ti::LD), lane);
        __syncthreads();
        for (int turn = 0;; turn ^= 1) {
            uint32_t next_head = head, next_query0 = query0 + BQ;
            if (next_query0 >= end) { ++next_head; next_query0 = begin; }
            const bool more = next_head <= last;
            if (more) load(next_head, next_query0);
            const uint32_t mine0 = query0 + half_of * 32;           // the wavefront's first query
            const bool large = __any(fabsf(stats[turn * 3 * BQ + half_of * 32 + (lane & (NB * 32 - 1))]) >= kLarge);
            const int lo = (int)k0 - (int)(mine0 + NB * 32 - 1);
            uint32_t bucket;
            float by;
            const bool one = bias.one(a, lo, lo + NB * 32 - 1 + 31, bucket, by);
            if (k0 < at.length && mine0 < at.length && (!a.causal || mine0 + NB * 32 - 1 >= k0) && !(one && by == -__builtin_inff())) {
                typedef float f4 __attribute__((ext_vector_type(4)));
                const f4 *st = (const f4 *)(stats + turn * 3 * BQ + half_of * 32) + (lane >> 5);       // a lane's rows are four next to each other at a time
                const bool edge = mine0 + NB * 32 > at.length || k0 + 32 > at.length || (a.causal && mine0 < k0 + 31);
                const bool plain = one && !edge && fabsf(by) < kLarge && !large;
                const uint32_t stream = (at.worker * a.seqs + at.seq) * a.heads + head;
                const float *biases = one ? nullptr : bias.at(a, wave, lo, (int)key - (int)mine0);        // of the first query
#pragma unroll 1
                for (int j = 0; j < NB; ++j) {
                    f32x16 s, dp;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.f;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) s = product<T>(rows.read(0, 0, c), kf[c], s);
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) dp = product<T>(rows.read(2 * Ti::BYTES, 0, c), vf[c], dp);
                    if constexpr (T != SAMS_F32) in_order<D / 8, D / 8, kAhead>();
                    // the queries' statistics, read here where there are registers for them (8,192 tokens of 128 columns: 1.10 -> 0.99 ms; where two wavefronts share
                    // a SIMD, 100 -> 106 us with 64 columns, 63 -> 84 with 72)
                    constexpr bool EARLY = T != SAMS_F32 && kWavesPerSimd<T, D> == 1;
                    auto four_of = [&](int which, int i) { return st[(which * BQ + 32 * j) / 4 + 2 * (i >> 2)]; };
                    f4 early[EARLY ? 3 : 1][4];
                    if constexpr (EARLY) {
#pragma unroll
                        for (int w = 0; w < 3; ++w)
#pragma unroll
                            for (int i = 0; i < 4; ++i) early[w][i] = four_of(w, 4 * i);
                        all_under_way();
                    }
                    auto stat_of = [&](int which, int i) {
                        if constexpr (EARLY) return early[which][i >> 2][i & 3];
                        else return four_of(which, i)[i & 3];
                    };
                    if (plain) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], scale, by - stat_of(0, i));
                    } else {
                        if (one) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], scale, by) - stat_of(0, i);
                        } else {
                            float b[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) b[i] = biases[-(32 * j + row_of(i, lane))];
                            all_under_way();
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], scale, b[i]) - stat_of(0, i);
                        }
                        if (edge) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const uint32_t query = mine0 + 32 * j + row_of(i, lane);
                                s[i] = live && query < at.length && (!a.causal || query >= key) ? s[i] : -__builtin_inff();
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i]) * stat_of(1, i);
                    f32x16 pd = s;
                    if constexpr (DROP) {
                        // A generator's call is for one query and eight keys: every lane makes two of the 128 calls for its query, and takes what
                        // is its key's from all of them.
                        char *mine = numbers_lds + wave * 32 * NUMBERS;
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            uint32_t numbers[4];
                            philox(seed, ((k0 + 16 * half) >> 4) * 2 + (lane >> 5), mine0 + 32 * j + (lane & 31), stream, numbers);
                            *(u32x4 *)(mine + (lane & 31) * NUMBERS + (half * 2 + (lane >> 5)) * 16) = u32x4{numbers[0], numbers[1], numbers[2], numbers[3]};
                        }
                        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                        __builtin_amdgcn_wave_barrier();
                        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                        const int c = lane & 31;
                        const char *from = mine + ((c >> 4) * 2 + ((c >> 2) & 1)) * 16 + (((c >> 3) & 1) * 4 + (c & 3)) * 2;
                        uint32_t number[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) number[i] = *(const uint16_t *)(from + row_of(i, lane) * NUMBERS);
                        all_under_way();
#pragma unroll
                        for (int i = 0; i < 16; ++i) pd[i] = number[i] >= a.keep.least ? s[i] : 0.f;
                        __builtin_amdgcn_wave_barrier();
                    }
                    // dS = m P dP - P delta, without the factor 1 / (1 - p), which delta has not either
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float delta = stat_of(2, i);
                        s[i] = DROP ? __builtin_fmaf(pd[i], dp[i], -(s[i] * delta)) : s[i] * (dp[i] - delta);
                    }
                    auto add_up = [&]() {
                        if (summed) {
                            if (one) sums.one(bucket, s, lane);
                            else sums.many(a, bias, (int)k0 - (int)(mine0 + 32 * j), s, lane);
                        }
                    };
                    // 16-bit floats: before they are scaled. 32-bit ones: behind the products stood a branch, and where it was
                    // taken the compiler read the last product's last register after 13 of the 18 wait states that a
                    // 32x32x2 product needs (dk wrong in that register's columns); in front, every such read has its 18
                    // (tests/test_isa_product_waits.py follows every path of the library's code).
                    if constexpr (T != SAMS_BF16) add_up();
                    fit.fit(s, dk);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const typename Ti::Frag wp = words_of<T>(pd, half), ws = words_of<T>(s, half);
#pragma unroll
                        for (int d = 0; d < D / 32; ++d) dv[d] = product<T>(columns.read(2 * Ti::BYTES, 16 * half, d), wp, dv[d]);
#pragma unroll
                        for (int d = 0; d < D / 32; ++d) dk[d] = product<T>(columns.read(0, 16 * half, d), ws, dk[d]);
                    }
                    if constexpr (T != SAMS_F32) in_order<D / 4, D / 8, 2 * kAhead>();
                    if constexpr (T == SAMS_BF16) add_up();         // while the matrix cores are at it
                    if constexpr (NB == 2) {
                        rows.move(32 * Ti::LD);
                        columns.move(32 * Ti::LD);
                    }
                }
            }
            if (next_head != head && a.buckets) {
                if (summed) sums.flush(lane);
                __syncthreads();
                if (summed) leave(head, true);
                if (more) {
                    bias.bring(a, next_head);
                    if (summed) {
                        __syncthreads();
                        clear();
                    }
                }
            }
            if (!more) break;
            store(next_query0, turn ^ 1);
            rows.move(Ti::BYTES);
            columns.move(Ti::BYTES);
            __syncthreads();
            head = next_head;
            query0 = next_query0;
        }
    }
    if constexpr (SPLIT == 2) {
        // the odd wavefronts' results, which their neighbours add to their own; tiles are done with
        float *there = (float *)lds + wave / 2 * (D * 64);
        __syncthreads();
        if (half_of) {
            float v[D];
#pragma unroll
            for (int i = 0; i < D / 2; ++i) { v[i] = dk[i / 16][i % 16] * (1.f / fit.by); v[D / 2 + i] = dv[i / 16][i % 16]; }
            give<D>(there, v, lane);
        }
        __syncthreads();
        if (half_of) return;
#pragma unroll
        for (int i = 0; i < D / 2; ++i) {
            dk[i / 16][i % 16] = __builtin_fmaf(dk[i / 16][i % 16], 1.f / fit.by, there[i * 64 + lane]);
            dv[i / 16][i % 16] += there[(D / 2 + i) * 64 + lane];
        }
        fit.by = 1.f;
    }
    if (!live) {
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.f;
    }
    const float by_k = a.scale * a.keep.scale / (fit.by * SHIFT), by_v = a.keep.scale / SHIFT;
    if (pieces == 1) {
        store_columns<T, D>(rows_of<T>(a.dk, a.dks, a, at, at.head) + (int64_t)key * a.dks.row, row_there, a.dim, dk, by_k, lane);
        store_columns<T, D>(rows_of<T>(a.dv, a.dvs, a, at, at.head) + (int64_t)key * a.dvs.row, row_there, a.dim, dv, by_v, lane);
    } else {
        const int64_t narrow = (int64_t)a.kv_heads * a.dim;
        const int64_t from = (((int64_t)piece * a.n + at.worker) * a.t + (int64_t)at.seq * a.len + key) * narrow + (int64_t)at.head * a.dim;
        store_columns<SAMS_F32, D>(a.dk_parts + from, row_there, a.dim, dk, by_k, lane);
        store_columns<SAMS_F32, D>(a.dv_parts + from, row_there, a.dim, dv, by_v, lane);
    }
}

// dk and dv from the workgroups' parts, which are added up in order
template <int T>
__global__ void __launch_bounds__(256) k_attn_join(Args a, uint32_t pieces, uint32_t first)
{
    typedef typename TypeOf<T>::type E;
    const uint32_t narrow = a.kv_heads * a.dim, fours = (narrow + 3) / 4;
    const uint64_t id = (uint64_t)(first + blockIdx.x) * 256 + threadIdx.x, row = id / fours;
    if (row >= a.n * (uint64_t)a.t) return;
    const uint32_t at = (uint32_t)(id - row * fours) * 4;
    const uint64_t worker = row / (uint64_t)a.t, token = row - worker * (uint64_t)a.t;
    const int64_t apart = (int64_t)a.n * a.t * narrow;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const float *p = (which ? a.dv_parts : a.dk_parts) + row * narrow;
        const Rows r = which ? a.dvs : a.dks;
        E *to = (E *)(which ? a.dv : a.dk) + worker * r.worker + token * r.row;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        for (uint32_t i = 0; i < pieces; ++i) {
            uint32_t raw[4] = {0, 0, 0, 0};
            load_piece<SAMS_F32>(p + i * apart, at, narrow, raw);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += __builtin_bit_cast(float, raw[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < narrow) to[at + e] = (E)v[e];
    }
}

// dbias of a worker's head: its parts added up, four threads a bucket, each its quarter of the parts in order
__global__ void __launch_bounds__(256) k_attn_dbias(const float *part, int64_t parts, uint32_t count, uint32_t heads, uint32_t buckets, float scale, float *dbias, int64_t dbias_worker, int accumulate)
{
    __shared__ float sums[4][64];
    const uint32_t lane = threadIdx.x & 63, q = threadIdx.x >> 6, b = blockIdx.y * 64 + lane;
    const uint32_t lo = (uint32_t)((uint64_t)count * q / 4), hi = (uint32_t)((uint64_t)count * (q + 1) / 4);
    float v = 0.f;
    if (b < buckets) {
        const float *p = part + (int64_t)blockIdx.x * parts * buckets + b;
        for (uint32_t i = lo; i < hi; ++i) v += p[(int64_t)i * buckets];
    }
    sums[q][lane] = v;
    __syncthreads();
    if (q || b >= buckets) return;
    v = ((sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane])) * scale;
    float *o = dbias + blockIdx.x / heads * dbias_worker + (int64_t)(blockIdx.x % heads) * buckets + b;
    *o = accumulate ? *o + v : v;
}

hipError_t prepare_backward(int type, uint32_t dim)
{
    hipError_t e = hipSuccess;
    auto allow = [&](const void *f) {
        if (e == hipSuccess) e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
    };
    SAMS_BY_TYPE(type, T, SAMS_BY_WIDTH(dim, D, {
        for (bool halves : {false, true})
            by_split<Tile<T, D>::ROWS>(halves, [&](auto split) {
                constexpr int SPLIT = decltype(split)::value;
                allow((const void *)k_attn_dq<T, D, true, SPLIT>);
                allow((const void *)k_attn_dq<T, D, false, SPLIT>);
                allow((const void *)k_attn_dkv<T, D, true, SPLIT>);
                allow((const void *)k_attn_dkv<T, D, false, SPLIT>);
            });
    }));
    return e;
}

// Workgroups that the keys' kernel is given at least, where cutting its sums into pieces gets it there: two for every CU (8,192 tokens, two heads of keys: 128
// workgroups uncut, 4.9 ms; in pieces for 512 1.13, for 1024 1.12 and 10 us more to join them).
constexpr int64_t kKeyBlocks = 512;
constexpr int kMostPieces = 16;

int64_t sums_room(int32_t n, int64_t t_max, int32_t heads, int32_t kv_heads, int32_t dim)
{
    const int64_t blocks = std::max<int64_t>(1, (int64_t)n * kv_heads * ((t_max + kRows - 1) / kRows));
    const int64_t pieces = std::min<int64_t>(kMostPieces, 2 * ((kKeyBlocks + blocks - 1) / blocks) - 1);       // more than are wanted: heads are cut evenly
    return pieces > 1 ? pieces * n * t_max * kv_heads * dim : 0;
}

// how a group's heads and a head's queries are cut: heads first, whose pieces need nothing more; a piece of queries has 8 tiles at least
static void cut(Args &a, int rows, int64_t parts, int64_t sums)
{
    const int64_t blocks = (int64_t)a.n * a.seqs * a.kv_heads * a.tiles, each = (int64_t)a.n * a.t * a.kv_heads * a.dim;
    const int64_t want = (kKeyBlocks + blocks - 1) / blocks, most = std::min<int64_t>(kMostPieces, sums / each);
    const uint32_t group = a.heads / a.kv_heads;
    a.head_pieces = 1;
    for (uint32_t p = 2; p <= group && p <= most && a.head_pieces < want; ++p)
        if (group % p == 0) a.head_pieces = p;
    const int64_t some = std::min<int64_t>({want / a.head_pieces, most / a.head_pieces, (a.len + rows - 1) / rows / 8, parts / a.tiles});
    a.query_pieces = (uint32_t)std::max<int64_t>(1, some);
}

void launch_backward(const Args &all, int type, int64_t parts, int64_t sums, float *dbias, int64_t dbias_worker, int accumulate, hipStream_t stream)
{
    Args a = all;
    if (!dbias) a.part = nullptr;
    const float scale = a.keep.scale * (type == SAMS_F16 ? 0x1p-14f : 1.f);         // what the parts of dbias were made without
    auto join = [&](uint32_t count, bool add) {
        hipLaunchKernelGGL(k_attn_dbias, dim3(a.n * a.heads, (a.buckets + 63) / 64), dim3(256), 0, stream, a.part, parts, count, a.heads, a.buckets, scale, dbias, dbias_worker, add);
    };
    if (a.len == 0) {
        if (dbias) join(0, accumulate);
        return;
    }
    uint32_t pieces = 1;
    SAMS_BY_TYPE(type, T, SAMS_BY_WIDTH(a.dim, D, {
        constexpr int ROWS = Tile<T, D>::ROWS;
        constexpr int TILES = 4 * Tile<T, D>::BYTES;
        by_split<ROWS>(in_halves((int64_t)a.n * a.seqs * a.heads, a.len), [&](auto split) {
            constexpr int SPLIT = decltype(split)::value;
            a.tiles = tiles_of<SPLIT>(a.len);
            const int bytes = std::max(TILES + Bias::bytes(a), 2 * (D + 1) * 256);
            gemm::in_launches((int64_t)a.n * a.seqs * a.heads * a.tiles, kThreads, [&](dim3 grid, gemm::Launch l) {
                if (a.keep.least) hipLaunchKernelGGL((k_attn_dq<T, D, true, SPLIT>), grid, dim3(kThreads), bytes, stream, a, l);
                else hipLaunchKernelGGL((k_attn_dq<T, D, false, SPLIT>), grid, dim3(kThreads), bytes, stream, a, l);
            });
        });
        by_split<ROWS>(in_halves((int64_t)a.n * a.seqs * a.heads, a.len), [&](auto split) {
            constexpr int SPLIT = decltype(split)::value;
            a.tiles = tiles_of<SPLIT>(a.len);
            cut(a, ROWS, parts, sums);
            pieces = a.head_pieces * a.query_pieces;
            // as many sequences at a time as there is room for their parts of the bias's gradient
            const uint32_t own = a.tiles * a.query_pieces, step = a.buckets ? (uint32_t)std::min<int64_t>(a.seqs, std::max<int64_t>(1, parts / own)) : a.seqs;
            const int bytes = std::max(TILES + 2 * 3 * ROWS * 4 + Bias::bytes(a, true) + (a.keep.least ? kWaves * 32 * 80 : 0) + (int)a.buckets * kWaves * 4, 2 * D * 256);
            if (dbias && a.seqs * own == 1) {                       // nothing to join
                a.part = nullptr;
                a.dbias = dbias; a.dbias_worker = dbias_worker; a.dbias_scale = scale; a.accumulate = accumulate;
            }
            for (uint32_t first = 0; first < all.seqs; first += step) {
                a.seq_first = first;
                a.seq_count = std::min(step, all.seqs - first);
                gemm::in_launches((int64_t)a.n * a.seq_count * a.kv_heads * pieces * a.tiles, kThreads, [&](dim3 grid, gemm::Launch l) {
                    if (a.keep.least) hipLaunchKernelGGL((k_attn_dkv<T, D, true, SPLIT>), grid, dim3(kThreads), bytes, stream, a, l, parts);
                    else hipLaunchKernelGGL((k_attn_dkv<T, D, false, SPLIT>), grid, dim3(kThreads), bytes, stream, a, l, parts);
                });
                if (a.part) join(a.seq_count * own, accumulate || first > 0);
            }
        });
    }));
    if (pieces > 1) {
        const int64_t blocks = ((int64_t)a.n * a.t * ((a.kv_heads * a.dim + 3) / 4) + 255) / 256;
        SAMS_BY_TYPE(type, T, gemm::in_launches(blocks, 256, [&](dim3 grid, gemm::Launch l) {
                         hipLaunchKernelGGL(k_attn_join<T>, grid, dim3(256), 0, stream, a, pieces, l.first);
                     }));
    }
}

}  // namespace attn
}  // namespace sams
