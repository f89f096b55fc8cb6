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
            most = fmaxf(most, other_half(most));
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

// Sums of dS by bucket.  A tile of one bucket adds to a lane's own number, which is joined when the bucket changes; in other tiles the 32 x 32 numbers
// of a wavefront are first added up along their diagonals: rotated by their row, a lane's numbers all belong to one of two distances.
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
    // by[x]: the bucket of the distance x - 32 from that of the block's corner, x = 1 .. 63
    __device__ __forceinline__ void many(const uint16_t *by, const f32x16 &ds, int lane)
    {
        float up = 0.f, down = 0.f;             // distances lane % 32 and lane % 32 - 32
        const int half = lane & 32;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = row_of(i, lane);
            const float v = __shfl(ds[i], ((r + lane) & 31) | half);
            if ((lane & 31) + r < 32) up += v;
            else down += v;
        }
        up += other_half(up);
        down += other_half(down);
        float v = half ? up : down;             // the distance lane - 32
        const int mine = by[lane ? lane : 1];
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
// sum is done, is put right at the end: dq = scale (sum P (dP - d) k + (d - delta) sum P k), with d = do . o.
template <int T, int D, bool DROP>
__global__ void __launch_bounds__(kThreads) k_attn_dq(Args a, gemm::Launch launch)
{
    typedef Tile<T, D> Ti;
    typedef typename TypeOf<T>::type E;
    constexpr int BN = Ti::ROWS, NB = BN / 32;
    constexpr float SHIFT = T == SAMS_F16 ? 0x1p14f : 1.f;          // P in 16-bit floats
    extern __shared__ __align__(16) char lds[];
    char *tile_k = lds, *tile_v = lds + 2 * Ti::BYTES;
    Window *window = (Window *)(lds + 4 * Ti::BYTES);
    int *starts_lds = (int *)(window + 2);

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Place at = place_of(a, launch, a.heads, a.causal);
    const uint32_t q0 = at.first + wave * 32, query = q0 + (lane & 31);
    const bool row_there = query < a.len, live = query < at.length;
    const int64_t stat = stats_of(a, at, at.head) + query;

    constexpr bool ROUNDED = T != SAMS_F32;
    f32x16 acc[D / 32], pk[ROUNDED ? D / 32 : 1];
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = pk[ROUNDED ? d : 0][i] = 0.f;
    ColumnScale<T, D> fit;
    fit.start();

    if (at.first < at.length) {
        for (uint32_t b = threadIdx.x; b < a.buckets; b += kThreads) starts_lds[b] = a.starts[b];
        const Starts starts = {starts_lds, a.buckets};
        const float *bias = a.bias + (int64_t)at.head * a.buckets;
        const uint32_t kv = at.head / (a.heads / a.kv_heads);
        const E *k = rows_of<T>(a.k, a.ks, a, at, kv), *v = rows_of<T>(a.v, a.vs, a, at, kv);
        const uint32_t end = a.causal && at.first + kRows < at.length ? at.first + kRows : at.length;
        Seed seed = {};
        if constexpr (DROP) seed = read_seed(a.rng);
        const uint32_t stream = (at.worker * a.seqs + at.seq) * a.heads + at.head;

        typename Ti::Frag qf[D / 16], df[D / 16];
        row_fragments<T, D>(rows_of<T>(a.q, a.qs, a, at, at.head) + (int64_t)query * a.qs.row, live, a.dim, lane, qf);
        row_fragments<T, D>(rows_of<T>(a.dout, a.douts, a, at, at.head) + (int64_t)query * a.douts.row, live, a.dim, lane, df);
        float delta = 0.f;
        {
            const E *o = rows_of<T>(a.o, a.os, a, at, at.head) + (int64_t)query * a.os.row;
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                float x[8], y[8];
                const uint32_t from = 16 * s + 8 * (lane >> 5);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = 0.f;
                if (live) load8<T>(o, from, a.dim, x);
                typename TypeOf<T>::type e[8];
                __builtin_memcpy(e, &df[s], sizeof(e));
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = (float)e[i];
#pragma unroll
                for (int i = 0; i < 8; ++i) delta = __builtin_fmaf(x[i], y[i], delta);
            }
            delta += other_half(delta);
        }
        const float top = live ? a.row_max[stat] : 0.f, total = live ? a.row_sum[stat] : 0.f;
        const float over = total == 0.f ? 0.f : SHIFT / total;
        float exact = 0.f;

        Bring<T, D> bk, bv;
        bk.load(k, a.ks.row, 0, at.length, a.dim);
        bv.load(v, a.vs.row, 0, at.length, a.dim);
        __syncthreads();
        bk.store(tile_k);
        bv.store(tile_v);
        const int lo = -(int)(at.first + kRows - 1);
        Band band = band_of(starts, bias, lo, BN + kRows - 1, window[0]);
        __syncthreads();
        int turn = 0;
        for (uint32_t key0 = 0; key0 < end; key0 += BN, turn ^= 1) {
            const bool more = key0 + BN < end;
            if (more) {
                bk.load(k, a.ks.row, key0 + BN, at.length, a.dim);
                bv.load(v, a.vs.row, key0 + BN, at.length, a.dim);
            }
            const bool needed = q0 < at.length && (!a.causal || key0 <= q0 + 31) && !(band.one && band.value == -__builtin_inff());
            if (needed) {
                const char *tk = tile_k + turn * Ti::BYTES, *tv = tile_v + turn * Ti::BYTES;
                const bool edge = key0 + BN > at.length || q0 + 32 > at.length || (a.causal && key0 + BN - 1 > q0);
                const int limit = (live ? (int)(a.causal ? query + 1 : at.length) : 0) - (int)key0;
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    f32x16 s, dp;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.f;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) s = product<T>(Ti::along(tk, 32 * j, c, lane), qf[c], s);
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) dp = product<T>(Ti::along(tv, 32 * j, c, lane), df[c], dp);
                    if (band.one) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], a.scale2, band.value);
                    } else {
                        const float *by = window[turn].value + (kRows - 1 - (int)(query - at.first)) + 32 * j;
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], a.scale2, by[row_of(i, lane)]);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] - top) * over;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        if constexpr (DROP) {
                            uint32_t numbers[4];
                            philox(seed, ((key0 + 32 * j + 16 * half) >> 4) * 2 + (lane >> 5), query, stream, numbers);
#pragma unroll
                            for (int e = 0; e < 8; ++e) dp[8 * half + e] = kept(numbers, e, a.keep.least) ? dp[8 * half + e] * a.keep.scale : 0.f;
                        }
                    }
                    if (edge) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const bool allowed = 32 * j + row_of(i, lane) < limit;
                            s[i] = allowed ? s[i] : 0.f;
                            dp[i] = allowed ? dp[i] : 0.f;
                        }
                    }
                    typename Ti::Frag wp[2];
                    if constexpr (ROUNDED) {
                        wp[0] = words_of<T>(s, 0);
                        wp[1] = words_of<T>(s, 1);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) exact = __builtin_fmaf(s[i], dp[i], exact);
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] *= dp[i] - delta;
                    fit.fit(s, acc);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const typename Ti::Frag w = words_of<T>(s, half);
#pragma unroll
                        for (int d = 0; d < D / 32; ++d) {
                            const typename Ti::Frag columns = Ti::across(tk, 32 * j + 16 * half, 32 * d, lane);
                            acc[d] = product<T>(columns, w, acc[d]);
                            if constexpr (ROUNDED) pk[d] = product<T>(columns, wp[half], pk[d]);
                        }
                    }
                }
            }
            if (more) {
                bk.store(tile_k + (turn ^ 1) * Ti::BYTES);
                bv.store(tile_v + (turn ^ 1) * Ti::BYTES);
                band = band_of(starts, bias, lo + (int)(key0 + BN), BN + kRows - 1, window[turn ^ 1]);
            }
            __syncthreads();
        }
        exact = (exact + other_half(exact)) * (1.f / SHIFT);
        if (live && lane < 32) a.delta[stat] = exact;
        if constexpr (ROUNDED) {
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] = __builtin_fmaf(acc[d][i], 1.f / fit.by, (delta - exact) * pk[d][i]);
        }
    }
    store_columns<T, D>(rows_of<T>(a.dq, a.dqs, a, at, at.head) + (int64_t)query * a.dqs.row, row_there, a.dim, acc, a.scale / SHIFT, lane);
}

// dk, dv and dbias.  A workgroup has 128 keys, a lane (and the lane 32 from it) one; queries and the output's gradients come by tiles.  The
// products are S = Q K' and dP = dO V', whose accumulators become the second operands of dV' = dO' P and dK' = Q' dS as they are.
template <int T, int D, bool DROP>
__global__ void __launch_bounds__(kThreads) k_attn_dkv(Args a, gemm::Launch launch, int64_t parts)
{
    typedef Tile<T, D> Ti;
    constexpr int BQ = Ti::ROWS, NB = BQ / 32;
    constexpr float SHIFT = T == SAMS_F16 ? 0x1p14f : 1.f;          // P in 16-bit floats
    constexpr int NUMBERS = 80;                                     // bytes of a query's numbers: 32 of 16 bits, and 16 that put the queries on different banks
    extern __shared__ __align__(16) char lds[];
    char *tile_q = lds, *tile_d = lds + 2 * Ti::BYTES;
    Window *window = (Window *)(lds + 4 * Ti::BYTES);
    float *stats = (float *)(window + 2);                           // [2][3][BQ]
    char *numbers_lds = (char *)(stats + 2 * 3 * BQ);               // [kWaves][32] queries' numbers
    int *starts_lds = (int *)(numbers_lds + (DROP ? kWaves * 32 * NUMBERS : 0));
    float *sums_lds = (float *)(starts_lds + a.buckets);            // [kWaves][buckets]

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Place at = place_of(a, launch, a.kv_heads, false);
    const uint32_t k0 = at.first + wave * 32, key = k0 + (lane & 31);
    const bool row_there = key < a.len, live = key < at.length;

    f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.f;
    ColumnScale<T, D> fit;
    fit.start();

    const uint32_t group = a.heads / a.kv_heads;
    BucketSums sums = {sums_lds + wave * a.buckets, 0.f, 0};
    const bool summed = a.part != nullptr;
    // a head's sums of the workgroup; between barriers
    auto leave = [&](uint32_t head, bool some) {
        float *part = a.part + (((int64_t)at.worker * a.heads + head) * parts + (int64_t)(at.seq - a.seq_first) * a.tiles + at.first / kRows) * a.buckets;
        for (uint32_t b = threadIdx.x; b < a.buckets; b += kThreads) {
            part[b] = some ? (sums_lds[b] + sums_lds[a.buckets + b]) + (sums_lds[2 * a.buckets + b] + sums_lds[3 * a.buckets + b]) : 0.f;
            for (int w = 0; w < kWaves; ++w) sums_lds[w * a.buckets + b] = 0.f;
        }
    };
    if (at.first >= at.length) {
        for (uint32_t h = 0; summed && h < group; ++h) leave(at.head * group + h, false);
    } else {
        for (uint32_t b = threadIdx.x; b < a.buckets; b += kThreads) {
            starts_lds[b] = a.starts[b];
            for (int w = 0; w < kWaves; ++w) sums_lds[w * a.buckets + b] = 0.f;
        }
        const Starts starts = {starts_lds, a.buckets};
        Seed seed = {};
        if constexpr (DROP) seed = read_seed(a.rng);
        const uint32_t begin = a.causal ? at.first / BQ * BQ : 0;   // 128 is a multiple of BQ: the first key's tile
        typename Ti::Frag kf[D / 16], vf[D / 16];
        row_fragments<T, D>(rows_of<T>(a.k, a.ks, a, at, at.head) + (int64_t)key * a.ks.row, live, a.dim, lane, kf);
        row_fragments<T, D>(rows_of<T>(a.v, a.vs, a, at, at.head) + (int64_t)key * a.vs.row, live, a.dim, lane, vf);

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
        auto store = [&](int turn) {
            bq.store(tile_q + turn * Ti::BYTES);
            bd.store(tile_d + turn * Ti::BYTES);
            if (threadIdx.x < BQ)
#pragma unroll
                for (int i = 0; i < 3; ++i) stats[(turn * 3 + i) * BQ + threadIdx.x] = stat[i];
        };
        // distances of a tile: from at.first - (query0 + BQ - 1) on
        auto band_at = [&](uint32_t head, uint32_t query0, int turn) {
            return band_of(starts, a.bias + (int64_t)head * a.buckets, (int)at.first - (int)(query0 + BQ - 1), BQ + kRows - 1, window[turn]);
        };
        uint32_t head = at.head * group, query0 = begin;
        const uint32_t last = head + group - 1;
        load(head, query0);
        __syncthreads();
        store(0);
        Band band = band_at(head, query0, 0);
        __syncthreads();
        for (int turn = 0;; turn ^= 1) {
            uint32_t next_head = head, next_query0 = query0 + BQ;
            if (next_query0 >= at.length) { ++next_head; next_query0 = begin; }
            const bool more = next_head <= last;
            if (more) load(next_head, next_query0);
            const bool needed = k0 < at.length && (!a.causal || query0 + BQ - 1 >= k0) && !(band.one && band.value == -__builtin_inff());
            if (needed) {
                const char *tq = tile_q + turn * Ti::BYTES, *td = tile_d + turn * Ti::BYTES;
                const float *st = stats + turn * 3 * BQ;
                const bool edge = query0 + BQ > at.length || k0 + 32 > at.length || (a.causal && query0 < k0 + 31);
                const uint32_t stream = (at.worker * a.seqs + at.seq) * a.heads + head;
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    f32x16 s, dp;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.f;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) s = product<T>(Ti::along(tq, 32 * j, c, lane), kf[c], s);
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) dp = product<T>(Ti::along(td, 32 * j, c, lane), vf[c], dp);
                    if (band.one) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], a.scale2, band.value);
                    } else {
                        const float *by = window[turn].value + (int)(key - at.first) + BQ - 1 - 32 * j;
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], a.scale2, by[-row_of(i, lane)]);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int r = 32 * j + row_of(i, lane);
                        s[i] = __builtin_amdgcn_exp2f(s[i] - st[r]) * st[BQ + r];
                    }
                    auto allowed = [&](int i) {
                        const uint32_t query = query0 + 32 * j + row_of(i, lane);
                        return live && query < at.length && (!a.causal || query >= key);
                    };
                    if (edge) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = allowed(i) ? s[i] : 0.f;
                    }
                    f32x16 pd = s;
                    if constexpr (DROP) {
                        // A generator's call is for one query and eight keys: every lane makes two of the 128 calls for its query, and takes what
                        // is its key's from all of them.
                        char *mine = numbers_lds + wave * 32 * NUMBERS;
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            uint32_t numbers[4];
                            philox(seed, ((k0 + 16 * half) >> 4) * 2 + (lane >> 5), query0 + 32 * j + (lane & 31), stream, numbers);
                            *(u32x4 *)(mine + (lane & 31) * NUMBERS + (half * 2 + (lane >> 5)) * 16) = u32x4{numbers[0], numbers[1], numbers[2], numbers[3]};
                        }
                        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                        __builtin_amdgcn_wave_barrier();
                        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                        const int c = lane & 31;
                        const char *from = mine + ((c >> 4) * 2 + ((c >> 2) & 1)) * 16 + (((c >> 3) & 1) * 4 + (c & 3)) * 2;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const bool keep = *(const uint16_t *)(from + row_of(i, lane) * NUMBERS) >= a.keep.least;
                            pd[i] = keep ? s[i] : 0.f;
                            dp[i] = keep ? dp[i] * a.keep.scale : 0.f;
                        }
                        __builtin_amdgcn_wave_barrier();
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] *= dp[i] - st[2 * BQ + 32 * j + row_of(i, lane)];
                    if (edge) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = allowed(i) ? s[i] : 0.f;
                    }
                    if (summed) {
                        if (band.one) sums.one(band.bucket, s, lane);
                        else sums.many(window[turn].bucket + (wave * 32 + BQ - 1 - 32 * j) - 32, s, lane);
                    }
                    fit.fit(s, dk);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const typename Ti::Frag wp = words_of<T>(pd, half), ws = words_of<T>(s, half);
#pragma unroll
                        for (int d = 0; d < D / 32; ++d) dv[d] = product<T>(Ti::across(td, 32 * j + 16 * half, 32 * d, lane), wp, dv[d]);
#pragma unroll
                        for (int d = 0; d < D / 32; ++d) dk[d] = product<T>(Ti::across(tq, 32 * j + 16 * half, 32 * d, lane), ws, dk[d]);
                    }
                }
            }
            if (next_head != head && summed) {
                sums.flush(lane);
                __syncthreads();
                leave(head, true);
            }
            if (!more) break;
            store(turn ^ 1);
            band = band_at(next_head, next_query0, turn ^ 1);
            __syncthreads();
            head = next_head;
            query0 = next_query0;
        }
    }
    if (!live) {
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.f;
    }
    store_columns<T, D>(rows_of<T>(a.dk, a.dks, a, at, at.head) + (int64_t)key * a.dks.row, row_there, a.dim, dk, a.scale / (fit.by * SHIFT), lane);
    store_columns<T, D>(rows_of<T>(a.dv, a.dvs, a, at, at.head) + (int64_t)key * a.dvs.row, row_there, a.dim, dv, a.keep.scale / SHIFT, lane);
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
    SAMS_BY_TYPE(type, T, SAMS_BY_WIDTH(dim, D, {
        for (const void *f : {(const void *)k_attn_dq<T, D, true>, (const void *)k_attn_dq<T, D, false>, (const void *)k_attn_dkv<T, D, true>, (const void *)k_attn_dkv<T, D, false>})
            if (e == hipSuccess) e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
    }));
    return e;
}

void launch_backward(const Args &all, int type, int64_t parts, float *dbias, int64_t dbias_worker, int accumulate, hipStream_t stream)
{
    Args a = all;
    if (!dbias) a.part = nullptr;
    const float scale = type == SAMS_F16 ? 0x1p-14f : 1.f;          // of the parts: P was held larger
    auto join = [&](uint32_t count, bool add) {
        hipLaunchKernelGGL(k_attn_dbias, dim3(a.n * a.heads, (a.buckets + 63) / 64), dim3(256), 0, stream, a.part, parts, count, a.heads, a.buckets, scale, dbias, dbias_worker, add);
    };
    if (a.len == 0) {
        if (dbias) join(0, accumulate);
        return;
    }
    SAMS_BY_TYPE(type, T, SAMS_BY_WIDTH(a.dim, D, {
        const int bytes = 4 * Tile<T, D>::BYTES + 2 * (int)sizeof(Window) + (int)a.buckets * 4;
        gemm::in_launches((int64_t)a.n * a.seqs * a.heads * a.tiles, kThreads, [&](dim3 grid, gemm::Launch l) {
            if (a.keep.least) hipLaunchKernelGGL((k_attn_dq<T, D, true>), grid, dim3(kThreads), bytes, stream, a, l);
            else hipLaunchKernelGGL((k_attn_dq<T, D, false>), grid, dim3(kThreads), bytes, stream, a, l);
        });
    }));
    // as many sequences at a time as there is room for their parts of the bias's gradient
    const uint32_t step = a.buckets ? (uint32_t)std::min<int64_t>(a.seqs, std::max<int64_t>(1, parts / a.tiles)) : a.seqs;
    for (uint32_t first = 0; first < all.seqs; first += step) {
        a.seq_first = first;
        a.seq_count = std::min(step, all.seqs - first);
        SAMS_BY_TYPE(type, T, SAMS_BY_WIDTH(a.dim, D, {
            const int bytes = 4 * Tile<T, D>::BYTES + 2 * (int)sizeof(Window) + 2 * 3 * Tile<T, D>::ROWS * 4 + (int)a.buckets * 4 * (1 + kWaves);
            gemm::in_launches((int64_t)a.n * a.seq_count * a.kv_heads * a.tiles, kThreads, [&](dim3 grid, gemm::Launch l) {
                if (a.keep.least) hipLaunchKernelGGL((k_attn_dkv<T, D, true>), grid, dim3(kThreads), bytes + kWaves * 32 * 80, stream, a, l, parts);
                else hipLaunchKernelGGL((k_attn_dkv<T, D, false>), grid, dim3(kThreads), bytes, stream, a, l, parts);
            });
        }));
        if (dbias) join(a.seq_count * a.tiles, accumulate || first > 0);
    }
}

}  // namespace attn
}  // namespace sams
