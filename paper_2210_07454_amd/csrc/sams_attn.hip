// Self-attention with a learned bias by buckets of the relative position and dropout of the probabilities, forward pass:
//
//   s_ij = scale q_i . k_j + bias[bucket(j - i)],   P = softmax over the keys j of a row,   o_i = sum_j m_ij / (1 - p) P_ij v_j
//
// one pass over the keys with a running maximum and sum of every row.
#include <new>

#include "sams_attn.h"

namespace sams {
namespace attn {

// A workgroup has 128 queries of a head, a wavefront 32 of them, a lane (and the lane 32 from it) one: the products are made as
// S' = K Q' and O' = V' P', so that a query's logits are a lane's own accumulators, which become the second product's operand as they are.
// Keys and values come by tiles through LDS, the next ones on their way in registers meanwhile.  Every wavefront reads all of them from LDS.
//
// Bound by waiting: within a wavefront loads from LDS, products, maximum, exponentials, second product and barrier follow each other, and one to three
// wavefronts a SIMD do not fill the gaps.  8 workers' 12 heads of 1024 x 64 bf16, causal, with bias and dropout, 46 us (36 without both), 280 TFLOP/s: vector
// instructions issue in 66 % of a SIMD's time (for every number a scale, a maximum, an exponential, which takes four times as long, a sum, half a
// conversion, an eighth of a generator's call), its matrix core is busy in 16 %, and a wavefront waits in 42 % of its time.  8,192 tokens' 16 heads of 128
// columns, 365 us, 750 TFLOP/s: 49, 38 and 40 %.  4 workers' 12 heads of 511 in 32 bits, whose products take eight instructions of twice the
// time each, 41 us: 24, 41 and 29 %.  Three wavefronts a SIMD up to 64 columns (51 -> 46 us; four keep registers in memory: 57).
template <int T, int D, bool DROP, int SPLIT>
__global__ void __launch_bounds__(kThreads, (T == SAMS_F32 ? kWavesPerSimd<T, D> : D <= 64 ? 3 : 2)) k_attn_forward(Args a, gemm::Launch launch)
{
    typedef Tile<T, D> Ti;
    typedef typename TypeOf<T>::type E;
    constexpr int BN = Ti::ROWS, NB = BN / 32 / SPLIT, OWN = kOwn<SPLIT>;
    constexpr float SHIFT = T == SAMS_F16 ? 14.f : 0.f;             // 16-bit floats of up to 2^14: small weights keep their digits
    extern __shared__ __align__(16) char lds[];
    char *tile_k = lds, *tile_v = lds + 2 * Ti::BYTES;
    Bias bias;
    bias.place(a, lds + 4 * Ti::BYTES);

    const int lane = threadIdx.x & 63, wave = uniform_wave();
    const int part = wave % SPLIT;                                 // which of a tile's keys
    const Place at = place_of<OWN>(a, launch, a.heads, a.causal);
    const uint32_t q0 = at.first + wave / SPLIT * 32, query = q0 + (lane & 31);
    const bool row_there = query < a.len, live = query < at.length;
    E *out = rows_of<T>(a.out, a.outs, a, at, at.head) + (int64_t)query * a.outs.row;
    const int64_t stat = stats_of(a, at, at.head) + query;

    f32x16 acc[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
    float top = -__builtin_inff(), sum = 0.f;

    if (at.first < at.length) {
        const uint32_t kv = at.head / (a.heads / a.kv_heads);
        const E *k = rows_of<T>(a.k, a.ks, a, at, kv), *v = rows_of<T>(a.v, a.vs, a, at, kv);
        const uint32_t end = a.causal && at.first + OWN < at.length ? at.first + OWN : at.length;
        Seed seed = {};
        if constexpr (DROP) seed = read_seed(a.rng);
        const uint32_t stream = (at.worker * a.seqs + at.seq) * a.heads + at.head, less = (a.keep.least - 1) * 0x10001u;

        Bring<T, D> bk, bv;
        bk.load(k, a.ks.row, 0, at.length, a.dim);
        bv.load(v, a.vs.row, 0, at.length, a.dim);
        typename Ti::Frag qf[D / 16];
        row_fragments<T, D>(rows_of<T>(a.q, a.qs, a, at, at.head), a.qs.row, query, at.length, a.dim, lane, qf);
        // the scale's sign goes into q (and, in dk's kernel, k), so that the largest product is the largest logit
        const float scale = fabsf(a.scale2);
        if (a.scale2 < 0.f) flip<T, D>(qf);
        bias.bring_starts(a);
        bias.bring(a, at.head);
        bk.store(tile_k, 0, at.length, a.dim);
        bv.store(tile_v, 0, at.length, a.dim);
        typename Ti::Along keys;
        typename Ti::Across values;
        keys.init(lds_address(lds) + part * (32 * Ti::LD), lane);
        values.init(lds_address(lds) + part * (32 * Ti::LD), lane);
        __syncthreads();
        int turn = 0;
        for (uint32_t key0 = 0; key0 < end; key0 += BN, turn ^= 1) {
            const bool more = key0 + BN < end;
            if (more) {
                bk.load(k, a.ks.row, key0 + BN, at.length, a.dim);
                bv.load(v, a.vs.row, key0 + BN, at.length, a.dim);
            }
            const uint32_t mine = key0 + part * 32;                 // the wavefront's first key
            const int lo = (int)mine - (int)(q0 + 31);
            uint32_t bucket;
            float by;
            const bool one = bias.one(a, lo, lo + NB * 32 - 1 + 31, bucket, by);
            if (q0 < at.length && mine < at.length && (!a.causal || mine <= q0 + 31) && !(one && by == -__builtin_inff())) {
                f32x16 s[NB];
#pragma unroll
                for (int j = 0; j < NB; ++j) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[j][i] = 0.f;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) s[j] = product<T>(keys.read(0, 32 * j, c), qf[c], s[j]);
                }
                // logits are times * s + by.  Within a tile of one bucket without a border nothing is done to s for that: the largest one is
                // found, and the exponents are made, from it.  (A large bias, as a mask has, is added first, so that it swallows the rest as it
                // does in any other tile and in the backward pass.)
                float times = scale;
                const bool edge = mine + NB * 32 > at.length || (a.causal && mine + NB * 32 - 1 > q0);
                if (edge || !one || !(fabsf(by) < kLarge)) {
                    add_bias<NB>(one ? nullptr : bias.at(a, wave, lo, lo + 31 - (lane & 31)), one, by, scale, lane, s);
                    times = 1.f;
                    by = 0.f;
                    if (edge) {
                        const int limit = (int)(a.causal && query < at.length ? query + 1 : at.length) - (int)mine;
#pragma unroll
                        for (int j = 0; j < NB; ++j)
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[j][i] = 32 * j + row_of(i, lane) < limit ? s[j][i] : -__builtin_inff();
                    }
                }
                float most = s[0][0];
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int i = 0; i < 16; ++i) most = fmaxf(most, s[j][i]);
                most = fmaxf(__builtin_fmaf(max_halves(most), times, by), top);
                if (__any(most > top)) {
                    const float less = most == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(top - most);
                    sum *= less;
#pragma unroll
                    for (int d = 0; d < D / 32; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[d][i] *= less;
                    top = most;
                }
                const float least = top == -__builtin_inff() ? 0.f : top;
                float from = by - (least - SHIFT);
                // Beside a large logit the shift's digits are lost, and what is taken off here is not what every product is rounded to: the largest logit is
                // taken from rounded ones first.  (Without, biases of -5e7 to -1e8 in all of a row made infinite words of 16-bit floats, from -1e9 on its sum
                // was 2^14 too small, and logits of 2^32 made infinities or zeros of weights of 1 in any type.)
                if (__any(fabsf(least) >= kLarge)) {
#pragma unroll
                    for (int j = 0; j < NB; ++j)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[j][i] = __builtin_fmaf(s[j][i], times, by) - least;
                    times = 1.f;
                    from = SHIFT;
                }
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float part[4];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][8 * half + e], times, from));
                            s[j][8 * half + e] = x;
                            part[e & 3] = e < 4 ? x : part[e & 3] + x;
                        }
                        sum += (part[0] + part[1]) + (part[2] + part[3]);
                        typename Ti::Frag w;
                        if constexpr (DROP) {
                            uint32_t numbers[4];
                            philox(seed, ((mine + 32 * j + 16 * half) >> 4) * 2 + (lane >> 5), query, stream, numbers);
                            w = words_of<T>(s[j], half);
                            if constexpr (T == SAMS_F32) {
#pragma unroll
                                for (int e = 0; e < 8; ++e) w[e] = kept(numbers, e, a.keep.least) ? w[e] : 0.f;
                            } else {
#pragma unroll
                                for (int e = 0; e < 4; ++e) w[e] = keep_words(w[e], numbers[e], less);
                            }
                        } else {
                            w = words_of<T>(s[j], half);
                        }
#pragma unroll
                        for (int d = 0; d < D / 32; ++d) acc[d] = product<T>(values.read(2 * Ti::BYTES, 32 * j + 16 * half, d), w, acc[d]);
                    }
            }
            if (more) {
                bk.store(tile_k + (turn ^ 1) * Ti::BYTES, key0 + BN, at.length, a.dim);
                bv.store(tile_v + (turn ^ 1) * Ti::BYTES, key0 + BN, at.length, a.dim);
            }
            keys.move(Ti::BYTES);
            values.move(Ti::BYTES);
            __syncthreads();
        }
    }
    sum = sum_halves(sum);
    if constexpr (SPLIT == 2) {
        // the odd wavefronts' results, which their neighbours add to their own; tiles are done with
        constexpr int N = D / 2 + 2;
        float *there = (float *)lds + wave / 2 * (N * 64);
        if (part) {
            float v[N];
#pragma unroll
            for (int i = 0; i < D / 2; ++i) v[i] = acc[i / 16][i % 16];
            v[N - 2] = top;
            v[N - 1] = sum;
            give<N>(there, v, lane);
        }
        __syncthreads();
        if (part) return;
        const float other = there[(N - 2) * 64 + lane], most = fmaxf(top, other);
        const float mine = most == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(top - most), theirs = most == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(other - most);
        sum = __builtin_fmaf(sum, mine, there[(N - 1) * 64 + lane] * theirs);
#pragma unroll
        for (int i = 0; i < D / 2; ++i) acc[i / 16][i % 16] = __builtin_fmaf(acc[i / 16][i % 16], mine, there[i * 64 + lane] * theirs);
        top = most;
    }
    const float by = live && sum != 0.f ? a.keep.scale / sum : 0.f;
    if (!live) {
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
    }
    store_columns<T, D>(out, row_there, a.dim, acc, by, lane);
    if (row_there && lane < 32) {
        a.row_max[stat] = live && top != -__builtin_inff() ? top : 0.f;
        a.row_sum[stat] = live ? sum * (T == SAMS_F16 ? 0x1p-14f : 1.f) : 0.f;
    }
}

template <int T, int D>
static int lds_forward(const Args &a)
{
    return std::max(4 * Tile<T, D>::BYTES + Bias::bytes(a), 2 * (D / 2 + 2) * 256);
}

// a context's kernels may take more LDS than a launch gets unasked
hipError_t prepare_forward(int type, uint32_t dim)
{
    hipError_t e = hipSuccess;
    auto allow = [&](const void *f) {
        if (e == hipSuccess) e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
    };
    SAMS_BY_TYPE(type, T, SAMS_BY_WIDTH(dim, D, {
        for (bool halves : {false, true})
            by_split<Tile<T, D>::ROWS>(halves, [&](auto split) {
                constexpr int SPLIT = decltype(split)::value;
                allow((const void *)k_attn_forward<T, D, true, SPLIT>);
                allow((const void *)k_attn_forward<T, D, false, SPLIT>);
            });
    }));
    return e;
}

void launch_forward(const Args &all, int type, hipStream_t stream)
{
    const int64_t heads = (int64_t)all.n * all.seqs * all.heads;
    SAMS_BY_TYPE(type, T, SAMS_BY_WIDTH(all.dim, D, by_split<Tile<T, D>::ROWS>(in_halves(heads, all.len), [&](auto split) {
        constexpr int SPLIT = decltype(split)::value;
        Args a = all;
        a.tiles = tiles_of<SPLIT>(a.len);
        const int bytes = lds_forward<T, D>(a);
        gemm::in_launches(heads * a.tiles, kThreads, [&](dim3 grid, gemm::Launch l) {
            if (a.keep.least) hipLaunchKernelGGL((k_attn_forward<T, D, true, SPLIT>), grid, dim3(kThreads), bytes, stream, a, l);
            else hipLaunchKernelGGL((k_attn_forward<T, D, false, SPLIT>), grid, dim3(kThreads), bytes, stream, a, l);
        });
    })));
}

}  // namespace attn
}  // namespace sams

struct sams_attn {
    int32_t n, heads, kv_heads, dim, buckets, type, train;
    int64_t t_max, parts, sums;
    int32_t edge_lo, edge_hi, table_first, table_count;
    hipStream_t stream;
    sams::Scratch scratch;
    int64_t starts, table, delta, part, dk_parts, dv_parts;
};

using namespace sams;

// what both passes take, checked; false: refused
static bool arguments(sams_attn *c, int64_t t, int64_t seqs, const int32_t *lengths, const void *q, Rows qs, const void *k, Rows ks, const void *v, Rows vs,
                      const float *bias, float scale, int32_t causal, const int64_t *rng, double p, attn::Args &a)
{
    if (!c || t < 0 || t > c->t_max || seqs < 1 || t % seqs || !__builtin_isfinite(scale) || !keep_of(p, a.keep)) return false;
    if ((c->buckets > 0) != (bias != nullptr) || !aligned_to(bias, 4) || !aligned_to(lengths, 4) || !aligned_to(rng, 8) || (a.keep.least && !rng)) return false;
    const int size = type_size(c->type);
    if (t > 0) {
        if (!q || !k || !v || !aligned_to(q, size) || !aligned_to(k, size) || !aligned_to(v, size)) return false;
        if (qs.row < 0 || qs.worker < 0 || ks.row < 0 || ks.worker < 0 || vs.row < 0 || vs.worker < 0) return false;
    }
    a.q = q; a.k = k; a.v = v;
    a.qs = qs; a.ks = ks; a.vs = vs;
    a.bias = bias;
    a.starts = c->scratch.at<int32_t>(c->starts);
    a.lengths = lengths;
    a.rng = rng;
    a.t = t;
    a.n = c->n; a.seqs = (uint32_t)seqs; a.len = (uint32_t)(t / seqs);
    a.heads = c->heads; a.kv_heads = c->kv_heads; a.dim = c->dim; a.buckets = c->buckets;
    a.seq_first = 0;
    a.seq_count = a.seqs;
    a.edge_lo = c->edge_lo; a.edge_hi = c->edge_hi;
    a.table_first = c->table_first; a.table_count = (uint32_t)c->table_count;
    a.table_buckets = c->scratch.at<uint16_t>(c->table);
    a.head_pieces = a.query_pieces = 1;
    a.scale = scale;
    a.scale2 = scale * attn::kLog2e;
    a.causal = causal != 0;
    a.delta = c->scratch.at<float>(c->delta);
    a.part = c->scratch.at<float>(c->part);
    return (int64_t)c->n * seqs * c->heads * attn::tiles_of<1>(a.len) < (int64_t)1 << 31;
}

extern "C" {

int sams_attn_create(sams_attn **out, int32_t n, int64_t t_max, int32_t heads, int32_t kv_heads, int32_t dim, int32_t buckets, const int32_t *starts_host,
                     int32_t type, int32_t train, void *hip_stream)
{
    if (!out) return SAMS_EINVAL;
    *out = nullptr;
    if (n < 1 || n > kMaxWorkers || t_max < 0 || t_max > SAMS_MAX_TOKENS / n || heads < 1 || heads > SAMS_MAX_HEADS || kv_heads < 1 || heads % kv_heads || dim < 8 ||
        dim > SAMS_MAX_HEAD_DIM || buckets < 0 || buckets > SAMS_MAX_BUCKETS || (buckets > 0 && !starts_host) || !type_ok(type)) return SAMS_EINVAL;
    for (int b = 1; b < buckets; ++b)
        if (starts_host[b] <= starts_host[b - 1]) return SAMS_EINVAL;
    sams_attn *c = new (std::nothrow) sams_attn();
    if (!c) return SAMS_ENOMEM;
    c->n = n; c->t_max = t_max; c->heads = heads; c->kv_heads = kv_heads; c->dim = dim; c->buckets = buckets; c->type = type; c->train = train != 0;
    c->stream = (hipStream_t)hip_stream;
    c->parts = (t_max + 31) / 32 + 64;
    c->starts = c->scratch.reserve((int64_t)buckets * 4);
    if (buckets > 1) {
        c->edge_lo = starts_host[1];
        c->edge_hi = starts_host[buckets - 1];
        const int64_t count = (int64_t)c->edge_hi - c->edge_lo + 2 * attn::kReach + 1;
        if (count <= attn::kMaxTable && c->edge_lo > INT32_MIN + attn::kReach) {
            c->table_first = c->edge_lo - attn::kReach;
            c->table_count = (int32_t)count;
        }
    }
    c->table = c->scratch.reserve((int64_t)c->table_count * 2);
    if (train) {
        c->sums = attn::sums_room(n, t_max, heads, kv_heads, dim);
        c->dk_parts = c->scratch.reserve(c->sums * 4);
        c->dv_parts = c->scratch.reserve(c->sums * 4);
        c->delta = c->scratch.reserve((int64_t)n * heads * t_max * 4);
        c->part = c->scratch.reserve((int64_t)n * heads * c->parts * buckets * 4);
    }
    int rc = c->scratch.take();
    if (rc == SAMS_OK) {
        hipError_t e = attn::prepare_forward(type, (uint32_t)dim);
        if (e == hipSuccess && train) e = attn::prepare_backward(type, (uint32_t)dim);
        if (e == hipSuccess && buckets) e = hipMemcpyAsync(c->scratch.base + c->starts, starts_host, (size_t)buckets * 4, hipMemcpyHostToDevice, c->stream);
        uint16_t table[attn::kMaxTable];                            // the distances' buckets, one after the other
        for (int32_t i = 0, b = 0; i < c->table_count; ++i) {
            while (b + 1 < buckets && starts_host[b + 1] <= c->table_first + i) ++b;
            table[i] = (uint16_t)b;
        }
        if (e == hipSuccess && c->table_count) e = hipMemcpyAsync(c->scratch.base + c->table, table, (size_t)c->table_count * 2, hipMemcpyHostToDevice, c->stream);
        if (e == hipSuccess && buckets) e = hipStreamSynchronize(c->stream);
        if (e != hipSuccess) {
            g_last_hip_error = (int)e;
            (void)hipGetLastError();
            if (c->scratch.base) (void)hipFree(c->scratch.base);
            rc = SAMS_EHIP;
        }
    }
    if (rc != SAMS_OK) { delete c; return rc; }
    *out = c;
    return SAMS_OK;
}

int sams_attn_destroy(sams_attn *c)
{
    if (!c) return SAMS_OK;
    hipError_t e = hipStreamSynchronize(c->stream);
    if (c->scratch.base) (void)hipFree(c->scratch.base);
    delete c;
    if (e != hipSuccess) { g_last_hip_error = (int)e; return SAMS_EHIP; }
    return SAMS_OK;
}

int64_t sams_attn_scratch_bytes(const sams_attn *c) { return c ? c->scratch.bytes : 0; }

int attention_forward(sams_attn *c, int64_t t, int64_t seqs, const int32_t *lengths, const void *q, int64_t q_worker, int64_t q_row, const void *k,
                      int64_t k_worker, int64_t k_row, const void *v, int64_t v_worker, int64_t v_row, const float *bias, float scale,
                      int32_t causal, const int64_t *rng, double p, void *o, int64_t o_worker, int64_t o_row, float *row_max, float *row_sum)
{
    attn::Args a = {};
    if (!arguments(c, t, seqs, lengths, q, Rows{q_worker, q_row}, k, Rows{k_worker, k_row}, v, Rows{v_worker, v_row}, bias, scale, causal, rng, p, a)) return SAMS_EINVAL;
    if (t == 0) return SAMS_OK;
    const int64_t wide = (int64_t)c->heads * c->dim;
    if (!o || !aligned_to(o, type_size(c->type)) || !row_max || !row_sum || !aligned_to(row_max, 4) || !aligned_to(row_sum, 4)) return SAMS_EINVAL;
    if ((t > 1 && o_row < wide) || (c->n > 1 && o_worker < wide)) return SAMS_EINVAL;
    a.out = o;
    a.outs = Rows{o_worker, o_row};
    a.row_max = row_max;
    a.row_sum = row_sum;
    attn::launch_forward(a, c->type, c->stream);
    SAMS_HIP(hipGetLastError());
    return SAMS_OK;
}

int attention_backward(sams_attn *c, int64_t t, int64_t seqs, const int32_t *lengths, const void *dout, int64_t dout_worker, int64_t dout_row, const void *q,
                       int64_t q_worker, int64_t q_row, const void *k, int64_t k_worker, int64_t k_row, const void *v, int64_t v_worker, int64_t v_row,
                       const float *bias, float scale, int32_t causal, const int64_t *rng, double p, const void *o, int64_t o_worker, int64_t o_row,
                       const float *row_max, const float *row_sum, void *dq, int64_t dq_worker, int64_t dq_row, void *dk, int64_t dk_worker,
                       int64_t dk_row, void *dv, int64_t dv_worker, int64_t dv_row, float *dbias, int64_t dbias_worker, int32_t accumulate)
{
    attn::Args a = {};
    if (!arguments(c, t, seqs, lengths, q, Rows{q_worker, q_row}, k, Rows{k_worker, k_row}, v, Rows{v_worker, v_row}, bias, scale, causal, rng, p, a)) return SAMS_EINVAL;
    if (!c->train || (dbias && (!c->buckets || !aligned_to(dbias, 4)))) return SAMS_EINVAL;
    const int64_t wide = (int64_t)c->heads * c->dim, narrow = (int64_t)c->kv_heads * c->dim;
    const int size = type_size(c->type);
    if (dbias && c->n > 1 && dbias_worker < (int64_t)c->heads * c->buckets) return SAMS_EINVAL;
    if (t > 0) {
        if (!dout || !o || !row_max || !row_sum || !dq || !dk || !dv) return SAMS_EINVAL;
        if (!aligned_to(dout, size) || !aligned_to(o, size) || !aligned_to(dq, size) || !aligned_to(dk, size) || !aligned_to(dv, size) || !aligned_to(row_max, 4) || !aligned_to(row_sum, 4)) return SAMS_EINVAL;
        if (dout_row < 0 || dout_worker < 0 || o_row < 0 || o_worker < 0) return SAMS_EINVAL;
        if (t > 1 && (dq_row < wide || dk_row < narrow || dv_row < narrow)) return SAMS_EINVAL;
        if (c->n > 1 && (dq_worker < wide || dk_worker < narrow || dv_worker < narrow)) return SAMS_EINVAL;
    }
    a.dout = dout; a.douts = Rows{dout_worker, dout_row};
    a.o = o; a.os = Rows{o_worker, o_row};
    a.row_max = (float *)row_max;
    a.row_sum = (float *)row_sum;
    a.dq = dq; a.dqs = Rows{dq_worker, dq_row};
    a.dk = dk; a.dks = Rows{dk_worker, dk_row};
    a.dv = dv; a.dvs = Rows{dv_worker, dv_row};
    a.dk_parts = c->scratch.at<float>(c->dk_parts);
    a.dv_parts = c->scratch.at<float>(c->dv_parts);
    attn::launch_backward(a, c->type, c->parts, c->sums, dbias, dbias_worker, accumulate, c->stream);
    SAMS_HIP(hipGetLastError());
    return SAMS_OK;
}

}  // extern "C"
