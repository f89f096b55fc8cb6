// The counter-based generator that dropout takes its decisions from, so that no mask is ever stored: Philox 4x32 (Salmon, Moraes, Dror,
// Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011), with the 7 rounds that the paper finds enough for every test of its battery.
#pragma once
#include "sams_train.h"

namespace sams {

// What a call's decisions come from: the caller's seed and step, and which 16-bit numbers are kept.
struct Keep {
    uint32_t least;         // an element is kept where its number is at least this (0: all are)
    float scale;            // one over the share that is kept
};

// The share p to drop as a number of 2^-16ths; false: p is no number in [0, 1), or rounds to 1.
static inline bool keep_of(double p, Keep &k)
{
    if (!(p >= 0. && p < 1.)) return false;
    k.least = (uint32_t)(p * 65536. + 0.5);
    if (k.least > 65535) return false;
    k.scale = (float)(65536. / (65536. - k.least));
    return true;
}

struct Seed { uint32_t key0, key1, step; };

__device__ __forceinline__ Seed read_seed(const int64_t *rng)
{
    const uint64_t seed = (uint64_t)rng[0];
    return Seed{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)(uint64_t)rng[1]};
}

__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

// Eight 16-bit numbers, two to a word, the first in its lower half: 14 products of 32 x 32 bits, which take a quarter of the rate of
// other instructions and most of the time; one call serves eight elements.
__device__ __forceinline__ void philox(const Seed &s, uint32_t c0, uint32_t c1, uint32_t c2, uint32_t (&out)[4])
{
    uint32_t c3 = s.step, k0 = s.key0, k1 = s.key1;
#pragma unroll
    for (int round = 0; round < 7; ++round) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = xor3((uint32_t)(b >> 32), c1, k0);
        c1 = (uint32_t)b;
        c2 = xor3((uint32_t)(a >> 32), c3, k1);
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0; out[1] = c1; out[2] = c2; out[3] = c3;
}

// whether element e of eight is kept
__device__ __forceinline__ bool kept(const uint32_t (&numbers)[4], int e, uint32_t least)
{
    return ((e & 1) ? numbers[e >> 1] >> 16 : numbers[e >> 1] & 0xffffu) >= least;
}

// Two 16-bit words, of which those are zero whose numbers are below least; less: least - 1 twice (least > 0).  The difference, which stops
// at 0, taken to 0 or 1, times the word: three instructions for two words, where comparing and selecting each takes four and what parts
// and joins them.  (Written out: the compiler would turn it into the latter.)
__device__ __forceinline__ uint32_t keep_words(uint32_t words, uint32_t numbers, uint32_t less)
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    uint32_t one;
    asm("v_pk_sub_u16 %0, %1, %2 clamp\n\tv_pk_min_u16 %0, %0, 1 op_sel_hi:[1,0]" : "=v"(one) : "v"(numbers), "s"(less));
    return __builtin_bit_cast(uint32_t, (u16x2)(__builtin_bit_cast(u16x2, words) * __builtin_bit_cast(u16x2, one)));
}

}  // namespace sams
