// What the training operators (layer norm, cross entropy of the output layer, orthogonalised updates) have in common: the
// types of their tensors, where a worker's rows lie, scratch memory.
#pragma once
#include "sams_ctx.h"

namespace sams {

// a tensor [n][t][dim] whose last axis is contiguous: distances in elements
struct Rows {
    int64_t worker, row;
};

template <int TYPE> struct TypeOf;
template <> struct TypeOf<SAMS_F32> { typedef float type; };
template <> struct TypeOf<SAMS_BF16> { typedef __bf16 type; };
template <> struct TypeOf<SAMS_F16> { typedef _Float16 type; };

static inline int type_size(int type) { return type == SAMS_F32 ? 4 : 2; }
static inline bool type_ok(int type) { return type == SAMS_F32 || type == SAMS_BF16 || type == SAMS_F16; }
static inline bool aligned_to(const void *p, int bytes) { return ((uintptr_t)p % (unsigned)bytes) == 0; }

// device memory of a context of the training operators, taken when it is created
struct Scratch {
    char *base;
    int64_t bytes;

    int64_t reserve(int64_t size)                    // before take(): offset of a part, 256-byte aligned
    {
        const int64_t at = bytes;
        bytes += (size + 255) / 256 * 256;
        return at;
    }
    int take()
    {
        if (bytes == 0) return SAMS_OK;
        hipError_t e = hipMalloc((void **)&base, (size_t)bytes);
        if (e != hipSuccess) {
            g_last_hip_error = (int)e;
            (void)hipGetLastError();
            base = nullptr;
            bytes = 0;
            return SAMS_ENOMEM;
        }
        return SAMS_OK;
    }
    template <typename T> T *at(int64_t offset) const { return (T *)(base + offset); }
};

// Sum over a wavefront, in every lane: shifted adds within 16 lanes, then across them, without a trip through LDS.
__device__ __forceinline__ float wave_sum(float v)
{
#define SAMS_ADD_DPP(ctrl, rows) \
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl, rows, 0xf, false))
    SAMS_ADD_DPP(0x111, 0xf);       // from 1, 2, 4, 8 lanes below
    SAMS_ADD_DPP(0x112, 0xf);
    SAMS_ADD_DPP(0x114, 0xf);
    SAMS_ADD_DPP(0x118, 0xf);
    SAMS_ADD_DPP(0x142, 0xa);       // lane 15 of the 16 below, into every other 16
    SAMS_ADD_DPP(0x143, 0xc);       // lane 31, into the upper 32
#undef SAMS_ADD_DPP
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// 16 bytes of a row, wherever it starts
template <int T> constexpr int kPiece = T == SAMS_F32 ? 4 : 8;
typedef uint32_t piece_t __attribute__((ext_vector_type(4), aligned(2)));

template <int T>
__device__ __forceinline__ void load_piece(const typename TypeOf<T>::type *p, int64_t at, int64_t dim, uint32_t (&raw)[4])
{
    constexpr int N = kPiece<T>;
    if (at + N <= dim) {
        const piece_t v = *(const piece_t *)(p + at);
        raw[0] = v[0]; raw[1] = v[1]; raw[2] = v[2]; raw[3] = v[3];
    } else {
        typename TypeOf<T>::type e[N];
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = at + i < dim ? p[at + i] : (typename TypeOf<T>::type)0.f;
        __builtin_memcpy(raw, e, 16);
    }
}

template <int T>
__device__ __forceinline__ void widen(const uint32_t (&raw)[4], float (&v)[kPiece<T>])
{
    typename TypeOf<T>::type e[kPiece<T>];
    __builtin_memcpy(e, raw, 16);
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) v[i] = (float)e[i];
}

template <int T>
__device__ __forceinline__ void store_piece(typename TypeOf<T>::type *p, int64_t at, int64_t dim, const float (&v)[kPiece<T>])
{
    constexpr int N = kPiece<T>;
    typename TypeOf<T>::type e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = (typename TypeOf<T>::type)v[i];
    if (at + N <= dim) {
        piece_t w;
        __builtin_memcpy(&w, e, 16);
        *(piece_t *)(p + at) = w;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (at + i < dim) p[at + i] = e[i];
    }
}

// Eight numbers of a row as 32-bit ones; past the row's end 0.
template <int T>
__device__ __forceinline__ void load8(const typename TypeOf<T>::type *p, int64_t at, int64_t limit, float (&v)[8])
{
    constexpr int N = kPiece<T>;
#pragma unroll
    for (int i = 0; i < 8; i += N) {
        uint32_t raw[4] = {0, 0, 0, 0};
        float part[N];
        if (at + i < limit) load_piece<T>(p, at + i, limit, raw);
        widen<T>(raw, part);
#pragma unroll
        for (int e = 0; e < N; ++e) v[i + e] = part[e];
    }
}

// runs body with the tensors' type as a compile-time constant
#define SAMS_BY_TYPE(type, T, ...)                                      \
    do {                                                                \
        if ((type) == SAMS_F32) { constexpr int T = SAMS_F32; __VA_ARGS__; }        \
        else if ((type) == SAMS_BF16) { constexpr int T = SAMS_BF16; __VA_ARGS__; } \
        else { constexpr int T = SAMS_F16; __VA_ARGS__; }               \
    } while (0)

}  // namespace sams
