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

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
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

// runs body with the tensors' type as a compile-time constant
#define SAMS_BY_TYPE(type, T, ...)                                      \
    do {                                                                \
        if ((type) == SAMS_F32) { constexpr int T = SAMS_F32; __VA_ARGS__; }        \
        else if ((type) == SAMS_BF16) { constexpr int T = SAMS_BF16; __VA_ARGS__; } \
        else { constexpr int T = SAMS_F16; __VA_ARGS__; }               \
    } while (0)

}  // namespace sams
