// amsim_q8.h -- helpers shared by the 8-bit decoder operators (amsim_norm.hip, amsim_gemm_i8.hip,
// amsim_cache.hip): element types, row loads and stores of any alignment, wave and workgroup
// reductions, and the quantisation rule.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "amsim.h"

namespace amsim_q8 __attribute__((visibility("hidden"))) {

// Magnitudes below this are held as zeros with scale 0: the reciprocal of a smaller scale would
// leave the FP32 range.
constexpr float kTiny = 0x1p-100f;

inline int launch_status() { return hipGetLastError() == hipSuccess ? AMSIM_OK : AMSIM_ERR_HIP; }

inline bool valid_type(int dtype) { return dtype == AMSIM_F32 || dtype == AMSIM_BF16 || dtype == AMSIM_F16; }

// Runs f with a value of the element type that `dtype` names.
template <typename F>
inline int with_type(int dtype, F &&f)
{
    switch (dtype) {
    case AMSIM_F32: return f(float{});
    case AMSIM_BF16: return f(__bf16{});
    default: return f(_Float16{});
    }
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A launch takes fewer than 2^32 threads: calls f(first, count) for runs of the workgroups (of up to 1024 threads).
template <typename F>
inline void in_launches(int64_t groups, F &&f)
{
    constexpr int64_t kMost = int64_t(1) << 21;
    for (int64_t first = 0; first < groups; first += kMost) f(first, unsigned(groups - first < kMost ? groups - first : kMost));
}

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Eight elements of a row from p on, `left` of them inside it (the others read as zero).  The
// copies have the element's alignment only; gfx950 loads and stores wide words at any address.
template <typename T>
__device__ __forceinline__ void load8(const T *p, int64_t left, float (&v)[8])
{
    T t[8];
    if (left >= 8) {
        __builtin_memcpy(t, p, sizeof t);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = e < left ? p[e] : T(0.0f);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = float(t[e]);
}

template <typename T>
__device__ __forceinline__ void store8(T *p, int64_t left, const float (&v)[8])
{
    T t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = T(v[e]);
    if (left >= 8) {
        __builtin_memcpy(p, t, sizeof t);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) p[e] = t[e];
    }
}

// The integer of x at the reciprocal scale inv: rounded to nearest, ties to even.  A NaN gives -127 (the scale beside
// it is a NaN too).
__device__ __forceinline__ int quantised(float x, float inv)
{
    const float q = __builtin_rintf(x * inv);
    return int(__builtin_fminf(__builtin_fmaxf(q, -127.0f), 127.0f));
}

__device__ __forceinline__ void store_q8(int8_t *p, int64_t left, const float (&v)[8], float inv)
{
    int q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = quantised(v[e], inv);
    if (left >= 8) {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e / 4] |= uint32_t(q[e] & 0xFF) << (8 * (e % 4));
        __builtin_memcpy(p, w, sizeof w);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) p[e] = int8_t(q[e]);
    }
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// The larger value; a NaN if either is one.
__device__ __forceinline__ float max_nan(float a, float b) { return a > b || a != a ? a : b; }

__device__ __forceinline__ float wave_max_nan(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max_nan(v, __shfl_xor(v, o));
    return v;
}

// Scale and reciprocal of values up to amax (Inf and NaN give a NaN scale, whose products are NaN).  The reciprocal is
// 127 (1 / amax), as plain FP32 tensor code on a GPU evaluates 127 / amax, a number over a tensor: with the quotient
// rounded once it is another number for every fourth row, and then a value next to the middle between two
// integers goes to the other one, in one of six products of 1000 x 1111 values.  (Past 2^125, 1 / amax would be flushed.)
struct Scale {
    float scale, inv;
};

__device__ __forceinline__ Scale scale_of(float amax)
{
    if (amax < kTiny) return {0.0f, 0.0f};
    if (!(amax < __builtin_inff())) return {__builtin_nanf(""), 0.0f};
    return {amax / 127.0f, amax <= 0x1p125f ? 127.0f * (1.0f / amax) : 127.0f / amax};
}

}  // namespace amsim_q8
