// Rows of fp32, fp16 and bf16 elements in pieces of 16 bytes, and kernels chosen by the element type.
#pragma once

#include <hip/hip_runtime.h>
#include <type_traits>

#include "recd.h"

typedef uint32_t recd_u32x4 __attribute__((ext_vector_type(4)));
typedef float recd_f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 recd_f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 recd_bf16x8 __attribute__((ext_vector_type(8)));

template <typename T> struct RecdPiece;
template <> struct RecdPiece<float> {
    using type = recd_f32x4;
};
template <> struct RecdPiece<_Float16> {
    using type = recd_f16x8;
};
template <> struct RecdPiece<__bf16> {
    using type = recd_bf16x8;
};

// The 16 / sizeof(T) elements at p (aligned to 16 bytes) in 32 bits.
template <typename T> __device__ inline void recd_load16(const T *p, float *out)
{
    const typename RecdPiece<T>::type v = *reinterpret_cast<const typename RecdPiece<T>::type *>(p);
    for (unsigned e = 0; e < 16 / sizeof(T); e++)
        out[e] = (float)v[e];
}

// Rounds to the nearest T, ties to even.
template <typename T> __device__ inline void recd_store16(T *p, const float *in)
{
    typename RecdPiece<T>::type v;
    for (unsigned e = 0; e < 16 / sizeof(T); e++)
        v[e] = (T)in[e];
    *reinterpret_cast<typename RecdPiece<T>::type *>(p) = v;
}

// f(T()) with the element type of dt, which the caller has checked.
template <typename F> void recd_with_type(recd_dtype dt, F f)
{
    if (dt == RECD_F32)
        f(float());
    else if (dt == RECD_F16)
        f((_Float16)0);
    else
        f((__bf16)0.0f);
}
