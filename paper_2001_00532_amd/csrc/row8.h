// Rows of any of the types by eight elements, at any address.
#pragma once
#include "psk_internal.h"
#include "psk_mfma.h"

namespace psk {

constexpr int I8 = 3;                                      // codes of psk_i8; no psk_type

typedef int8_t v8i8 __attribute__((ext_vector_type(8)));
typedef int8_t v8i8_u __attribute__((ext_vector_type(8), aligned(1)));
typedef unsigned short v8s __attribute__((ext_vector_type(8)));
typedef unsigned short v8s_u __attribute__((ext_vector_type(8), aligned(2)));

template <int T> struct Bits { typedef unsigned short type; };
template <> struct Bits<F32> { typedef float type; };
template <> struct Bits<I8> { typedef int8_t type; };

template <int T>
__device__ __forceinline__ float element(const void *p, int64_t i)
{
    if constexpr (T == F32) return static_cast<const float *>(p)[i];
    else if constexpr (T == I8) return (float)static_cast<const int8_t *>(p)[i];
    else return widen<T>(static_cast<const unsigned short *>(p)[i]);
}

// As they are stored: so many loads are in flight before the first is widened.
template <int T> struct Raw8;
template <> struct Raw8<F32> { v4f a, b; };
template <> struct Raw8<F16> { v8s a; };
template <> struct Raw8<BF16> { v8s a; };
template <> struct Raw8<I8> { v8i8 a; };
template <int T>
__device__ __forceinline__ void load_raw(Raw8<T> &r, const typename Bits<T>::type *p)
{
    if constexpr (T == F32) {
        r.a = *reinterpret_cast<const v4f_e *>(p);
        r.b = *reinterpret_cast<const v4f_e *>(p + 4);
    } else if constexpr (T == I8) {
        r.a = *reinterpret_cast<const v8i8_u *>(p);
    } else {
        r.a = *reinterpret_cast<const v8s_u *>(p);
    }
}
template <int T>
__device__ __forceinline__ void widen_raw(const Raw8<T> &r, float (&v)[8])
{
    if constexpr (T == F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = r.a[i]; v[4 + i] = r.b[i]; }
    } else if constexpr (T == I8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)r.a[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = widen<T>(r.a[i]);
    }
}
template <int T>
__device__ __forceinline__ void store8(typename Bits<T>::type *p, const float (&v)[8])
{
    if constexpr (T == F32) {
        *reinterpret_cast<v4f_e *>(p) = v4f{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<v4f_e *>(p + 4) = v4f{v[4], v[5], v[6], v[7]};
    } else {
        v8s r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = narrow<T>(v[i]);
        *reinterpret_cast<v8s_u *>(p) = r;
    }
}

}  // namespace psk
