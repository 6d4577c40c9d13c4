// Rows of any of the types by eight or four elements, at any address.
#pragma once
#include "psk_internal.h"
#include "psk_mfma.h"

namespace psk {

constexpr int I8 = 3;                                      // codes of psk_i8; no psk_type

typedef int8_t v8i8 __attribute__((ext_vector_type(8)));
typedef int8_t v8i8_u __attribute__((ext_vector_type(8), aligned(1)));
typedef int8_t v4i8 __attribute__((ext_vector_type(4)));
typedef int8_t v4i8_u __attribute__((ext_vector_type(4), aligned(1)));
typedef unsigned short v4s __attribute__((ext_vector_type(4)));
typedef unsigned short v4s_u __attribute__((ext_vector_type(4), aligned(2)));
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
// A result, past the caches if it is one that leaves them anyway.  (The empty statements keep the compiler from making one store of the two, which then goes
// to them.  A template over the type would lose the pointer's alignment.)
#define PSK_PUT_RESULT(V) \
    __device__ __forceinline__ void put_result(V *p, V v, bool aside) \
    { \
        if (aside) { \
            asm volatile(""); \
            __builtin_nontemporal_store(v, p); \
            asm volatile(""); \
        } else { \
            *p = v; \
        } \
    }
PSK_PUT_RESULT(v4f_e)
PSK_PUT_RESULT(v4u_u)
PSK_PUT_RESULT(v4s_u)
PSK_PUT_RESULT(v8s_u)
#undef PSK_PUT_RESULT
constexpr int64_t ASIDE = 32 << 20;                        // bytes of a result from which on it goes past them
template <int T>                                           // 16 bits
__device__ __forceinline__ void store_row(typename Bits<T>::type *p, const float (&v)[8], bool aside)
{
    v8s r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = narrow<T>(v[i]);
    put_result(reinterpret_cast<v8s_u *>(p), r, aside);
}

// Four elements: of 32 bits a wave's load or store is then one piece of 1 KB, where eight to a lane would be two with gaps.
template <int T> struct Raw4;
template <> struct Raw4<F32> { v4f a; };
template <> struct Raw4<F16> { v4s a; };
template <> struct Raw4<BF16> { v4s a; };
template <> struct Raw4<I8> { v4i8 a; };
template <int T>
__device__ __forceinline__ void load_raw(Raw4<T> &r, const typename Bits<T>::type *p)
{
    if constexpr (T == F32) r.a = *reinterpret_cast<const v4f_e *>(p);
    else if constexpr (T == I8) r.a = *reinterpret_cast<const v4i8_u *>(p);
    else r.a = *reinterpret_cast<const v4s_u *>(p);
}
template <int T>
__device__ __forceinline__ void widen_raw(const Raw4<T> &r, float (&v)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (T == F32) v[i] = r.a[i];
        else if constexpr (T == I8) v[i] = (float)r.a[i];
        else v[i] = widen<T>(r.a[i]);
    }
}
template <int T>
__device__ __forceinline__ void store_row(typename Bits<T>::type *p, const float (&v)[4], bool aside)
{
    if constexpr (T == F32) put_result(reinterpret_cast<v4f_e *>(p), v4f{v[0], v[1], v[2], v[3]}, aside);
    else put_result(reinterpret_cast<v4s_u *>(p), v4s{narrow<T>(v[0]), narrow<T>(v[1]), narrow<T>(v[2]), narrow<T>(v[3])}, aside);
}
template <int T, int W> struct RawOf { typedef Raw8<T> type; };
template <int T> struct RawOf<T, 4> { typedef Raw4<T> type; };

// Columns of a row go by W; the last W are the row's last, so some of them may be among those before too (`skip` of them).
struct Unit { int col, skip; };
template <int W>
__device__ __forceinline__ Unit unit_of(int unit, int dim)
{
    const int at = W * unit, col = min(at, dim - W);
    return Unit{col, at - col};
}

}  // namespace psk
