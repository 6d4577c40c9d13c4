// Products of 8-bit integers with a scale for each token and channel.
//
//   q[t][j] = the integer nearest to 127 X[t][j] / m_t (ties to even), m_t = max_j |X[t][j]|, s_t = m_t / 127
//   Y[t][i] = (sum_j q[t][j] A[i][j]) a_i s_t + b_i
//
// Sums are whole numbers in 32 bits and exact (2^14 times 131071 columns is less than 2^31), so they do not depend on their order.
#pragma once
#include "row8.h"

namespace psk {


// Eight elements from column k on, zeros from column `cols` on, of a row that has eight: asked for by row_load and had by row_get.  Where the row ends
// among them, its last eight are loaded and moved.
template <int T>
__device__ __forceinline__ void row_load(Raw8<T> &r, const void *row, int k, int cols)
{
    load_raw<T>(r, static_cast<const typename Bits<T>::type *>(row) + min(k, cols - 8));
}
template <int T>
__device__ __forceinline__ void row_get(const Raw8<T> &r, int k, int cols, float (&v)[8])
{
    widen_raw<T>(r, v);
    if (cols & 7) {
        const int by = k < cols ? max(k + 8 - cols, 0) : 0;
#pragma unroll
        for (int d = 4; d > 0; d /= 2)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = by & d ? (i + d < 8 ? v[(i + d) & 7] : 0.0f) : v[i];
    }
    const bool behind = k >= cols;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = behind ? 0.0f : v[i];
}

// The sizes' bits, which order as the sizes do, infinity and NaN last.
__device__ __forceinline__ unsigned size_bits(float v) { return __builtin_bit_cast(unsigned, v) & 0x7fffffffu; }
constexpr unsigned INFINITE = 0x7f800000u;

// How a token is quantised.  A quotient in 32 bits is off by less than 2^-14, so where it is farther than 2^-10 from the middle between two integers,
// the nearest one is right; nearer, 254 |x| and (2k + 1) m, which 64 bits hold without rounding, are compared.  `up` keeps the reciprocal of a small m finite.
struct Quantiser {
    float m, up, inverse;
    bool none;                                             // only zeros, or something that is not finite: the codes are zeros
    __device__ __forceinline__ Quantiser(unsigned bits)
    {
        m = __builtin_bit_cast(float, bits);
        none = bits == 0 || bits >= INFINITE;
        up = m < 0x1p-100f ? 0x1p100f : 1.0f;
        inverse = none ? 0.0f : 127.0f / (m * up);
    }
    __device__ __forceinline__ float scale() const { return none && m != 0.0f ? __builtin_nanf("") : m / 127.0f; }
    __device__ __forceinline__ int code(float x) const
    {
        if (none) return 0;
        const float q = x * up * inverse, r = rintf(q);
        int c = (int)r;
        if (fabsf(fabsf(q - r) - 0.5f) < 0x1p-10f) {
            const int k = (int)fabsf(q);
            const double d = 254.0 * fabs((double)x) - (double)(2 * k + 1) * (double)m;
            c = k + (d > 0.0 || (d == 0.0 && (k & 1)));
            c = x < 0.0f ? -c : c;
        }
        return c;
    }
};
__device__ __forceinline__ unsigned pack4(const int *c)
{
    return (unsigned)(c[0] & 255) | (unsigned)(c[1] & 255) << 8 | (unsigned)(c[2] & 255) << 16 | (unsigned)c[3] << 24;
}

// Largest of a wave, for every lane; in registers (through LDS each of the six exchanges takes a hundred cycles).
template <int CTRL>
__device__ __forceinline__ unsigned dpp_max(unsigned v) { return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true)); }
__device__ __forceinline__ unsigned wave_max(unsigned v)
{
    v = dpp_max<0xB1>(v);                                  // neighbours, pairs, eights, sixteens
    v = dpp_max<0x4E>(v);
    v = dpp_max<0x141>(v);
    v = dpp_max<0x140>(v);
    auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(a[0], a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(b[0], b[1]);
}

// The first `left` of 16 bytes.
__device__ __forceinline__ v4i first_bytes(v4i v, int left)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int b = min(max(left - 4 * i, 0), 4);
        v[i] = b == 0 ? 0 : v[i] & (int)(0xffffffffu >> (32 - 8 * b));
    }
    return v;
}

// What becomes of a sum.
struct Finish {
    const float *a, *s, *bias;                             // of channels, of tokens, of channels or NULL
    bool aside;                                            // put_result
};
// In every way of a product the same three roundings: of the sum to 24 bits, of its product with the channel's scale, of the fused multiply-add.  To f16 the last
// one is made at once (v_fma_mix*_f16), to bf16 from 32 bits.  (With __builtin_fmaf the compiler puts some conversions to f16 in pairs, and these round to 32 bits
// first: tokens of one tile were then rounded in two ways.)
__device__ __forceinline__ float finish(int sum, float a, float s, float b)
{
#pragma clang fp contract(fast)
    return (float)sum * a * s + b;
}

}  // namespace psk
