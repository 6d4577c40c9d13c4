// Products of dense rows (16-bit or 4-bit weights) with a few vectors on the matrix cores (gfx950, wave64).
//
// One matrix instruction multiplies 16 vectors by 16 rows of weights over 32 columns:
//   D[m][n] += sum_k X[m][k] W[n][k],   lane l holds X and W at row l % 16, columns 8 (l / 16) .. + 7, and D at n = l % 16,
//   m = 4 (l / 16) + i, i = 0 .. 3.
// The weights are the second operand, so a lane dequantises, loads the scale of and sums up the same row n.  Vectors past the
// last one repeat it (their rows of D are not looked at), rows past the last one likewise; only columns need zeros.
// Sums are held in 32 bits.
#pragma once
#include "psk_dev.h"
#include <type_traits>

namespace psk {

typedef __bf16   v8b __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v4u_u __attribute__((ext_vector_type(4), aligned(2)));
typedef float    v4f_e __attribute__((ext_vector_type(4), aligned(4)));

// psk_type
constexpr int F32 = 0, F16 = 1, BF16 = 2;

template <int T>
__device__ __forceinline__ v4f mfma16(v4u x, v4u w, v4f c)
{
    if constexpr (T == F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, x), __builtin_bit_cast(v8h, w), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, x), __builtin_bit_cast(v8b, w), c, 0, 0, 0);
}

template <int T>
__device__ __forceinline__ float widen(unsigned short v)
{
    if constexpr (T == F16) return (float)__builtin_bit_cast(_Float16, v);
    else return __builtin_bit_cast(float, (unsigned)v << 16);
}
template <int T>
__device__ __forceinline__ unsigned short narrow(float v)      // to nearest even
{
    if constexpr (T == F16) return __builtin_bit_cast(unsigned short, (_Float16)v);
    else return __builtin_bit_cast(unsigned short, (__bf16)v);
}
template <int T>
__device__ __forceinline__ void store_as(void *y, int64_t i, float v)
{
    if constexpr (T == F32) static_cast<float *>(y)[i] = v;
    else static_cast<unsigned short *>(y)[i] = narrow<T>(v);
}

// Eight 16-bit elements from column k on, zeros from column `left` on.  (A loop of one load: written out it would cost the kernels
// around it more registers than all the rest.)
__device__ __forceinline__ v4u load8(const unsigned short *p, int k, int left)
{
    if (k + 8 <= left) return *reinterpret_cast<const v4u_u *>(p + k);
    v4u r = {0, 0, 0, 0};
    if (k < left) {
#pragma unroll 1
        for (int i = k + 7; i >= k; --i) {
            const unsigned e = i < left ? p[i] : 0u;
            r = v4u{r[0] << 16 | e, r[1] << 16 | r[0] >> 16, r[2] << 16 | r[1] >> 16, r[3] << 16 | r[2] >> 16};
        }
    }
    return r;
}

// ---- vectors
// Few vectors, up to four: row 4v + j of the first operand is block j (32 columns) of four blocks of vector v, so one load per lane
// brings four blocks.  The instruction that multiplies it by block j of the weights leaves the product of the two in element j
// of the lanes of quarter v (and products of blocks that do not belong together in the other elements).
// Tiles: row m of an operand is vector m of the tile, four loads for four blocks.
// A vector may have several parts whose products add up; P of them, the last one with a factor of its own if LO (see Halves).
template <int T>
struct Plain16 {                                           // 16 bits
    static constexpr int P = 1;
    static constexpr bool LO = false;
    struct Raw { v4u v; };
    const unsigned short *p;
    __device__ __forceinline__ void set(const void *X, int64_t at) { p = static_cast<const unsigned short *>(X) + at; }
    template <bool TAIL>
    __device__ __forceinline__ void load(Raw &r, int k, int left) const { r.v = TAIL ? load8(p, k, left) : *reinterpret_cast<const v4u_u *>(p + k); }
    static __device__ __forceinline__ void operands(const Raw &r, v4u (&x)[P]) { x[0] = r.v; }
};
// 32 bits as three parts of bf16: v = a + b + c with 8 significant bits in each, cut off and not rounded, so the sum is exact and a
// value near the largest does not become infinite.  Infinity and NaN stand in the first part alone.
struct Parts32 {
    static constexpr int P = 3;
    static constexpr bool LO = false;
    struct Raw { v4f_e a, b; };
    const float *p;
    __device__ __forceinline__ void set(const void *X, int64_t at) { p = static_cast<const float *>(X) + at; }
    template <bool TAIL>
    __device__ __forceinline__ void load(Raw &r, int k, int left) const
    {
        if (!TAIL || k + 8 <= left) {
            r.a = *reinterpret_cast<const v4f_e *>(p + k);
            r.b = *reinterpret_cast<const v4f_e *>(p + k + 4);
            return;
        }
        r.a = r.b = v4f_e{0, 0, 0, 0};
        if (k < left) {
#pragma unroll 1
            for (int i = k + 7; i >= k; --i) {
                r.b = v4f_e{r.a[3], r.b[0], r.b[1], r.b[2]};
                r.a = v4f_e{i < left ? p[i] : 0.0f, r.a[0], r.a[1], r.a[2]};
            }
        }
    }
    static __device__ __forceinline__ void operands(const Raw &r, v4u (&x)[P])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unsigned part[2][P];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float v = __builtin_canonicalizef(i < 2 ? r.a[2 * i + e] : r.b[2 * i - 4 + e]);      // a NaN keeps its first bit
                const float a = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, v) & 0xffff0000u), d = v - a;
                const float rest = __builtin_isfinite(v) ? d : 0.0f;
                const float b = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, rest) & 0xffff0000u), c = rest - b;
                part[e][0] = __builtin_bit_cast(unsigned, a);
                part[e][1] = __builtin_bit_cast(unsigned, b);
                part[e][2] = __builtin_bit_cast(unsigned, c);
            }
#pragma unroll
            for (int q = 0; q < P; ++q) x[q][i] = __builtin_amdgcn_perm(part[1][q], part[0][q], 0x07060302u);
        }
    }
};
// Two 16-bit numbers per value, the nearest one and the nearest one to what is left, in two arrays.  f16 has too small a range for
// that: the value is scaled by 2^-8 (up to 2^24 it is finite) and what is left by 2^11, and the second sum is kept apart.
template <int T>
struct Halves {
    static constexpr int P = 2;
    static constexpr bool LO = T == F16;
    static constexpr float scale = T == F16 ? 0x1p-8f : 1.0f, rest = T == F16 ? 0x1p11f : 1.0f;
    struct Raw { v4u v[2]; };
    const unsigned short *p;
    int64_t apart;                                         // from the first array to the second one
    __device__ __forceinline__ void set(const unsigned short *h, int64_t at, int64_t to_rest) { p = h + at; apart = to_rest; }
    template <bool TAIL>
    __device__ __forceinline__ void load(Raw &r, int k, int left) const
    {
        r.v[0] = TAIL ? load8(p, k, left) : *reinterpret_cast<const v4u_u *>(p + k);
        r.v[1] = TAIL ? load8(p + apart, k, left) : *reinterpret_cast<const v4u_u *>(p + apart + k);
    }
    static __device__ __forceinline__ void operands(const Raw &r, v4u (&x)[P]) { x[0] = r.v[0]; x[1] = r.v[1]; }
    static __device__ __forceinline__ void split(float h, unsigned short &a, unsigned short &b)
    {
        const float v = h * scale;
        a = narrow<T>(v);
        const float w = widen<T>(a), r = (v - w) * rest;
        b = __builtin_isfinite(w) ? narrow<T>(r) : (unsigned short)0;
    }
};
// Sum of products of the parts with weights w.
template <int T, class X>
__device__ __forceinline__ v4f product(const v4u (&x)[X::P], v4u w, v4f c)
{
#pragma unroll
    for (int q = 0; q < X::P; ++q)
        if (!(X::LO && q == X::P - 1)) c = mfma16<T>(x[q], w, c);
    if constexpr (X::LO) {
        const v4f d = mfma16<T>(x[X::P - 1], w, v4f{0, 0, 0, 0});
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = fmaf(d[e], 1.0f / X::rest, c[e]);
    }
    return c;
}

// ---- weights of 16 bits: count matrices of rows x cols
struct Weights16 {
    const unsigned short *base;
    int64_t ld, stride;
    int rows, cols;
};
// B: blocks of 32 columns in a chunk: four for few vectors, two (a line of 128 bytes per row) for tiles.
template <int T_, int R_, int B_>
struct Span16 {
    static constexpr int T = T_, R = R_, B = B_, CH = 32 * B, PIECES = 1;
    const unsigned short *p[R];
    int left;                                              // columns from the lane's first one on
    struct Regs { v4u w[R][B]; };
    struct Few { v4f d[R][4]; };
    __device__ __forceinline__ void set(int r, const Weights16 &W, int64_t m, int row, int quarter, int columns)
    {
        p[r] = W.base + m * W.stride + (int64_t)row * W.ld + 8 * quarter;
        left = columns - 8 * quarter;
    }
    template <bool TAIL>
    __device__ __forceinline__ void load(Regs &g, int c) const
    {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < B; ++j)
                g.w[r][j] = TAIL ? load8(p[r], c * CH + 32 * j, left) : __builtin_nontemporal_load(reinterpret_cast<const v4u *>(p[r] + c * CH + 32 * j));
    }
    static __device__ __forceinline__ void clear(Few &f)
    {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) f.d[r][j] = v4f{0, 0, 0, 0};
    }
    static __device__ __forceinline__ float finish(const Few &f, int r) { return (f.d[r][0][0] + f.d[r][1][1]) + (f.d[r][2][2] + f.d[r][3][3]); }
    template <bool TAIL, class X>
    __device__ __forceinline__ void few(const Regs &g, int, const typename X::Raw (&raw)[PIECES], Few &f) const
    {
        static_assert(B == 4, "four blocks");
        v4u x[X::P];
        X::operands(raw[0], x);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < R; ++r) f.d[r][j] = product<T, X>(x, g.w[r][j], f.d[r][j]);
    }
    template <bool TAIL, int NT, class X>
    __device__ __forceinline__ void tiles(const Regs &g, int, const typename X::Raw (&raw)[NT][B], v4f (&acc)[R][NT]) const
    {
#pragma unroll
        for (int j = 0; j < B; ++j)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                v4u x[X::P];
                X::operands(raw[t][j], x);
#pragma unroll
                for (int r = 0; r < R; ++r) acc[r][t] = product<T, X>(x, g.w[r][j], acc[r][t]);
            }
    }
};

// ---- weights of 4 bits
// A row of codes is two columns to a byte, the low half first.  A lane loads 16 bytes, so the four quarters of a wave hold 32
// columns each; swapping words between the quarters (a 4 x 4 transposition, four instructions) leaves the words that one
// matrix instruction takes, its 32 columns in order, in one register.
struct WeightsQ4 {
    const unsigned char *codes, *zeros;                   // zeros NULL: 8
    const void *scales;
    int64_t ld_codes, ld_scales, stride_codes, stride_scales;
    int rows, cols, shift;                                // 2^shift columns share a scale
};

__device__ __forceinline__ v4u transpose_quarters(v4u w)
{
    auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return v4u{c[0], c[1], d[0], d[1]};
}

// Eight codes less their zero point, exact in 16 bits.
// f16: a code in the low bits of 1024.0 or, from four bits up, of 64.0 adds its value; the subtraction leaves code - zero.
// Columns come in the order 0 4 1 5 2 6 3 7.
// bf16: a byte that holds a code is that code times 2^-9 in e4m3, so a conversion takes two of them to 32 bits; what is left
// after the subtraction has 8 bits at most and is cut to bf16.  The factor 2^9 is in the scale.  Columns in order.
template <int T> struct Zero;
template <> struct Zero<F16> {
    v2h lo, hi;
    __device__ __forceinline__ explicit Zero(int z)
    {
        const _Float16 a = (_Float16)(float)(-1024 - z), b = (_Float16)(float)(-64 - z);
        lo = v2h{a, a};
        hi = v2h{b, b};
    }
};
template <> struct Zero<BF16> {
    float z;
    __device__ __forceinline__ explicit Zero(int v) : z((float)v * 0x1p-9f) {}
};
__device__ __forceinline__ v4u dequantise(unsigned w, const Zero<F16> &z)
{
    const unsigned w8 = w >> 8;
    const v2h a = __builtin_bit_cast(v2h, (w & 0x000f000fu) | 0x64006400u) + z.lo;
    const v2h b = __builtin_bit_cast(v2h, (w & 0x00f000f0u) | 0x54005400u) + z.hi;
    const v2h c = __builtin_bit_cast(v2h, (w8 & 0x000f000fu) | 0x64006400u) + z.lo;
    const v2h d = __builtin_bit_cast(v2h, (w8 & 0x00f000f0u) | 0x54005400u) + z.hi;
    return v4u{__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, c), __builtin_bit_cast(unsigned, d)};
}
__device__ __forceinline__ unsigned high_halves(float a, float b)
{
    return __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, a), 0x07060302u);
}
__device__ __forceinline__ v4u dequantise(unsigned w, const Zero<BF16> &z)
{
    const int even = (int)(w & 0x0f0f0f0fu), odd = (int)((w >> 4) & 0x0f0f0f0fu);
    const v2f e0 = __builtin_amdgcn_cvt_pk_f32_fp8(even, false), e1 = __builtin_amdgcn_cvt_pk_f32_fp8(even, true);
    const v2f o0 = __builtin_amdgcn_cvt_pk_f32_fp8(odd, false), o1 = __builtin_amdgcn_cvt_pk_f32_fp8(odd, true);
    return v4u{high_halves(e0[0] - z.z, o0[0] - z.z), high_halves(e0[1] - z.z, o0[1] - z.z),
               high_halves(e1[0] - z.z, o1[0] - z.z), high_halves(e1[1] - z.z, o1[1] - z.z)};
}
template <int T>
__device__ __forceinline__ v4u code_order(v4u x)           // eight elements in the order of the codes
{
    if constexpr (T == BF16) return x;
    else
        return v4u{__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u),
                   __builtin_amdgcn_perm(x[3], x[1], 0x05040100u), __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
}

// N scales or zero points that lie side by side, as one load.
template <typename E, int N> struct Run { typedef E type __attribute__((ext_vector_type(N), aligned(sizeof(E)))); };

// P: pieces of 128 columns in a chunk; two read whole lines of 128 bytes per row.  GB: blocks of 32 columns that share a scale: 1, 2 and
// 4 for groups of just 32, 64 and 128 columns (then the scales of a chunk are one load), 8 for larger ones; 4 also for those if P is 1.
// S: type of the scales.  T: type of the operands.  Z: some matrix has zero points; one that has none reads its codes in
// their place and puts 8 for what it read, so that no load stands under a condition.
template <int T_, int R_, int P, int GB, int S, bool Z>
struct SpanQ4 {
    static constexpr int T = T_, R = R_, B = 4 * P, CH = 32 * B, PIECES = P, NG = 4 * P > GB ? 4 * P / GB : 1, PER = GB < 4 ? GB : 4;     // PER: blocks of a piece that share one
    typedef typename std::conditional<S == F32, float, unsigned short>::type Scale;
    typedef typename Run<Scale, NG>::type Scales;
    typedef typename Run<unsigned char, NG>::type Zeros;
    const unsigned char *q[R], *z[R];
    const Scale *s[R];
    int cols, offset, shift[R];
    unsigned zmask[R], zelse[R];
    struct Regs { v4u w[R][P]; Scales s[R]; Zeros z[Z ? R : 1]; };
    struct Few { float y[R]; };
    __device__ __forceinline__ void set(int r, const WeightsQ4 &W, int64_t m, int row, int quarter, int columns)
    {
        q[r] = W.codes + m * W.stride_codes + (int64_t)row * W.ld_codes + 16 * quarter;
        const int64_t at = m * W.stride_scales + (int64_t)row * W.ld_scales;
        s[r] = static_cast<const Scale *>(W.scales) + at;
        z[r] = W.zeros ? W.zeros + at : q[r] - 16 * quarter;
        zmask[r] = W.zeros ? 255 : 0;
        zelse[r] = W.zeros ? 0 : 8;
        cols = columns;
        shift[r] = W.shift;
        offset = 32 * quarter;
    }
    // Nothing is computed from what is loaded, so that it can be requested a chunk ahead.
    template <bool TAIL>
    __device__ __forceinline__ void load(Regs &g, int c) const
    {
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int h = 0; h < P; ++h) {
                if constexpr (TAIL) g.w[r][h] = v4u{0, 0, 0, 0};
                if (!TAIL || c * CH + 128 * h + offset < cols)
                    g.w[r][h] = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(q[r] + c * (CH / 2) + 64 * h));
            }
            if constexpr (TAIL) {
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    const int at = min(c * CH + 32 * GB * i, cols - 1) >> shift[r];
                    g.s[r][i] = s[r][at];
                    if constexpr (Z) g.z[r][i] = z[r][at];
                }
            } else {
                const int at = (c * CH) >> shift[r];
                g.s[r] = *reinterpret_cast<const Scales *>(s[r] + at);
                if constexpr (Z) g.z[r] = *reinterpret_cast<const Zeros *>(z[r] + at);
            }
        }
    }
    __device__ __forceinline__ Zero<T> zero(const Regs &g, int r, int i) const
    {
        if constexpr (Z) return Zero<T>((int)((g.z[r][i] & zmask[r]) | zelse[r]));
        else return Zero<T>(8);
    }
    static __device__ __forceinline__ float factor(Scale v)
    {
        float f;
        if constexpr (S == F32) f = v;
        else f = widen<S>(v);
        return T == BF16 ? f * 0x1p9f : f;
    }
    static __device__ __forceinline__ void clear(Few &f)
    {
#pragma unroll
        for (int r = 0; r < R; ++r) f.y[r] = 0;
    }
    static __device__ __forceinline__ float finish(const Few &f, int r) { return f.y[r]; }
    // A block past the last column counts nothing: its sum is zero, and so has the scale to be (it could be infinite).
    template <bool TAIL, class X>
    __device__ __forceinline__ void few(const Regs &g, int c, const typename X::Raw (&raw)[PIECES], Few &f) const
    {
#pragma unroll
        for (int h = 0; h < P; ++h) {
            v4u x[X::P];
            X::operands(raw[h], x);
#pragma unroll
            for (int q = 0; q < X::P; ++q) x[q] = code_order<T>(x[q]);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const v4u w = transpose_quarters(g.w[r][h]);
#pragma unroll
                for (int i = 0; i < 4 / PER; ++i) {
                    const int at = 4 * h / GB + i;
                    const Zero<T> less = zero(g, r, at);
                    float sum = 0;
#pragma unroll
                    for (int b = 0; b < PER; ++b) {
                        const int j = i * PER + b;
                        const v4f d = product<T, X>(x, dequantise(w[j], less), v4f{0, 0, 0, 0});
                        sum = b ? sum + d[j] : d[j];
                    }
                    f.y[r] = fmaf(sum, !TAIL || c * CH + 128 * h + 32 * PER * i < cols ? factor(g.s[r][at]) : 0.0f, f.y[r]);
                }
            }
        }
    }
    template <bool TAIL, int NT, class X>
    __device__ __forceinline__ void tiles(const Regs &g, int c, const typename X::Raw (&raw)[NT][4], v4f (&acc)[R][NT]) const
    {
        static_assert(P == 1, "one piece");
        v4u w[R];
#pragma unroll
        for (int r = 0; r < R; ++r) w[r] = transpose_quarters(g.w[r][0]);
#pragma unroll
        for (int i = 0; i < 4 / PER; ++i) {
            v4f sum[R][NT];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int t = 0; t < NT; ++t) sum[r][t] = v4f{0, 0, 0, 0};
#pragma unroll
            for (int b = 0; b < PER; ++b) {
                const int j = i * PER + b;
                v4u wv[R];
#pragma unroll
                for (int r = 0; r < R; ++r) wv[r] = dequantise(w[r][j], zero(g, r, i));
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    v4u x[X::P];
                    X::operands(raw[t][j], x);
#pragma unroll
                    for (int q = 0; q < X::P; ++q) x[q] = code_order<T>(x[q]);
#pragma unroll
                    for (int r = 0; r < R; ++r) sum[r][t] = product<T, X>(x, wv[r], sum[r][t]);
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float f = !TAIL || c * CH + 32 * PER * i < cols ? factor(g.s[r][i]) : 0.0f;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[r][t][e] = fmaf(sum[r][t][e], f, acc[r][t][e]);
            }
        }
    }
};

// Chunks first, first + step, ... of the columns, weights and vectors requested a chunk ahead.  The last chunk, if it is
// not whole, comes after the others and is the only one whose loads look at where the columns end.
template <class SPAN, class LOAD, class APPLY>
__device__ __forceinline__ void chunks(int cols, int first, int step, LOAD load, APPLY apply)
{
    const int whole = cols / SPAN::CH;
    int c = first;
    if (c >= whole) return;
    load(0, c);
    for (;;) {                                             // no load stands under a condition: waiting for one would wait for all
        if (c + step >= whole) { apply(0, c); return; }
        load(1, c + step);
        apply(0, c);
        c += step;
        if (c + step >= whole) { apply(1, c); return; }
        load(0, c + step);
        apply(1, c);
        c += step;
    }
}
template <class SPAN, class X>
__device__ __forceinline__ void few_product(const SPAN &s, const X &x, int cols, int first, int step, int lane, float (&y)[SPAN::R])
{
    typename SPAN::Regs g[2];
    typename X::Raw raw[2][SPAN::PIECES];
    typename SPAN::Few f;
    SPAN::clear(f);
    const int xleft = cols - 32 * (lane & 3) - 8 * (lane >> 4), whole = cols / SPAN::CH;
    chunks<SPAN>(cols, first, step,
        [&](int b, int c) {
            s.template load<false>(g[b], c);
#pragma unroll
            for (int h = 0; h < SPAN::PIECES; ++h) x.template load<false>(raw[b][h], c * SPAN::CH + 128 * h, xleft);
        },
        [&](int b, int c) { s.template few<false, X>(g[b], c, raw[b], f); });
    if (whole * SPAN::CH < cols && whole % step == first) {
        s.template load<true>(g[0], whole);
#pragma unroll
        for (int h = 0; h < SPAN::PIECES; ++h) x.template load<true>(raw[0][h], whole * SPAN::CH + 128 * h, xleft);
        s.template few<true, X>(g[0], whole, raw[0], f);
    }
#pragma unroll
    for (int r = 0; r < SPAN::R; ++r) y[r] = SPAN::finish(f, r);
}
template <class SPAN, int NT, class X>
__device__ __forceinline__ void tile_product(const SPAN &s, const X (&x)[NT], int cols, int first, int step, int lane, v4f (&acc)[SPAN::R][NT])
{
    typename SPAN::Regs g[2];
    typename X::Raw raw[2][NT][SPAN::B];
#pragma unroll
    for (int r = 0; r < SPAN::R; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[r][t] = v4f{0, 0, 0, 0};
    const int xleft = cols - 8 * (lane >> 4), whole = cols / SPAN::CH;
    chunks<SPAN>(cols, first, step,
        [&](int b, int c) {
            s.template load<false>(g[b], c);
#pragma unroll
            for (int j = 0; j < SPAN::B; ++j)
#pragma unroll
                for (int t = 0; t < NT; ++t) x[t].template load<false>(raw[b][t][j], c * SPAN::CH + 32 * j, xleft);
        },
        [&](int b, int c) { s.template tiles<false, NT, X>(g[b], c, raw[b], acc); });
    if (whole * SPAN::CH < cols && whole % step == first) {
        s.template load<true>(g[0], whole);
#pragma unroll
        for (int j = 0; j < SPAN::B; ++j)
#pragma unroll
            for (int t = 0; t < NT; ++t) x[t].template load<true>(raw[0][t][j], whole * SPAN::CH + 32 * j, xleft);
        s.template tiles<true, NT, X>(g[0], whole, raw[0], acc);
    }
}

// Sums of the W waves of a workgroup, in the order of the waves.  Tiles: 16 vectors x 16 rows each; few vectors: 4 x 16.
template <int TILES>
__device__ __forceinline__ void put_sums(float *lds, int wave, int lane, const v4f (&acc)[TILES])
{
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) lds[((wave * TILES + t) * 16 + 4 * (lane >> 4) + i) * 16 + (lane & 15)] = acc[t][i];
}
template <int R>
__device__ __forceinline__ void put_few(float *lds, int wave, int lane, const float (&y)[R])
{
#pragma unroll
    for (int r = 0; r < R; ++r) lds[(wave * R + r) * 64 + lane] = y[r];
}
// V: vectors of a tile (16, or 4)
template <int W, int TILES, int V>
__device__ __forceinline__ float get_sum(const float *lds, int t, int m, int n)
{
    float v = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) v += lds[((w * TILES + t) * V + m) * 16 + n];
    return v;
}

}  // namespace psk
