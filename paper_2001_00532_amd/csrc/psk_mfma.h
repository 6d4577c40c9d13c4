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

// Eight 16-bit elements from column k on, zeros from column `cols` on.
__device__ __forceinline__ v4u load8(const unsigned short *p, int k, int cols)
{
    if (k + 8 <= cols) return *reinterpret_cast<const v4u_u *>(p + k);
    v4u r = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k + i < cols) r[i / 2] |= (unsigned)p[k + i] << (16 * (i & 1));
    return r;
}

// ---- vectors
// Sixteen vectors of 16 bits per tile, one row pointer per lane and tile.
template <int NT>
struct Rows16 {
    const unsigned short *p[NT];
    int cols;
    __device__ __forceinline__ v4u load(int t, int k) const { return load8(p[t], k, cols); }
};

// Vectors of 32 bits as three rows of bf16 each: v = a + b + c with 8 significant bits in each, cut off and not rounded, so the
// sum is exact and a value near the largest does not become infinite.  Rows 3v, 3v + 1, 3v + 2 of a tile are the parts of
// vector v (5 vectors per tile); their sums are added up at the end.  Infinity and NaN stand in the first part alone.
template <int NT>
struct Rows32 {
    const float *p[NT];
    int cols, part;
    __device__ __forceinline__ v4u load(int t, int k) const
    {
        float v[8];
        if (k + 8 <= cols) {
            const v4f_e a = *reinterpret_cast<const v4f_e *>(p[t] + k), b = *reinterpret_cast<const v4f_e *>(p[t] + k + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k + i < cols ? p[t][k + i] : 0.0f;
        }
        v4u r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = part_of(v[2 * i]) >> 16 | (part_of(v[2 * i + 1]) & 0xffff0000u);
        return r;
    }
    __device__ __forceinline__ unsigned part_of(float v) const
    {
        const unsigned u = __builtin_bit_cast(unsigned, v);
        if ((u & 0x7f800000u) == 0x7f800000u) return part ? 0u : (u & 0x7fffffu ? 0x7fc00000u : u);
        const float a = __builtin_bit_cast(float, u & 0xffff0000u), r = v - a;
        const float b = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, r) & 0xffff0000u);
        return __builtin_bit_cast(unsigned, part == 0 ? a : (part == 1 ? b : r - b));
    }
};

// ---- weights of 16 bits: count matrices of rows x cols
struct Weights16 {
    const unsigned short *base;
    int64_t ld, stride;
    int rows, cols;
};
template <int T_, int R_>
struct Span16 {
    static constexpr int T = T_, R = R_, CH = 64;         // columns of a chunk: two pieces of 64 bytes per row
    const unsigned short *p[R];
    int cols;
    struct Regs { v4u w[R][2]; };
    __device__ __forceinline__ void set(int r, const Weights16 &W, int64_t m, int row, int quarter)
    {
        p[r] = W.base + m * W.stride + (int64_t)row * W.ld + 8 * quarter;
        cols = W.cols - 8 * quarter;
    }
    __device__ __forceinline__ void load(Regs &g, int c) const
    {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < 2; ++j) g.w[r][j] = load8(p[r], c * CH + 32 * j, cols);
    }
    template <int NT, class X>
    __device__ __forceinline__ void apply(const Regs &g, int c, int quarter, const X &x, v4f (&acc)[R][NT]) const
    {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const v4u xv = x.load(t, c * CH + 32 * j + 8 * quarter);
#pragma unroll
                for (int r = 0; r < R; ++r) acc[r][t] = mfma16<T>(xv, g.w[r][j], acc[r][t]);
            }
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

// GB: blocks of 32 columns that share a scale for certain (1, 2, 4).  S: type of the scales.  T: type of the operands.
template <int T_, int R_, int GB, int S>
struct SpanQ4 {
    static constexpr int T = T_, R = R_, CH = 128, NG = 4 / GB;
    const unsigned char *q[R], *z[R];
    const void *s[R];
    int cols, offset, shift[R], last[R];
    bool zeros[R];
    struct Regs { v4u w[R]; float s[R][NG]; int z[R][NG]; };
    __device__ __forceinline__ void set(int r, const WeightsQ4 &W, int64_t m, int row, int quarter)
    {
        q[r] = W.codes + m * W.stride_codes + (int64_t)row * W.ld_codes + 16 * quarter;
        const int64_t at = m * W.stride_scales + (int64_t)row * W.ld_scales;
        s[r] = static_cast<const char *>(W.scales) + at * (S == F32 ? 4 : 2);
        zeros[r] = W.zeros != nullptr;
        z[r] = W.zeros + (zeros[r] ? at : 0);
        cols = W.cols;
        shift[r] = W.shift;
        last[r] = (W.cols - 1) >> W.shift;
        offset = 32 * quarter;
    }
    __device__ __forceinline__ void load(Regs &g, int c) const
    {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            g.w[r] = v4u{0, 0, 0, 0};
            if (c * CH + offset < cols) g.w[r] = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(q[r] + c * (CH / 2)));
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                const int at = min((c * CH + 32 * GB * i) >> shift[r], last[r]);
                if constexpr (S == F32) g.s[r][i] = static_cast<const float *>(s[r])[at];
                else g.s[r][i] = widen<S>(static_cast<const unsigned short *>(s[r])[at]);
                g.z[r][i] = zeros[r] ? (int)z[r][at] : 8;
            }
        }
    }
    template <int NT, class X>
    __device__ __forceinline__ void apply(const Regs &g, int c, int quarter, const X &x, v4f (&acc)[R][NT]) const
    {
        v4u w[R];
#pragma unroll
        for (int r = 0; r < R; ++r) w[r] = transpose_quarters(g.w[r]);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            if (c * CH + 32 * GB * i >= cols) break;
            v4f sum[R][NT];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int t = 0; t < NT; ++t) sum[r][t] = v4f{0, 0, 0, 0};
#pragma unroll
            for (int b = 0; b < GB; ++b) {
                v4u wv[R];
#pragma unroll
                for (int r = 0; r < R; ++r) wv[r] = dequantise(w[r][i * GB + b], Zero<T>(g.z[r][i]));
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const v4u xv = code_order<T>(x.load(t, c * CH + 32 * (i * GB + b) + 8 * quarter));
#pragma unroll
                    for (int r = 0; r < R; ++r) sum[r][t] = mfma16<T>(xv, wv[r], sum[r][t]);
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float f = T == BF16 ? g.s[r][i] * 0x1p9f : g.s[r][i];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[r][t][e] = fmaf(sum[r][t][e], f, acc[r][t][e]);
            }
        }
    }
};

// Chunks first, first + step, ... of the columns, one chunk of weights requested ahead.
template <class SPAN, int NT, class X>
__device__ __forceinline__ void span_product(const SPAN &s, const X &x, int cols, int first, int step, int quarter, v4f (&acc)[SPAN::R][NT])
{
    const int n = (cols + SPAN::CH - 1) / SPAN::CH;
    if (first >= n) return;
    typename SPAN::Regs g;
    s.load(g, first);
    for (int c = first; c < n; c += step) {
        typename SPAN::Regs next;
        if (c + step < n) s.load(next, c + step);
        s.template apply<NT, X>(g, c, quarter, x, acc);
        g = next;
    }
}

// Sums of the W waves of a workgroup, in the order of the waves: tile t of `sums` as 16 vectors x 16 rows.
template <int TILES>
__device__ __forceinline__ void put_sums(float *lds, int wave, int lane, const v4f (&acc)[TILES])
{
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) lds[((wave * TILES + t) * 16 + 4 * (lane >> 4) + i) * 16 + (lane & 15)] = acc[t][i];
}
template <int W, int TILES>
__device__ __forceinline__ float get_sum(const float *lds, int t, int m, int n)
{
    float v = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) v += lds[((w * TILES + t) * 16 + m) * 16 + n];
    return v;
}

}  // namespace psk
