// Products of dense rows (16-bit or 4-bit weights) with a few vectors on the matrix cores (gfx950, wave64).
//
// One matrix instruction multiplies 16 vectors by 16 rows of weights over 32 columns:
//   D[m][n] += sum_k X[m][k] W[n][k],   lane l holds X and W at row l % 16, columns 8 (l / 16) .. + 7, and D at n = l % 16,
//   m = 4 (l / 16) + i, i = 0 .. 3.
// The weights are the second operand, so a lane dequantises, loads the scale of and sums up the same row n.  Vectors past the
// last one repeat it (their rows of D are not looked at), rows past the last one likewise; only columns need zeros.
// Sums are held in 32 bits.
//
// What bounds these kernels, after memory itself, is how loads are taken apart:
//  - a load of 16 bytes per lane costs a compute unit 65 cycles where neighbouring lanes read other rows, as the operands' layout would
//    have them, and 17 to 35 where four and more neighbours read on in one row or all read one place (lines in the L1; 90
//    cycles per kilobyte is what 7 TB/s leave);
//  - 134 MB of rows of 4 KB by 16 rows x 64 bytes to a load take 29.9 us, by 8 rows x 128 bytes (whole lines) 25.3, and 21.9 where a
//    wave reads on for 1 KB in each row before the next wave's part begins; in one piece 21.7.
// So weights are loaded eight lanes to a row and change places through LDS (Exchange), a wave owns consecutive columns, the
// scales of several groups are one load, and vectors come four blocks to a load (few of them) or from a copy in the order of the
// operands (many).
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

// Eight 16-bit elements from column k on, zeros from column `left` on.  Where the row ends among them, the eight before its end are loaded
// and moved.  At a row's beginning there may not be eight: a loop of one load (written out it would cost the kernels around it more registers
// than all the rest).
__device__ __forceinline__ v4u load8(const unsigned short *p, int k, int left)
{
    if (k + 8 <= left) return *reinterpret_cast<const v4u_u *>(p + k);
    v4u r = {0, 0, 0, 0};
    if (k >= 8 && k < left) {
        r = *reinterpret_cast<const v4u_u *>(p + left - 8);
        const int by = k + 8 - left;
        if (by & 4) r = v4u{r[2], r[3], 0, 0};
        if (by & 2) r = v4u{r[1], r[2], r[3], 0};
        if (by & 1) r = v4u{r[0] >> 16 | r[1] << 16, r[1] >> 16 | r[2] << 16, r[2] >> 16 | r[3] << 16, r[3] >> 16};
    } else if (k < left) {
#pragma unroll 1
        for (int i = k + 7; i >= k; --i) {
            const unsigned e = i < left ? p[i] : 0u;
            r = v4u{r[0] << 16 | e, r[1] << 16 | r[0] >> 16, r[2] << 16 | r[1] >> 16, r[3] << 16 | r[2] >> 16};
        }
    }
    return r;
}

// Two loads of a wave, rows 0 to 7 and 8 to 15 with 128 bytes each, into the order of the operands: for half h of the 128 bytes, row
// lane % 16, bytes 64 h + 16 (lane / 16).  The place of a piece of 16 bytes within its row is chosen so that neither side's lanes meet on
// the banks of LDS.
__device__ __forceinline__ int load_row(int lane, int i) { return 8 * i + (lane >> 3); }
__device__ __forceinline__ int load_piece(int lane) { return (lane & 7) ^ (lane >> 3); }
struct Exchange {
    v4u *put;
    const v4u *get[2];
    __device__ __forceinline__ Exchange(v4u *space, int lane) : put(space + lane)
    {
        for (int h = 0; h < 2; ++h) get[h] = space + 8 * (lane & 15) + ((4 * h + (lane >> 4)) ^ (lane & 7));
    }
    __device__ __forceinline__ void operator()(const v4u (&w)[2], v4u (&out)[2]) const
    {
        // LDS operations of one wave are carried out in their order; the compiler is kept from changing it
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        put[0] = w[0];
        put[64] = w[1];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        out[0] = *get[0];
        out[1] = *get[1];
    }
};
constexpr int EXCHANGE = 128;                              // v4u of a wave

// ---- vectors
// Few vectors, up to four: row 4v + j of the first operand is block j (32 columns) of four blocks of vector v, so one load per lane
// brings four blocks.  The instruction that multiplies it by block j of the weights leaves the product of the two in element j
// of the lanes of quarter v (and products of blocks that do not belong together in the other elements).
// Tiles: row m of an operand is vector m of the tile; they come from a copy of the vectors in the order of the operands (Copied).
// A vector may have several parts whose products add up; P of them.
template <int T>
struct Plain16 {                                           // 16 bits
    static constexpr int P = 1;
    struct Raw { v4u v; };
    const unsigned short *p;
    __device__ __forceinline__ void set(const void *X, int64_t at) { p = static_cast<const unsigned short *>(X) + at; }
    template <bool TAIL>
    __device__ __forceinline__ void load(Raw &r, int k, int left) const { r.v = TAIL ? load8(p, k, left) : *reinterpret_cast<const v4u_u *>(p + k); }
    static __device__ __forceinline__ void operands(const Raw &r, v4u (&x)[P]) { x[0] = r.v; }
};
// 32 bits as three parts of bf16: v = a + b + c with 8 significant bits in each, cut off and not rounded, so the sum is exact and a
// value near the largest does not become infinite.  Exact from 2^-110 on: below, the last bits are less than 2^-133, the smallest number of bf16, and are
// lost.  Infinity and NaN stand in the first part alone.
__device__ __forceinline__ void cut(float value, unsigned (&part)[3])      // the upper halves are the parts
{
    const float v = __builtin_canonicalizef(value);        // a NaN keeps its first bit
    const float a = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, v) & 0xffff0000u), d = v - a;
    const float rest = __builtin_isfinite(v) ? d : 0.0f;
    const float b = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, rest) & 0xffff0000u), c = rest - b;
    part[0] = __builtin_bit_cast(unsigned, a);
    part[1] = __builtin_bit_cast(unsigned, b);
    part[2] = __builtin_bit_cast(unsigned, c);
}
struct Parts32 {
    static constexpr int P = 3;
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
        if (k >= 8 && k < left) {                          // as load8
            r.a = *reinterpret_cast<const v4f_e *>(p + left - 8);
            r.b = *reinterpret_cast<const v4f_e *>(p + left - 4);
            const int by = k + 8 - left;
            if (by & 4) { r.a = r.b; r.b = v4f_e{0, 0, 0, 0}; }
            if (by & 2) { r.a = v4f_e{r.a[2], r.a[3], r.b[0], r.b[1]}; r.b = v4f_e{r.b[2], r.b[3], 0, 0}; }
            if (by & 1) { r.a = v4f_e{r.a[1], r.a[2], r.a[3], r.b[0]}; r.b = v4f_e{r.b[1], r.b[2], r.b[3], 0}; }
        } else if (k < left) {
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
            for (int e = 0; e < 2; ++e) cut(i < 2 ? r.a[2 * i + e] : r.b[2 * i - 4 + e], part[e]);
#pragma unroll
            for (int q = 0; q < P; ++q) x[q][i] = __builtin_amdgcn_perm(part[1][q], part[0][q], 0x07060302u);
        }
    }
};
// The same three parts, cut where the value is written and read many times: each in an array of its own.
struct Thirds {
    static constexpr int P = 3;
    struct Raw { v4u v[P]; };
    const unsigned short *p;
    int64_t apart;                                         // from one array to the next
    __device__ __forceinline__ void set(const unsigned short *h, int64_t at, int64_t to_next) { p = h + at; apart = to_next; }
    template <bool TAIL>
    __device__ __forceinline__ void load(Raw &r, int k, int left) const
    {
#pragma unroll
        for (int q = 0; q < P; ++q) r.v[q] = TAIL ? load8(p + q * apart, k, left) : *reinterpret_cast<const v4u_u *>(p + q * apart + k);
    }
    static __device__ __forceinline__ void operands(const Raw &r, v4u (&x)[P])
    {
#pragma unroll
        for (int q = 0; q < P; ++q) x[q] = r.v[q];
    }
    static __device__ __forceinline__ void store(unsigned short *h, int64_t at, int64_t to_next, float v)
    {
        unsigned part[P];
        cut(v, part);
#pragma unroll
        for (int q = 0; q < P; ++q) h[at + q * to_next] = (unsigned short)(part[q] >> 16);
    }
};
// 32 bits as two parts of f16, the nearest one and the nearest one to what is left, which is as close as 32 bits are: 2^-24 of the value.  f16 has
// a small range, so a wave scales its columns of a vector by a power of two that takes the largest finite value to 2^14 .. 2^15 (keep_scaled); what lies
// 2^17 and more below that is off by 2^-25 / 2^14 of it.
struct Scaled {
    static constexpr int P = 2;
    static __device__ __forceinline__ void operands(const v4f (&v)[2], int up, v4u (&x)[P])      // in the order of the codes
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const v2f s = {__builtin_amdgcn_ldexpf(v[0][i], up), __builtin_amdgcn_ldexpf(v[1][i], up)};
            const v2h hi = __builtin_convertvector(s, v2h);
            // what is left is 8 at most; of an infinity it is no number, and then -16, which leaves the product with the first part as it is
            const v2f rest = {fmaxf(s[0] - (float)hi[0], -16.0f), fmaxf(s[1] - (float)hi[1], -16.0f)};
            x[0][i] = __builtin_bit_cast(unsigned, hi);
            x[1][i] = __builtin_bit_cast(unsigned, __builtin_convertvector(rest, v2h));
        }
    }
};
// The copy: for every tile and block of 32 columns, P kilobytes, one per part, the 16 bytes of lane l at 16 l.  Columns are padded with zeros
// to a multiple of 256.  spread: the weights of a piece of 128 columns stay as they are loaded, lane quarter q with columns 32 q to 32 q + 31,
// so block j of the piece is columns 32 q + 8 j; otherwise 32 j + 8 q.
__host__ __device__ __forceinline__ int copied_blocks(int cols) { return (cols + 255) / 256 * 8; }
__device__ __forceinline__ int copied_column(int block, int quarter, bool spread)
{
    return spread ? 128 * (block >> 2) + 32 * quarter + 8 * (block & 3) : 32 * block + 8 * quarter;
}
template <class X>
struct Copied {
    typedef X Parts;
    struct Raw { v4u v[X::P]; };
    const v4u *p;
    __device__ __forceinline__ void set(const void *copy, int tile, int blocks, int lane)
    {
        p = static_cast<const v4u *>(copy) + (int64_t)tile * blocks * X::P * 64 + lane;
    }
    __device__ __forceinline__ void load(Raw &r, int block) const
    {
#pragma unroll
        for (int q = 0; q < X::P; ++q) r.v[q] = p[(block * X::P + q) * 64];
    }
};
// Sum of products of the parts with weights w.
template <int T, class X>
__device__ __forceinline__ v4f product(const v4u (&x)[X::P], v4u w, v4f c)
{
#pragma unroll
    for (int q = 0; q < X::P; ++q) c = mfma16<T>(x[q], w, c);
    return c;
}

// ---- weights of 16 bits: count matrices of rows x cols
struct Weights16 {
    const unsigned short *base;
    int64_t ld, stride;
    int rows, cols;
};
// f16 weights for vectors in parts of bf16: 11 significant bits are two parts, cut off like those of the vectors.
__device__ __forceinline__ void cut_f16(v4u w, v4u &hi, v4u &lo)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = widen<F16>((unsigned short)w[i]), b = widen<F16>((unsigned short)(w[i] >> 16));
        const float p = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, a) & 0xffff0000u), q = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, b) & 0xffff0000u);
        hi[i] = __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, a), 0x07060302u);
        lo[i] = __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, b - q), __builtin_bit_cast(unsigned, a - p), 0x07060302u);
    }
}
// B: blocks of 32 columns in a chunk: four for few vectors, two for tiles.  XT: type of the vectors' operands.
template <int T_, int XT, int R_, int B_>
struct Span16 {
    static constexpr int T = XT, R = R_, B = B_, CH = 32 * B, PIECES = 1;
    static constexpr bool CUT = XT != T_;
    static_assert(!CUT || T_ == F16, "f16 weights");
    static constexpr bool SPREAD = false, CODES = false;
    static constexpr float unit = 1;
    const unsigned short *p[R][2];
    int left;                                              // columns from the lane's first one on
    struct Regs { v4u w[R][B / 2][2]; };
    struct Few { v4f d[R][4]; };
    __device__ __forceinline__ void set(int r, const Weights16 &W, int64_t m, int row0, int rows, int lane, int columns)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) p[r][i] = W.base + m * W.stride + (int64_t)min(row0 + load_row(lane, i), rows - 1) * W.ld + 8 * load_piece(lane);
        left = columns - 8 * load_piece(lane);
    }
    template <bool TAIL>
    __device__ __forceinline__ void load(Regs &g, int c) const
    {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int u = 0; u < B / 2; ++u)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    g.w[r][u][i] = TAIL ? load8(p[r][i], c * CH + 64 * u, left)
                                        : __builtin_nontemporal_load(reinterpret_cast<const v4u_u *>(p[r][i] + c * CH + 64 * u));
    }
    static __device__ __forceinline__ void exchange(const Regs &g, const Exchange &place, v4u (&all)[R][B])
    {
#pragma unroll
        for (int u = 0; u < B / 2; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                v4u o[2];
                place(g.w[r][u], o);
                all[r][2 * u] = o[0];
                all[r][2 * u + 1] = o[1];
            }
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
    __device__ __forceinline__ void few(const Regs &g, int, const Exchange &place, const typename X::Raw (&raw)[PIECES], Few &f) const
    {
        static_assert(B == 4, "four blocks");
        v4u x[X::P];
        X::operands(raw[0], x);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                v4u w[2];
                place(g.w[r][u], w);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    v4u p[2] = {w[j], w[j]};
                    if constexpr (CUT) {
                        cut_f16(w[j], p[0], p[1]);
                        f.d[r][2 * u + j] = product<T, X>(x, p[1], f.d[r][2 * u + j]);
                    }
                    f.d[r][2 * u + j] = product<T, X>(x, p[0], f.d[r][2 * u + j]);
                }
            }
    }
    template <bool TAIL, int NT, class X>
    __device__ __forceinline__ void tiles(const Regs &, int, int, const v4u (&all)[R][B], const typename Copied<X>::Raw (&raw)[NT][B], v4f (&acc)[R][NT]) const
    {
#pragma unroll
        for (int j = 0; j < B; ++j)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                v4u w[2] = {all[r][j], all[r][j]};
                if constexpr (CUT) cut_f16(all[r][j], w[0], w[1]);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    if constexpr (CUT) acc[r][t] = product<T, X>(raw[t][j].v, w[1], acc[r][t]);
                    acc[r][t] = product<T, X>(raw[t][j].v, w[0], acc[r][t]);
                }
            }
    }
};

// ---- weights of 4 bits
// A row of codes is two columns to a byte, the low half first.  A lane loads 16 bytes, so after the exchange the four quarters of a wave
// hold 32 columns each.  With groups of 128 columns and more the operands take them so (SPREAD); with smaller ones a matrix
// instruction may not reach over the quarters, and swapping words between them (a 4 x 4 transposition, four instructions) leaves the
// words of 32 columns in one register.
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
// after the subtraction has 8 bits at most and is cut to bf16.  The finished sum is multiplied by 2^9 (unit): in the scale 2^9 would make
// one of 2^119 infinite, in the codes a sum of a group of activations of 2^125.  Columns in order.
template <int T> constexpr float code_unit = T == BF16 ? 0x1p9f : 1.0f;
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
    // A constant that the compiler does not see stays in a register, and then "and" with "or" is one instruction: 8192 x 4096 times 64 vectors
    // 16.5 us, without it 18.0.
    unsigned low = 0x64006400u, high = 0x54005400u;
    asm("" : "+v"(low), "+v"(high));
    const unsigned w8 = w >> 8;
    const v2h a = __builtin_bit_cast(v2h, (w & 0x000f000fu) | low) + z.lo;
    const v2h b = __builtin_bit_cast(v2h, (w & 0x00f000f0u) | high) + z.hi;
    const v2h c = __builtin_bit_cast(v2h, (w8 & 0x000f000fu) | low) + z.lo;
    const v2h d = __builtin_bit_cast(v2h, (w8 & 0x00f000f0u) | high) + z.hi;
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

// P: pieces of 128 columns in a chunk, two to a line of 128 bytes per row.  GB: blocks of 32 columns that share a scale: 1, 2 and 4 for
// groups of just 32, 64 and 128 columns (then the scales of a chunk are one load), 4 P for groups of a chunk and more.
// S: type of the scales.  T: type of the operands.  Z: some matrix has zero points; one that has none reads its codes in
// their place and puts 8 for what it read, so that no load stands under a condition.
template <int T_, int R_, int P, int GB, int S, bool Z>
struct SpanQ4 {
    static constexpr bool SPREAD = GB >= 4, CODES = true;
    static constexpr float unit = code_unit<T_>;           // what the sums are to be multiplied by
    static constexpr int T = T_, R = R_, B = 4 * P, CH = 32 * B, PIECES = P, NG = 4 * P > GB ? 4 * P / GB : 1, PER = GB < 4 ? GB : 4;     // PER: blocks of a piece that share one
    typedef typename std::conditional<S == F32, float, unsigned short>::type Scale;
    typedef typename Run<Scale, NG>::type Scales;
    typedef typename Run<unsigned char, NG>::type Zeros;
    const unsigned char *q[R][2], *z[R];
    const Scale *s[R];
    int cols, offset, shift[R];
    unsigned zmask[R], zelse[R];
    struct Regs { v4u w[R][P / 2][2]; Scales s[R]; Zeros z[Z ? R : 1]; };
    struct Few { float y[R]; };
    __device__ __forceinline__ void set(int r, const WeightsQ4 &W, int64_t m, int row0, int rows, int lane, int columns)
    {
        const unsigned char *codes = W.codes + m * W.stride_codes;
#pragma unroll
        for (int i = 0; i < 2; ++i) q[r][i] = codes + (int64_t)min(row0 + load_row(lane, i), rows - 1) * W.ld_codes + 16 * load_piece(lane);
        const int row = min(row0 + (lane & 15), rows - 1);
        const int64_t at = m * W.stride_scales + row * W.ld_scales;
        s[r] = static_cast<const Scale *>(W.scales) + at;
        z[r] = W.zeros ? W.zeros + at : codes + row * W.ld_codes;
        zmask[r] = W.zeros ? 255 : 0;
        zelse[r] = W.zeros ? 0 : 8;
        cols = columns;
        shift[r] = W.shift;
        offset = 32 * load_piece(lane);
    }
    // Nothing is computed from what is loaded, so that it can be requested a chunk ahead.
    template <bool TAIL>
    __device__ __forceinline__ void load(Regs &g, int c) const
    {
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int u = 0; u < P / 2; ++u)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if constexpr (TAIL) g.w[r][u][i] = v4u{0, 0, 0, 0};
                    if (!TAIL || c * CH + 256 * u + offset < cols)
                        g.w[r][u][i] = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(q[r][i] + c * (CH / 2) + 128 * u));
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
    static __device__ __forceinline__ void exchange(const Regs &g, const Exchange &place, v4u (&all)[R][P])
    {
#pragma unroll
        for (int u = 0; u < P / 2; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                v4u o[2];
                place(g.w[r][u], o);
                all[r][2 * u] = o[0];
                all[r][2 * u + 1] = o[1];
            }
    }
    static __device__ __forceinline__ v4u words(v4u w) { return SPREAD ? w : transpose_quarters(w); }
    static __device__ __forceinline__ float factor(Scale v)
    {
        if constexpr (S == F32) return v;
        else return widen<S>(v);
    }
    static __device__ __forceinline__ void clear(Few &f)
    {
#pragma unroll
        for (int r = 0; r < R; ++r) f.y[r] = 0;
    }
    static __device__ __forceinline__ float finish(const Few &f, int r) { return f.y[r]; }
    // A block past the last column counts nothing: its sum is zero, and so has the scale to be (it could be infinite).
    template <bool TAIL, class X>
    __device__ __forceinline__ void few(const Regs &g, int c, const Exchange &place, const typename X::Raw (&raw)[PIECES], Few &f) const
    {
        v4u all[R][P];
        exchange(g, place, all);
#pragma unroll
        for (int h = 0; h < P; ++h) {
            v4u x[X::P];
            X::operands(raw[h], x);
#pragma unroll
            for (int q = 0; q < X::P; ++q) x[q] = code_order<T>(x[q]);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const v4u w = words(all[r][h]);
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
    // Piece h of the chunk, whose words are in `all`.
    template <bool TAIL, int NT, class X>
    __device__ __forceinline__ void tiles(const Regs &g, int c, int h, const v4u (&all)[R][P], const typename Copied<X>::Raw (&raw)[NT][4], v4f (&acc)[R][NT]) const
    {
        v4u w[R];
#pragma unroll
        for (int r = 0; r < R; ++r) w[r] = words(all[r][h]);
#pragma unroll
        for (int i = 0; i < 4 / PER; ++i) {
            const int at = 4 * h / GB + i;
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
                for (int r = 0; r < R; ++r) wv[r] = dequantise(w[r][j], zero(g, r, at));
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int r = 0; r < R; ++r) sum[r][t] = product<T, X>(raw[t][j].v, wv[r], sum[r][t]);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float f = !TAIL || c * CH + 128 * h + 32 * PER * i < cols ? factor(g.s[r][at]) : 0.0f;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[r][t][e] = fmaf(sum[r][t][e], f, acc[r][t][e]);
            }
        }
    }
};

// A wave's share of the columns: chunks from `first` to before `end`, all whole but the last one of the matrix.
struct Share { int first, end, whole; };
template <class SPAN>
__device__ __forceinline__ Share share_of(int cols, int wave, int waves)
{
    const int n = (cols + SPAN::CH - 1) / SPAN::CH;
    Share s;
    s.first = n * wave / waves;
    s.end = n * (wave + 1) / waves;
    s.whole = min(s.end, cols / SPAN::CH);
    return s;
}

// The lane's first column of few vectors, counted from the chunk's.
template <class SPAN>
__device__ __forceinline__ int few_column(int lane) { return copied_column(lane & 3, lane >> 4, SPAN::SPREAD); }

// Weights and vectors are requested a chunk ahead.  The matrix's last chunk, if it is not whole, is the only one whose loads look at where
// the columns end.  (No load stands under a condition inside the loops: waiting for one would wait for all.)
template <class SPAN, class X>
__device__ __forceinline__ void few_product(const SPAN &s, const X &x, int cols, int wave, int waves, int lane, const Exchange &place, float (&y)[SPAN::R])
{
    typename SPAN::Regs g[2];
    typename X::Raw raw[2][SPAN::PIECES];
    typename SPAN::Few f;
    SPAN::clear(f);
    const Share sh = share_of<SPAN>(cols, wave, waves);
    const int left = cols - few_column<SPAN>(lane);
    const auto load = [&](int b, int c) {
        s.template load<false>(g[b], c);
#pragma unroll
        for (int h = 0; h < SPAN::PIECES; ++h) x.template load<false>(raw[b][h], c * SPAN::CH + 128 * h, left);
    };
    const auto apply = [&](int b, int c) { s.template few<false, X>(g[b], c, place, raw[b], f); };
    int c = sh.first;
    if (c < sh.whole) {
        load(0, c);
        for (;;) {
            if (c + 1 >= sh.whole) { apply(0, c++); break; }
            load(1, c + 1);
            apply(0, c++);
            if (c + 1 >= sh.whole) { apply(1, c++); break; }
            load(0, c + 1);
            apply(1, c++);
        }
    }
    if (c < sh.end) {
        s.template load<true>(g[0], c);
#pragma unroll
        for (int h = 0; h < SPAN::PIECES; ++h) x.template load<true>(raw[0][h], c * SPAN::CH + 128 * h, left);
        s.template few<true, X>(g[0], c, place, raw[0], f);
    }
#pragma unroll
    for (int r = 0; r < SPAN::R; ++r) y[r] = SPAN::finish(f, r);
}
// The same for tiles.  Vectors are requested by pieces: those of a chunk's first piece while the one before it is multiplied, the others ahead
// of the next chunk's weights, so that waiting for them does not wait for these.
template <class SPAN, int NT, class X>
__device__ __forceinline__ void tile_product(const SPAN &s, const Copied<X> (&x)[NT], int cols, int wave, int waves, const Exchange &place, v4f (&acc)[SPAN::R][NT])
{
    constexpr int PB = SPAN::B / SPAN::PIECES, N = SPAN::PIECES > 1 ? SPAN::PIECES : 2;      // blocks of a piece, sets of registers for pieces
    typename SPAN::Regs g[2];
    typename Copied<X>::Raw raw[N][NT][PB];
    v4u all[SPAN::R][SPAN::PIECES > 1 ? SPAN::PIECES : SPAN::B];
#pragma unroll
    for (int r = 0; r < SPAN::R; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[r][t] = v4f{0, 0, 0, 0};
    const Share sh = share_of<SPAN>(cols, wave, waves);
    const auto vectors = [&](int set, int c, int h) {
#pragma unroll
        for (int j = 0; j < PB; ++j)
#pragma unroll
            for (int t = 0; t < NT; ++t) x[t].load(raw[set][t][j], c * SPAN::B + h * PB + j);
    };
    const auto rest = [&](int c) {
#pragma unroll
        for (int h = 1; h < SPAN::PIECES; ++h) vectors(h, c, h);
    };
    const auto multiply_rest = [&](int b, int c) {
#pragma unroll
        for (int h = 1; h < SPAN::PIECES; ++h) s.template tiles<false, NT, X>(g[b], c, h, all, raw[h], acc);
    };
    const auto step = [&](int b, int c) {                  // chunk c, another one after it
        const int set = SPAN::PIECES > 1 ? 0 : b, next = SPAN::PIECES > 1 ? 0 : 1 - b;
        rest(c);
        s.template load<false>(g[1 - b], c + 1);
        if (SPAN::PIECES == 1) vectors(next, c + 1, 0);
        SPAN::exchange(g[b], place, all);
        s.template tiles<false, NT, X>(g[b], c, 0, all, raw[set], acc);
        if (SPAN::PIECES > 1) vectors(next, c + 1, 0);
        multiply_rest(b, c);
    };
    const auto last = [&](int b, int c) {
        rest(c);
        SPAN::exchange(g[b], place, all);
        s.template tiles<false, NT, X>(g[b], c, 0, all, raw[SPAN::PIECES > 1 ? 0 : b], acc);
        multiply_rest(b, c);
    };
    int c = sh.first;
    if (c < sh.whole) {
        s.template load<false>(g[0], c);
        vectors(0, c, 0);
        for (;;) {
            if (c + 1 >= sh.whole) { last(0, c++); break; }
            step(0, c++);
            if (c + 1 >= sh.whole) { last(1, c++); break; }
            step(1, c++);
        }
    }
    if (c < sh.end) {
        s.template load<true>(g[0], c);
        SPAN::exchange(g[0], place, all);
#pragma unroll
        for (int h = 0; h < SPAN::PIECES; ++h) {
            vectors(0, c, h);
            s.template tiles<true, NT, X>(g[0], c, h, all, raw[0], acc);
        }
    }
}

// One lane's part of the copy: block `block` of the row that x points at.
template <class SPAN, class X>
__device__ __forceinline__ void copy_block(const X &x, int cols, int block, int lane, v4u *tile)
{
    const int k = copied_column(block, lane >> 4, SPAN::SPREAD);
    typename X::Raw raw;
    x.template load<true>(raw, k, cols);
    v4u v[X::P];
    X::operands(raw, v);
#pragma unroll
    for (int q = 0; q < X::P; ++q) tile[(block * X::P + q) * 64 + lane] = SPAN::CODES ? code_order<SPAN::T>(v[q]) : v[q];
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

// ---- 4-bit weights and tiles of vectors, the vectors kept
// A tile takes a kilobyte of vectors for each 256 bytes of weights.  So a wave keeps the vectors of its 256 columns in registers, and
// the weights of one set of 16 R rows after the other pass by; the KW waves of a workgroup share up to 256 KW columns, their sums meet in LDS
// for every set.  Scales and zero points of a set lie far apart, row by row, and would cost as much as the weights where each lane
// loads its own: all threads bring them to LDS, a set ahead.
constexpr int KEPT_CHUNK = 256, KEPT_COLUMNS = 16 * KEPT_CHUNK;
inline bool kept_fits(const WeightsQ4 &A) { return A.cols <= KEPT_COLUMNS && A.ld_codes < (1 << 26) && A.ld_scales < (1 << 24); }
template <int KW, int R, int GB, int S>
struct KeptSpace {
    typedef typename std::conditional<S == F32, float, unsigned short>::type Scale;
    static constexpr int GROUPS = KW * 8 / GB, LD = GROUPS + (S == F32 ? 4 : 8), LDZ = GROUPS + 16;     // a row's neighbours on other banks
    float sums[2][KW * R * 256];
    v4u places[KW * EXCHANGE];
    __align__(16) Scale s[2][R][16][LD];
    __align__(16) unsigned char z[2][R][16][LDZ];
};
template <int T, int R, int GB, int S, int KW, class X>
struct KeptQ4 {
    typedef KeptSpace<KW, R, GB, S> Space;
    typedef typename Space::Scale Scale;
    static constexpr int THREADS = 64 * KW, NG = GB < 8 ? 8 / GB : 1, PER = GB < 4 ? GB : 4;
    static constexpr bool SCALED = std::is_same<X, Scaled>::value;
    static constexpr float unit = SCALED ? 0x1p9f : code_unit<T>;
    static constexpr int E = GB == 1 ? 2 : 1;              // scales of 16 rows that a thread brings: 2 / GB for each of them
    Space &sp;
    const WeightsQ4 (&w)[R];
    int64_t m;
    int rows, cols, c, lane, wave;
    bool any, partial;                                     // whether the wave has columns, and fewer than a chunk
    typename Copied<X>::Raw x[2][4];
    int lift[4];                                           // SCALED: powers of two of the lane's four vectors, less those of unit (as code_unit)
    v4u g[2][R][2];
    Scale s[R][E];
    unsigned char z[R][E];
    Exchange place;
    __device__ __forceinline__ KeptQ4(Space &space, const WeightsQ4 (&weights)[R], int64_t matrix, int n_rows, int n_cols)
        : sp(space), w(weights), m(matrix), rows(n_rows), cols(n_cols), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)),
          place(space.places + EXCHANGE * wave, lane)
    {
        asm volatile("" : "+v"(lane));                     // (nothing is kept for the next tile of vectors)
        c = wave;
        any = c * KEPT_CHUNK < cols;
        partial = (c + 1) * KEPT_CHUNK > cols;
    }
    // Weights and scales of a set.  Where it begins is computed once per wave, a lane's offset from there has 32 bits (KeptQ4 is for such
    // leading dimensions).  A thread with none of the scales brings one that another thread brings too, and past the last set all lanes
    // load from where the matrix begins: a load under a condition would be waited for with all others.
    template <int B>
    __device__ __forceinline__ void request(int set, int sets)
    {
        const unsigned real = set < sets ? ~0u : 0u;
        const int row0 = set < sets ? 16 * set : 0, last = rows - 1 - row0;
        // the scales before the weights: they are waited for first, and loads arrive in their order
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t at = m * w[r].stride_scales + row0 * w[r].ld_scales;
            const Scale *scales = static_cast<const Scale *>(w[r].scales) + at;
            const unsigned char *zeros = w[r].zeros ? w[r].zeros + at : w[r].codes;            // (no load under a condition)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int i = threadIdx.x + e * THREADS, row = min(i / Space::GROUPS % 16, last), group = min(i % Space::GROUPS, (cols - 1) >> w[0].shift);
                const unsigned off = ((unsigned)row * (unsigned)w[r].ld_scales + group) & real;
                s[r][e] = scales[off];
                z[r][e] = zeros[w[r].zeros ? off : 0u];
            }
        }
        const unsigned k = c * KEPT_CHUNK + 32 * load_piece(lane);                // past the last column, the row's beginning: its products are with zeros
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const unsigned char *base = w[r].codes + m * w[r].stride_codes + row0 * w[r].ld_codes;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                g[B][r][i] = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(
                    base + (((unsigned)min(load_row(lane, i), last) * (unsigned)w[r].ld_codes + ((int)k < cols ? k / 2 : 0u)) & real)));
        }
    }
    template <int B>
    __device__ __forceinline__ void put_scales()
    {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int i = threadIdx.x + e * THREADS, row = i / Space::GROUPS % 16, group = i % Space::GROUPS;
                sp.s[B][r][row][group] = s[r][e];
                sp.z[B][r][row][group] = w[r].zeros ? z[r][e] : (unsigned char)8;
            }
    }
    static __device__ __forceinline__ float factor(Scale v)
    {
        if constexpr (S == F32) return v;
        else return widen<S>(v);
    }
    template <int B>
    __device__ __forceinline__ void multiply()
    {
        v4f acc[R];
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r] = v4f{0, 0, 0, 0};
        if (any) {
            const int g0 = GB <= 8 ? c * (8 / (GB < 8 ? GB : 8)) : 0;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (r) __builtin_amdgcn_sched_barrier(0);      // one after the other: together they take more registers than four waves may have
                v4u all[2];
                place(g[B][r], all);
                Scale fs[NG];
                unsigned char zs[NG];
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    const int at = GB == 8 ? (c * KEPT_CHUNK) >> w[0].shift : g0 + i;
                    fs[i] = sp.s[B][r][lane & 15][at];
                    zs[i] = sp.z[B][r][lane & 15][at];
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const v4u words = transpose_quarters(all[h]);
#pragma unroll
                    for (int i = 0; i < 4 / PER; ++i) {
                        const int at = 4 * h / GB + i;
                        const Zero<T> zero((int)zs[at]);
                        v4f sum = v4f{0, 0, 0, 0};
#pragma unroll
                        for (int b = 0; b < PER; ++b) sum = product<T, X>(x[h][i * PER + b].v, dequantise(words[i * PER + b], zero), sum);
                        // a block past the last column counts nothing: its sum is zero, and so has the scale to be
                        const float f = c * KEPT_CHUNK + 128 * h + 32 * PER * i < cols ? factor(fs[at]) : 0.0f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[r][e] = fmaf(SCALED ? __builtin_amdgcn_ldexpf(sum[e], lift[e]) : sum[e], f, acc[r][e]);
                    }
                }
            }
        }
        put_sums<R>(sp.sums[B], wave, lane, acc);
    }
    // Sets first, first + step, ... before `sets`; done(set, sums) takes over the sums of one.
    template <class DONE>
    __device__ __forceinline__ void run(int set, int step, int sets, DONE done)
    {
        request<0>(set, sets);
        put_scales<0>();
        __syncthreads();
        while (one<0>(set, step, sets, done) && one<1>(set, step, sets, done)) {}
        __syncthreads();                                   // (the next tile's first set)
    }
    template <int B, class DONE>
    __device__ __forceinline__ bool one(int &set, int step, int sets, DONE done)
    {
        request<1 - B>(set + step, sets);
        multiply<B>();
        put_scales<1 - B>();
        __syncthreads();
        done(set, sp.sums[B]);
        set += step;
        return set < sets;
    }
};
// The vectors of the wave's columns: from a copy in natural order,
template <class K, class X>
__device__ __forceinline__ void keep_copied(K &k, const Copied<X> &x)
{
    if (k.any) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) x.load(k.x[h][j], 8 * k.c + 4 * h + j);
    }
}
// or from one of 32 bits, where 16 bytes of a lane are two times 16 (vectors from `live` on repeat the one before),
template <class K>
__device__ __forceinline__ void keep_scaled(K &k, const v4f *copy, int live)
{
    if (!k.any) return;
    v4f v[8][2];
    float top = 0;
#pragma unroll
    for (int b = 0; b < 8; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e) v[b][e] = copy[((8 * k.c + b) * 2 + e) * 64 + (k.lane & 48) + min(k.lane & 15, live - 1)];
#pragma unroll
    for (int b = 0; b < 8; ++b)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            top = fmaxf(top, __builtin_fabsf(v[b][e >> 2][e & 3]));
        }
    top = fmaxf(top, __shfl_xor(top, 16, WAVE));
    top = fmaxf(top, __shfl_xor(top, 32, WAVE));
    // (with an infinity no sum of its vector is finite, whatever the others are rounded to)
    const int up = 15 - __builtin_amdgcn_frexp_expf(fminf(top, __FLT_MAX__));
#pragma unroll
    for (int b = 0; b < 8; ++b) Scaled::operands(v[b], up, k.x[b >> 2][b & 3].v);
#pragma unroll
    for (int i = 0; i < 4; ++i) k.lift[i] = -9 - __shfl(up, 4 * (k.lane >> 4) + i, WAVE);
}
// or 16-bit vectors 16 tile and on as they are, whole lines at a time, through LDS like the weights.
template <int T, class K>
__device__ __forceinline__ void keep_rows(K &k, const unsigned short *X, int64_t ldx, int n, int tile)
{
    if (!k.any) return;
    v4u w[4][2], o[2];
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const unsigned short *p = X + min(16 * tile + load_row(k.lane, i), n - 1) * ldx + 8 * load_piece(k.lane);
            const int at = KEPT_CHUNK * k.c + 64 * b;
            w[b][i] = k.partial ? load8(p, at, k.cols - 8 * load_piece(k.lane)) : *reinterpret_cast<const v4u_u *>(p + at);
        }
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        k.place(w[b], o);
#pragma unroll
        for (int i = 0; i < 2; ++i) k.x[b >> 1][2 * (b & 1) + i].v[0] = code_order<T>(o[i]);
    }
}

}  // namespace psk
