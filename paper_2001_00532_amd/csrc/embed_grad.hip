// The gradient of the embedding lookup (formulas: embed.h): the product by the transpose of S.
//
// Tokens are sorted (a stable sort by digits, so a row's positions ascend and its sum has one order), and the sorted positions are cut into equal
// tiles, as the stored entries of any sparse operand here: a tile adds up the rows of dY of its positions and writes the rows of dE that
// begin and end in it.  Of a row that spans tiles, each tile leaves its part in 32 bits, and a third step adds the parts in order.
// Rows that no token has are cleared beside the tiles.  Bound by reading dY and writing dE.
#include "embed.h"

namespace psk {
namespace {

constexpr int SORT = 2048;                                 // positions per workgroup of the sort
constexpr int MAX_BITS = 9;                                // of a digit

// Key of a position: its token, or `rows` for one that is in no row.
__device__ __forceinline__ int key_of(const int *ids, int64_t t, int rows, int padding)
{
    const int id = ids[t];
    return (unsigned)id >= (unsigned)rows || id == padding ? rows : id;
}

// FIRST: keys come from the tokens, and a position is its own place.
template <bool FIRST>
__global__ __launch_bounds__(256) void k_sort_count(const int *__restrict__ keys, int n, int rows, int padding, int shift, int bits, int *__restrict__ count)
{
    __shared__ int s[1 << MAX_BITS];
    for (int d = threadIdx.x; d < 1 << bits; d += 256) s[d] = 0;
    __syncthreads();
    const int begin = blockIdx.x * SORT;
    for (int i = threadIdx.x; i < SORT && begin + i < n; i += 256) {
        const int k = FIRST ? key_of(keys, begin + i, rows, padding) : keys[begin + i];
        atomicAdd(&s[k >> shift & ((1 << bits) - 1)], 1);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < 1 << bits; d += 256) count[(int64_t)d * gridDim.x + blockIdx.x] = s[d];
}

// Lanes of the wave with the same digit as this one, of those that have one.
__device__ __forceinline__ unsigned long long same_digit(int d, int bits, bool valid)
{
    unsigned long long m = __ballot(valid);
    for (int b = 0; b < bits; ++b) {
        const unsigned long long one = __ballot(d >> b & 1);
        m &= d >> b & 1 ? one : ~one;
    }
    return m;
}

// A wave takes a quarter of the workgroup's positions, 64 at a time in order.
template <bool FIRST>
__global__ __launch_bounds__(256) void k_sort_place(const int *__restrict__ keys, const int *__restrict__ at, int n, int rows, int padding, int shift, int bits,
                                                    const int *__restrict__ base, int *__restrict__ keys_out, int *__restrict__ at_out)
{
    constexpr int ROUNDS = SORT / 256;
    __shared__ int s[4][1 << MAX_BITS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, begin = blockIdx.x * SORT + wave * (SORT / 4);
    for (int d = threadIdx.x; d < 4 << bits; d += 256) s[d >> bits][d & ((1 << bits) - 1)] = 0;
    __syncthreads();
    int key[ROUNDS], rank[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i = begin + 64 * r + lane;
        const bool valid = i < n;
        key[r] = valid ? (FIRST ? key_of(keys, i, rows, padding) : keys[i]) : 0;
        const int d = key[r] >> shift & ((1 << bits) - 1);
        const unsigned long long same = same_digit(d, bits, valid);
        const int before = __popcll(same & ((1ull << lane) - 1));
        rank[r] = valid ? s[wave][d] + before : 0;
        wave_fence();
        if (valid && before == 0) s[wave][d] += __popcll(same);
        wave_fence();
    }
    __syncthreads();
    for (int d = threadIdx.x; d < 1 << bits; d += 256) {
        int sum = base[(int64_t)d * gridDim.x + blockIdx.x];
        for (int w = 0; w < 4; ++w) {
            const int c = s[w][d];
            s[w][d] = sum;
            sum += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i = begin + 64 * r + lane;
        if (i >= n) break;
        const int to = s[wave][key[r] >> shift & ((1 << bits) - 1)] + rank[r];
        keys_out[to] = key[r];
        at_out[to] = FIRST ? i : at[i];
    }
}

// ------------------------------------------------------------------ sums
constexpr int TILE = 64;                                   // positions per tile, one to a lane
constexpr int CHUNK = 512;                                 // columns per wave, eight to a lane

struct Grad {
    int n, rows, dim, accumulate;
    const int *keys, *at;
    const void *dY;
    int64_t ldy;
    void *dE;
    int64_t lde;
    float factor;
    float *head, *tail;                                    // of each tile, dim: the part of a row that began before it, of one that goes on behind it
};

template <int GT>
__device__ __forceinline__ void put_element(const Grad &g, int64_t at, float sum)
{
    const float v = g.factor * sum;
    store_as<GT>(g.dE, at, g.accumulate ? element<GT>(g.dE, at) + v : v);
}
// Eight columns of row `row` of dE from column u.col on, without the first u.skip.
template <int GT>
__device__ __forceinline__ void put_row(const Grad &g, int row, Unit u, const float (&sum)[8])
{
    typedef typename Bits<GT>::type B;
    const int64_t at = row * g.lde + u.col;
    if (u.skip == 0) {
        float v[8];
        B *p = static_cast<B *>(g.dE) + at;
        if (g.accumulate) {
            Raw8<GT> r;
            load_raw<GT>(r, p);
            widen_raw<GT>(r, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += g.factor * sum[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = g.factor * sum[i];
        }
        store8<GT>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= u.skip) put_element<GT>(g, at + i, sum[i]);
    }
}

// One wave: the tile's positions, columns from `unit` of this lane on.
template <int T, int GT>
__device__ __forceinline__ void tile_sum(const Grad &g, int tile, int chunk, int lane)
{
    constexpr int U = 8;                                   // rows of dY in flight
    typedef typename Bits<T>::type B;
    const int p0 = tile * TILE, count = min(TILE, g.n - p0), p = min(p0 + lane, g.n - 1);
    const int key = g.keys[p], at = g.at[p];
    const int before = p0 > 0 ? g.keys[p0 - 1] : -1, behind = p0 + count < g.n ? g.keys[p0 + count] : -1;
    const int next = __shfl_down(key, 1);
    // positions behind which a row ends within the tile, and those that are in a row at all
    const bool last = lane == count - 1;
    const unsigned long long ends = __ballot(lane < count && (last || next != key));
    const int valid = __popcll(__ballot(lane < count && key < g.rows));
    const int unit = chunk * (CHUNK / 8) + lane;
    const bool mine = 8 * unit < g.dim;
    const Unit u = unit_of(mine ? unit : 0, g.dim);
    float sum[8] = {};
    for (int i = 0; i < valid; i += U) {
        Raw8<T> r[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int64_t row = rl(at, min(i + j, valid - 1));
            load_raw<T>(r[j], static_cast<const B *>(g.dY) + row * g.ldy + u.col);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (i + j >= valid) break;
            float v[8];
            widen_raw<T>(r[j], v);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += v[k];
            if (ends >> (i + j) & 1) {
                const int row = rl(key, i + j);
                const bool began = row != before, goes_on = i + j == count - 1 && row == behind;
                if (mine) {
                    if (began && !goes_on) {
                        put_row<GT>(g, row, u, sum);
                    } else {
                        float *to = (began ? g.tail : g.head) + (int64_t)tile * g.dim + u.col;
                        *reinterpret_cast<v4f_e *>(to) = v4f{sum[0], sum[1], sum[2], sum[3]};      // what is there twice is the same
                        *reinterpret_cast<v4f_e *>(to + 4) = v4f{sum[4], sum[5], sum[6], sum[7]};
                    }
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
            }
        }
    }
}

// Rows of less than eight columns: a wave per tile, a lane per column.
template <int T, int GT>
__device__ __forceinline__ void tile_sum_narrow(const Grad &g, int tile, int lane)
{
    const int p0 = tile * TILE, p1 = min(p0 + TILE, g.n);
    if (lane >= g.dim) return;
    const int before = p0 > 0 ? g.keys[p0 - 1] : -1, behind = p1 < g.n ? g.keys[p1] : -1;
    float sum = 0.0f;
    for (int p = p0; p < p1; ++p) {
        const int row = g.keys[p];
        if (row >= g.rows) break;
        sum += element<T>(g.dY, g.at[p] * g.ldy + lane);
        if (p + 1 < p1 && g.keys[p + 1] == row) continue;
        const bool began = row != before, goes_on = p == p1 - 1 && row == behind;
        if (began && !goes_on) put_element<GT>(g, row * g.lde + lane, sum);
        else (began ? g.tail : g.head)[(int64_t)tile * g.dim + lane] = sum;
        sum = 0.0f;
    }
}

// A wave clears those of 64 rows that no token has.
template <int GT>
__device__ __forceinline__ void clear_rows(const Grad &g, int64_t first, int lane)
{
    typedef typename Bits<GT>::type B;
    const int row = (int)min(first + lane, (int64_t)g.rows - 1);
    int lo = 0, hi = g.n;                                  // the first position whose key is not less than row
    while (lo < hi) {
        const int mid = (int)(((unsigned)lo + (unsigned)hi) >> 1);
        if (g.keys[mid] < row) lo = mid + 1;
        else hi = mid;
    }
    unsigned long long empty = __ballot(first + lane < g.rows && !(lo < g.n && g.keys[lo] == row));
    const float zeros[8] = {};
    for (; empty; empty &= empty - 1) {
        B *p = static_cast<B *>(g.dE) + (first + __builtin_ctzll(empty)) * g.lde;
        if (g.dim < 8) {
            if (lane < g.dim) p[lane] = B(0);
        } else {
            for (int unit = lane; 8 * unit < g.dim; unit += 64) store8<GT>(p + unit_of(unit, g.dim).col, zeros);
        }
    }
}

template <int T, int GT>
__global__ __launch_bounds__(256) void k_grad_sum(Grad g, int tiles, int chunks, int64_t sums, int64_t all)
{
    const int lane = threadIdx.x & 63;
    for (int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); w < all; w += (int64_t)gridDim.x * 4) {
        if (w >= sums) clear_rows<GT>(g, (w - sums) * 64, lane);
        else if (g.dim < 8) tile_sum_narrow<T, GT>(g, (int)w, lane);
        else tile_sum<T, GT>(g, (int)(w / chunks), (int)(w % chunks), lane);
    }
}

// A row that begins in a tile and goes on behind it: its parts in order.  A wave per tile and chunk of columns.
template <int GT>
__global__ __launch_bounds__(256) void k_grad_join(Grad g, int tiles, int chunks)
{
    const int lane = threadIdx.x & 63;
    const int64_t all = (int64_t)tiles * chunks;
    for (int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); w < all; w += (int64_t)gridDim.x * 4) {
        const int tile = (int)(w / chunks), p0 = tile * TILE, p1 = p0 + TILE;
        if (p1 >= g.n) continue;
        const int row = g.keys[p1 - 1];
        if (row >= g.rows || g.keys[p1] != row || (p0 > 0 && g.keys[p0 - 1] == row)) continue;
        const int unit = (int)(w % chunks) * (CHUNK / 8) + lane;
        if (g.dim < 8 ? lane >= g.dim : 8 * unit >= g.dim) continue;
        if (g.dim < 8) {
            float sum = g.tail[(int64_t)tile * g.dim + lane];
            for (int t = tile + 1; t < tiles && g.keys[t * TILE] == row; ++t) sum += g.head[(int64_t)t * g.dim + lane];
            put_element<GT>(g, row * g.lde + lane, sum);
            continue;
        }
        const Unit u = unit_of(unit, g.dim);
        float sum[8];
        Raw8<F32> r;
        load_raw<F32>(r, g.tail + (int64_t)tile * g.dim + u.col);
        widen_raw<F32>(r, sum);
        for (int t = tile + 1; t < tiles && g.keys[t * TILE] == row; ++t) {
            float v[8];
            load_raw<F32>(r, g.head + (int64_t)t * g.dim + u.col);
            widen_raw<F32>(r, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
        }
        put_row<GT>(g, row, u, sum);
    }
}

struct Space {
    int *keys[2], *at[2], *count, *scan;
    float *head, *tail;
    size_t bytes;
};
Space carve_grad(void *base, int64_t n, int64_t dim)
{
    char *p = static_cast<char *>(base);
    size_t used = 0;
    auto take = [&](size_t bytes) {
        char *const q = p + used;
        used += align256(bytes + 1);
        return q;
    };
    const int64_t blocks = (n + SORT - 1) / SORT, tiles = (n + TILE - 1) / TILE, counts = blocks << MAX_BITS;
    Space w;
    for (int i = 0; i < 2; ++i) {
        w.keys[i] = reinterpret_cast<int *>(take((size_t)n * 4));
        w.at[i] = reinterpret_cast<int *>(take((size_t)n * 4));
    }
    w.count = reinterpret_cast<int *>(take((size_t)counts * 4));
    w.scan = reinterpret_cast<int *>(take(scan_tmp_ints(counts) * 4));
    w.head = reinterpret_cast<float *>(take((size_t)tiles * (size_t)dim * 4));
    w.tail = reinterpret_cast<float *>(take((size_t)tiles * (size_t)dim * 4));
    w.bytes = used;
    return w;
}

unsigned grid_of(int64_t waves)
{
    const int64_t blocks = (waves + 3) / 4;
    return (unsigned)(blocks < 65536 ? blocks : 65536);
}

template <int T, int GT>
void sums(const Grad &g, hipStream_t s)
{
    const int tiles = (g.n + TILE - 1) / TILE, chunks = g.dim < 8 ? 1 : (g.dim + CHUNK - 1) / CHUNK;
    const int64_t sums = (int64_t)tiles * chunks, all = sums + (g.accumulate ? 0 : ((int64_t)g.rows + 63) / 64);
    PSK_LAUNCH((k_grad_sum<T, GT>), dim3(grid_of(all)), dim3(256), 0, s, g, tiles, chunks, sums, all);
    if (tiles > 1) PSK_LAUNCH((k_grad_join<GT>), dim3(grid_of(sums)), dim3(256), 0, s, g, tiles, chunks);
}

}  // namespace

size_t embed_grad_workspace_bytes(int64_t n, int64_t dim) { return carve_grad(nullptr, n, dim).bytes; }

hipError_t launch_embed_grad(int n, int rows, int dim, const int *ids, int padding, float factor, int type, const void *dY, int64_t ldy, int gtype, void *dE,
                             int64_t lde, int accumulate, void *workspace, hipStream_t s)
{
    const Space w = carve_grad(workspace, n, dim);
    const unsigned blocks = (unsigned)((n + SORT - 1) / SORT);
    int bits = 1;
    while (rows >> bits) ++bits;                           // keys are 0 .. rows
    const int passes = (bits + MAX_BITS - 1) / MAX_BITS, each = (bits + passes - 1) / passes;
    const int *keys = ids, *at = nullptr;
    for (int pass = 0; n > 0 && pass < passes; ++pass) {
        const int shift = pass * each;
        if (pass == 0) PSK_LAUNCH((k_sort_count<true>), dim3(blocks), dim3(256), 0, s, keys, n, rows, padding, shift, each, w.count);
        else PSK_LAUNCH((k_sort_count<false>), dim3(blocks), dim3(256), 0, s, keys, n, rows, padding, shift, each, w.count);
        const hipError_t e = launch_exclusive_scan(w.count, w.count, (int64_t)blocks << each, w.scan, s);
        if (e != hipSuccess) return e;
        int *const k = w.keys[pass & 1], *const a = w.at[pass & 1];
        if (pass == 0) PSK_LAUNCH((k_sort_place<true>), dim3(blocks), dim3(256), 0, s, keys, at, n, rows, padding, shift, each, w.count, k, a);
        else PSK_LAUNCH((k_sort_place<false>), dim3(blocks), dim3(256), 0, s, keys, at, n, rows, padding, shift, each, w.count, k, a);
        keys = k;
        at = a;
    }
    const Grad g = {n, rows, dim, accumulate, keys, at, dY, ldy, dE, lde, factor, w.head, w.tail};
    if (type == F32) sums<F32, F32>(g, s);
    else if (type == F16) gtype == F32 ? sums<F16, F32>(g, s) : sums<F16, F16>(g, s);
    else gtype == F32 ? sums<BF16, F32>(g, s) : sums<BF16, BF16>(g, s);
    return take_launch_status();
}

}  // namespace psk
