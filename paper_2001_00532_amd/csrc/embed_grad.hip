// The gradient of the embedding lookup (formulas: embed.h): the product by the transpose of S.
//
// Tokens are sorted (a stable sort by digits, so a row's positions ascend and its sum has one order), and the sorted positions are cut into equal
// tiles, as the stored entries of any sparse operand here: a tile adds up the rows of dY of its positions and writes the rows of dE that
// begin and end in it.  Of a row that spans tiles, each tile leaves its part in 32 bits, and a third step adds the parts in order.
// Rows that no token has are cleared beside the tiles.  Bound by reading dY and writing dE.
#include "embed.h"

namespace psk {
namespace {

constexpr int SORT = 2048;                                 // positions per workgroup where several sort
constexpr int ONE = 16384;                                 // positions that one workgroup sorts by itself
constexpr int MAX_BITS = 9;                                // of a digit
constexpr int BASES = 128;                                 // workgroups whose counts every one of them adds up by itself

// Key of a position: its token, or `rows` for one that is in no row.
__device__ __forceinline__ int key_of(const int *ids, int64_t t, int rows, int padding)
{
    const int id = ids[t];
    return (unsigned)id >= (unsigned)rows || id == padding ? rows : id;
}

// ------------------------------------------------------------------ rows without a token
struct Clear {
    void *dE;
    int64_t lde;
    int rows, dim;
};
constexpr int RANGE = 1 << 15;                             // rows whose bits are in LDS at once

// L lanes to a row.
template <int GT>
__device__ __forceinline__ void clear_row(const Clear &c, int64_t row, int sub, int lanes)
{
    typedef typename Bits<GT>::type B;
    B *const p = static_cast<B *>(c.dE) + row * c.lde;
    const float zeros[8] = {};
    if (c.dim < 8) {
        if (sub < c.dim) p[sub] = B(0);
    } else {
        for (int unit = sub; 8 * unit < c.dim; unit += lanes) store8<GT>(p + unit_of(unit, c.dim).col, zeros);
    }
}
__device__ __forceinline__ int lanes_log(int dim)
{
    int log = 3;
    while (log < 6 && (8 << log) < dim) ++log;
    return log;
}
// Beside the sort: workgroup `part` of `parts` reads all tokens and clears those of its rows that none of them names.
template <int GT, int THREADS>
__device__ __forceinline__ void clear_unnamed(const Clear &c, const int *__restrict__ ids, int n, int padding, int part, int parts, unsigned *bits)
{
    const int64_t per = ((int64_t)c.rows + parts - 1) / parts, begin = part * per, end = min(begin + per, (int64_t)c.rows);
    const int log = lanes_log(c.dim), sub = threadIdx.x & ((1 << log) - 1);
    for (int64_t first = begin; first < end; first += RANGE) {
        const int count = (int)min(end - first, (int64_t)RANGE);
        for (int i = threadIdx.x; i < (count + 31) / 32; i += THREADS) bits[i] = 0;
        __syncthreads();
        for (int t = threadIdx.x; t < n; t += THREADS) {
            const int id = ids[t];
            const int64_t at = id - first;
            if (id != padding && at >= 0 && at < count) atomicOr(&bits[at >> 5], 1u << (at & 31));
        }
        __syncthreads();
        for (int r = threadIdx.x >> log; r < count; r += THREADS >> log)
            if (!(bits[r >> 5] >> (r & 31) & 1)) clear_row<GT>(c, first + r, sub, 1 << log);
        __syncthreads();
    }
}
// Behind the sort: a workgroup clears those of 256 rows that are no key.
template <int GT>
__device__ __forceinline__ void clear_absent(const Clear &c, const int *__restrict__ keys, int n, int64_t first, unsigned long long *empty)
{
    const int row = (int)min(first + threadIdx.x, (int64_t)c.rows - 1);
    int lo = 0, hi = n;                                    // the first position whose key is not less than row
    while (lo < hi) {
        const int mid = (int)(((unsigned)lo + (unsigned)hi) >> 1);
        if (keys[mid] < row) lo = mid + 1;
        else hi = mid;
    }
    const unsigned long long m = __ballot(first + threadIdx.x < c.rows && !(lo < n && keys[lo] == row));
    __syncthreads();                                       // the last rows' bits have been read
    if ((threadIdx.x & 63) == 0) empty[threadIdx.x >> 6] = m;
    __syncthreads();
    const int log = lanes_log(c.dim), sub = threadIdx.x & ((1 << log) - 1);
    for (int r = threadIdx.x >> log; r < 256; r += 256 >> log)
        if (empty[r >> 6] >> (r & 63) & 1) clear_row<GT>(c, first + r, sub, 1 << log);
}

// ------------------------------------------------------------------ the sort
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
// Place of a position among those of its wave with the same digit, rounds of 64 positions in order; `seen`: the wave's count of each digit.
__device__ __forceinline__ int place_in_wave(int d, int bits, bool valid, int lane, int *seen)
{
    const unsigned long long same = same_digit(d, bits, valid);
    const int before = __popcll(same & ((1ull << lane) - 1));
    const int rank = valid ? seen[d] + before : 0;
    wave_fence();
    if (valid && before == 0) seen[d] += __popcll(same);
    wave_fence();
    return rank;
}
// Exclusive sums over the threads of a workgroup.
template <int THREADS>
__device__ __forceinline__ int block_exclusive(int v, int *part)
{
    int inc = v;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < WAVE; d *= 2) {
        const int o = __shfl_up(inc, d, WAVE);
        if (lane >= d) inc += o;
    }
    if (lane == 63) part[wave] = inc;
    __syncthreads();
    int sum = inc - v;
    for (int w = 0; w < wave; ++w) sum += part[w];
    __syncthreads();
    return sum;
}

// Up to ONE positions: the first workgroup sorts them, in LDS, while the others clear.  A wave owns a sixteenth of the positions, and each thread holds
// its own in registers while their order in LDS changes.
template <int GT, bool CLEAR>
__global__ __launch_bounds__(1024) void k_sort_one(const int *__restrict__ ids, int n, int padding, int digit, int passes, int *__restrict__ keys_out,
                                                   int *__restrict__ at_out, Clear c)
{
    constexpr int EACH = ONE / 1024, WAVES = 16;
    __shared__ int keys[ONE];
    __shared__ unsigned short at[ONE];
    __shared__ int seen[WAVES][1 << MAX_BITS];
    __shared__ int part[WAVES];
    if (CLEAR && blockIdx.x > 0) {
        clear_unnamed<GT, 1024>(c, ids, n, padding, blockIdx.x - 1, gridDim.x - 1, reinterpret_cast<unsigned *>(keys));
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, mask = (1 << digit) - 1;
    const int rounds = (n + 1023) / 1024;                  // of 64 positions per wave
    const int begin = wave * rounds * 64;
    int key[EACH], rank[EACH], from[EACH];
#pragma unroll
    for (int r = 0; r < EACH; ++r) {
        const int i = begin + 64 * r + lane;
        from[r] = i;
        key[r] = r < rounds && i < n ? key_of(ids, i, c.rows, padding) : c.rows;
    }
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * digit;
        for (int d = threadIdx.x; d < WAVES << MAX_BITS; d += 1024) (&seen[0][0])[d] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < EACH; ++r)
            if (r < rounds) rank[r] = place_in_wave(key[r] >> shift & mask, digit, begin + 64 * r + lane < n, lane, seen[wave]);
        __syncthreads();
        int sum = 0;
        if (threadIdx.x <= (unsigned)mask) {
            for (int w = 0; w < WAVES; ++w) {
                const int v = seen[w][threadIdx.x];
                seen[w][threadIdx.x] = sum;
                sum += v;
            }
        }
        const int base = block_exclusive<1024>(sum, part);
        if (threadIdx.x <= (unsigned)mask)
            for (int w = 0; w < WAVES; ++w) seen[w][threadIdx.x] += base;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < EACH; ++r) {
            const int i = begin + 64 * r + lane;
            if (r >= rounds || i >= n) continue;
            const int to = seen[wave][key[r] >> shift & mask] + rank[r];
            if (pass == passes - 1) {
                keys_out[to] = key[r];
                at_out[to] = from[r];
            } else {
                keys[to] = key[r];
                at[to] = (unsigned short)from[r];
            }
        }
        if (pass == passes - 1) break;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < EACH; ++r) {
            const int i = begin + 64 * r + lane;
            if (r >= rounds || i >= n) continue;
            key[r] = keys[i];
            from[r] = at[i];
        }
    }
}

// Several workgroups: they count their digits, and then put their positions behind those of smaller digits and of earlier workgroups.
// FIRST: keys come from the tokens, and a position is its own place; workgroups behind the counting ones clear.
template <bool FIRST, int GT>
__global__ __launch_bounds__(256) void k_sort_count(const int *__restrict__ keys, int n, int padding, int shift, int bits, int blocks, int *__restrict__ count,
                                                    Clear c)
{
    __shared__ int s[RANGE / 32];
    static_assert(RANGE / 32 >= 1 << MAX_BITS, "room for the counts");
    if (FIRST && (int)blockIdx.x >= blocks) {
        clear_unnamed<GT, 256>(c, keys, n, padding, blockIdx.x - blocks, gridDim.x - blocks, reinterpret_cast<unsigned *>(s));
        return;
    }
    for (int d = threadIdx.x; d < 1 << bits; d += 256) s[d] = 0;
    __syncthreads();
    const int begin = blockIdx.x * SORT;
    for (int i = threadIdx.x; i < SORT && begin + i < n; i += 256) {
        const int k = FIRST ? key_of(keys, begin + i, c.rows, padding) : keys[begin + i];
        atomicAdd(&s[k >> shift & ((1 << bits) - 1)], 1);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < 1 << bits; d += 256) count[(int64_t)d * blocks + blockIdx.x] = s[d];
}

// SCANNED: `count` holds the places where each workgroup's digits begin; otherwise the counts.  A wave takes a quarter of the workgroup's
// positions, 64 at a time in order.
template <bool FIRST, bool SCANNED>
__global__ __launch_bounds__(256) void k_sort_place(const int *__restrict__ keys, const int *__restrict__ at, int n, int rows, int padding, int shift, int bits,
                                                    const int *__restrict__ count, int *__restrict__ keys_out, int *__restrict__ at_out)
{
    constexpr int ROUNDS = SORT / 256, DIGITS = (1 << MAX_BITS) / 256;
    __shared__ int s[4][1 << MAX_BITS];
    __shared__ int part[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, begin = blockIdx.x * SORT + wave * (SORT / 4), blocks = gridDim.x;
    for (int d = threadIdx.x; d < 4 << MAX_BITS; d += 256) (&s[0][0])[d] = 0;
    // a thread's digits are neighbours: sums of the smaller ones are sums over the threads before
    int base[DIGITS];
#pragma unroll
    for (int e = 0; e < DIGITS; ++e) base[e] = 0;
    if constexpr (SCANNED) {
#pragma unroll
        for (int e = 0; e < DIGITS; ++e) {
            const int d = threadIdx.x * DIGITS + e;
            if (d < 1 << bits) base[e] = count[(int64_t)d * blocks + blockIdx.x];
        }
        __syncthreads();
    } else {
        int all[DIGITS], sum = 0;
#pragma unroll
        for (int e = 0; e < DIGITS; ++e) {
            const int d = threadIdx.x * DIGITS + e;
            all[e] = 0;
            for (int b = 0; d < 1 << bits && b < blocks; ++b) {
                const int v = count[(int64_t)d * blocks + b];
                if (b < (int)blockIdx.x) base[e] += v;
                all[e] += v;
            }
            sum += all[e];
        }
        int smaller = block_exclusive<256>(sum, part);
#pragma unroll
        for (int e = 0; e < DIGITS; ++e) {
            base[e] += smaller;
            smaller += all[e];
        }
    }
    int key[ROUNDS], rank[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i = begin + 64 * r + lane;
        key[r] = i < n ? (FIRST ? key_of(keys, i, rows, padding) : keys[i]) : 0;
    }
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) rank[r] = place_in_wave(key[r] >> shift & ((1 << bits) - 1), bits, begin + 64 * r + lane < n, lane, s[wave]);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < DIGITS; ++e) {
        const int d = threadIdx.x * DIGITS + e;
        int sum = base[e];
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

template <int T, int GT>
__global__ __launch_bounds__(256) void k_grad_sum(Grad g, int chunks, int64_t sums, int64_t all)
{
    __shared__ unsigned long long empty[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t b = blockIdx.x; b < all; b += gridDim.x) {
        const int64_t w = b * 4 + wave;
        if (b * 4 >= sums) clear_absent<GT>(Clear{g.dE, g.lde, g.rows, g.dim}, g.keys, g.n, (b - (sums + 3) / 4) * 256, empty);
        else if (w >= sums) continue;
        else if (g.dim < 8) tile_sum_narrow<T, GT>(g, (int)w, lane);
        else tile_sum<T, GT>(g, (int)(w / chunks), (int)(w % chunks), lane);
    }
}

// A row that begins in a tile and goes on behind it: its parts in order, a quarter of them to a wave, whose sums meet in LDS.  A workgroup per tile
// and chunk of columns; most have nothing to do.
template <int GT>
__global__ __launch_bounds__(256) void k_grad_join(Grad g, int tiles, int chunks)
{
    constexpr int U = 8;                                   // parts in flight
    __shared__ float meet[3][64][8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t all = (int64_t)tiles * chunks;
    for (int64_t w = blockIdx.x; w < all; w += gridDim.x) {
        const int tile = (int)(w / chunks), p0 = tile * TILE, p1 = p0 + TILE;
        if (p1 >= g.n) continue;
        const int row = g.keys[p1 - 1];
        if (row >= g.rows || g.keys[p1] != row || (p0 > 0 && g.keys[p0 - 1] == row)) continue;
        int more = 0;                                      // tiles behind it that begin with the row
        for (;;) {
            const int t = tile + 1 + more + lane;
            const int same = __builtin_ctzll(~__ballot(t < tiles && g.keys[t < tiles ? t * TILE : 0] == row) | (1ull << 63));
            more += same;                                  // at most 63 of a round
            if (same < 63) break;
        }
        const bool narrow = g.dim < 8;
        const int unit = (int)(w % chunks) * (CHUNK / 8) + lane;
        const bool mine = narrow ? lane < g.dim : 8 * unit < g.dim;
        const Unit u = narrow ? Unit{mine ? lane : 0, 0} : unit_of(mine ? unit : 0, g.dim);
        const int each = (more + 3) / 4, from = min(wave * each, more), to = min(from + each, more);
        const float *const head = g.head + (int64_t)(tile + 1) * g.dim + u.col;
        float sum[8] = {};
        if (narrow) {
            for (int i = from; i < to; ++i) sum[0] += head[(int64_t)i * g.dim];
        } else {
            for (int i = from; i < to; i += U) {
                Raw8<F32> r[U];
#pragma unroll
                for (int j = 0; j < U; ++j) load_raw<F32>(r[j], head + (int64_t)min(i + j, to - 1) * g.dim);
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    if (i + j >= to) break;
                    float v[8];
                    widen_raw<F32>(r[j], v);
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum[k] += v[k];
                }
            }
        }
        __syncthreads();                                   // the last row's sums have been read
        if (wave > 0) {
#pragma unroll
            for (int k = 0; k < 8; ++k) meet[wave - 1][lane][k] = sum[k];
        }
        __syncthreads();
        if (wave > 0 || !mine) continue;
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += meet[q][lane][k];
        const float *const tail = g.tail + (int64_t)tile * g.dim + u.col;
        if (narrow) {
            put_element<GT>(g, row * g.lde + lane, sum[0] + tail[0]);
        } else {
            float v[8];
            Raw8<F32> r;
            load_raw<F32>(r, tail);
            widen_raw<F32>(r, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += v[k];
            put_row<GT>(g, row, u, sum);
        }
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

unsigned at_most(int64_t blocks, int64_t most) { return (unsigned)(blocks < most ? blocks : most); }

// BESIDE: rows without a token are cleared in the launch of the sort's first step, by workgroups that read all tokens.  More than 64 K tokens
// take these longer than the search in the sorted ones.
template <int T, int GT>
hipError_t run(int n, int rows, int dim, const int *ids, int padding, float factor, const void *dY, int64_t ldy, void *dE, int64_t lde, int accumulate,
               const Space &w, hipStream_t s)
{
    const Clear c = {dE, lde, rows, dim};
    const bool beside = !accumulate && n > 0 && n <= 65536;
    const int blocks = (n + SORT - 1) / SORT;
    int bits = 1;
    while (rows >> bits) ++bits;                           // keys are 0 .. rows
    const int passes = (bits + MAX_BITS - 1) / MAX_BITS, digit = (bits + passes - 1) / passes;
    const int *keys = ids, *at = nullptr;
    if (n > 0 && n <= ONE) {
        const unsigned clear = beside ? at_most(((int64_t)rows + 15) / 16, 255) : 0;
        if (beside) PSK_LAUNCH((k_sort_one<GT, true>), dim3(1 + clear), dim3(1024), 0, s, ids, n, padding, digit, passes, w.keys[0], w.at[0], c);
        else PSK_LAUNCH((k_sort_one<GT, false>), dim3(1), dim3(1024), 0, s, ids, n, padding, digit, passes, w.keys[0], w.at[0], c);
        keys = w.keys[0];
        at = w.at[0];
    } else {
        for (int pass = 0; n > 0 && pass < passes; ++pass) {
            const int shift = pass * digit;
            const unsigned clear = beside && pass == 0 ? at_most(((int64_t)rows + 3) / 4, 1024) : 0;
            if (pass == 0) PSK_LAUNCH((k_sort_count<true, GT>), dim3(blocks + clear), dim3(256), 0, s, keys, n, padding, shift, digit, blocks, w.count, c);
            else PSK_LAUNCH((k_sort_count<false, GT>), dim3(blocks), dim3(256), 0, s, keys, n, padding, shift, digit, blocks, w.count, c);
            const bool scan = blocks > BASES;
            if (scan) {
                const hipError_t e = launch_exclusive_scan(w.count, w.count, (int64_t)blocks << digit, w.scan, s);
                if (e != hipSuccess) return e;
            }
            int *const k = w.keys[pass & 1], *const a = w.at[pass & 1];
            const auto place = pass == 0 ? (scan ? k_sort_place<true, true> : k_sort_place<true, false>) : (scan ? k_sort_place<false, true> : k_sort_place<false, false>);
            PSK_LAUNCH(place, dim3(blocks), dim3(256), 0, s, keys, at, n, rows, padding, shift, digit, w.count, k, a);
            keys = k;
            at = a;
        }
    }
    const Grad g = {n, rows, dim, accumulate, keys, at, dY, ldy, dE, lde, factor, w.head, w.tail};
    const int tiles = (n + TILE - 1) / TILE, chunks = dim < 8 ? 1 : (dim + CHUNK - 1) / CHUNK;
    const int64_t sums = (int64_t)tiles * chunks, all = (sums + 3) / 4 + (accumulate || beside ? 0 : ((int64_t)rows + 255) / 256);
    PSK_LAUNCH((k_grad_sum<T, GT>), dim3(at_most(all, 65536)), dim3(256), 0, s, g, chunks, sums, all);
    if (tiles > 1) PSK_LAUNCH((k_grad_join<GT>), dim3(at_most(sums, 65536)), dim3(256), 0, s, g, tiles, chunks);
    return take_launch_status();
}

}  // namespace

size_t embed_grad_workspace_bytes(int64_t n, int64_t dim) { return carve_grad(nullptr, n, dim).bytes; }

hipError_t launch_embed_grad(int n, int rows, int dim, const int *ids, int padding, float factor, int type, const void *dY, int64_t ldy, int gtype, void *dE,
                             int64_t lde, int accumulate, void *workspace, hipStream_t s)
{
    const Space w = carve_grad(workspace, n, dim);
    const auto go = type == F32 ? run<F32, F32> : (type == F16 ? (gtype == F32 ? run<F16, F32> : run<F16, F16>) : (gtype == F32 ? run<BF16, F32> : run<BF16, BF16>));
    return go(n, rows, dim, ids, padding, factor, dY, ldy, dE, lde, accumulate, w, s);
}

}  // namespace psk
