// The gradient of the embedding lookup (formulas: embed.h): the product by the transpose of S.
//
// Tokens are sorted (stably, so a row's positions ascend), and the sorted positions are cut into equal tiles, as the stored entries of any sparse
// operand here: a tile adds up the rows of dY of its positions and writes the rows of dE that begin and end in it.  Of a row that spans tiles, each tile leaves
// its part in 32 bits, and a third step adds the parts.  In which order a row is added up depends on the sizes, the type of dY and the tokens alone.
// Rows that no token has are cleared beside the sort, or with many tokens beside the sums.  Bound by reading dY and writing dE.
//
// 16384 x 4096 bf16 into 32768 rows of f32: 151 us, 4.4 TB/s (sort and clearing 91, sums 54, joins 8); other tiles, waves or rows in flight
// change nothing.  Added to dE: 16, 83 and 10.  40001 x 1027 f16 into 50001 rows, a third one token: 84 us (42, 30, 13); without that token 40, 30 and 8;
// added to dE 34, 48 and 13.  131072 x 1024 bf16 into 32768 rows of f32: sort 40, sums and clearing 90, joins 10.
#include "embed.h"
#include "embed_plan.h"

namespace psk {
namespace {

constexpr int MAX_BITS = 9;                                // of a digit

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

// Zeros for a row, `lanes` lanes to it, 16 bytes at a time; the last 16 are the row's last.  Less than 16: element by element.
// They pass the caches by: 512 x 1024 f32 into 8192 rows 12.2 us for 14.2, 16384 x 4096 into 32768 153 for 157.
template <int GT>
__device__ __forceinline__ void clear_row(const Clear &c, int64_t row, int sub, int lanes)
{
    typedef typename Bits<GT>::type B;
    constexpr int EACH = 16 / sizeof(B);
    typedef B piece __attribute__((ext_vector_type(EACH), aligned(sizeof(B))));
    B *const p = static_cast<B *>(c.dE) + row * c.lde;
    if (c.dim < EACH) {
        if (sub < c.dim) p[sub] = B(0);
    } else {
        for (int k = EACH * sub; k < c.dim; k += EACH * lanes) __builtin_nontemporal_store(piece(B(0)), reinterpret_cast<piece *>(p + min(k, c.dim - EACH)));
    }
}
template <int GT>
__device__ __forceinline__ int lanes_log(int dim)
{
    constexpr int EACH = GT == F32 ? 4 : 8;
    int log = 3;
    while (log < 6 && (EACH << log) < dim) ++log;
    return log;
}
// Beside the sort: workgroup `part` of `parts` reads all tokens and clears those of its rows that none of them names.  (Rows that are `parts` apart, so that all
// write in one place: no difference.)
template <int GT, int THREADS>
__device__ __forceinline__ void clear_unnamed(const Clear &c, const int *__restrict__ ids, int n, int padding, int part, int parts, unsigned *bits)
{
    const int64_t per = ((int64_t)c.rows + parts - 1) / parts, begin = part * per, end = min(begin + per, (int64_t)c.rows);
    const int log = lanes_log<GT>(c.dim), sub = threadIdx.x & ((1 << log) - 1);
    for (int64_t first = begin; first < end; first += RANGE) {
        const int count = (int)min(end - first, (int64_t)RANGE);
        for (int i = threadIdx.x; i < (count + 31) / 32; i += THREADS) bits[i] = 0;
        __syncthreads();
        for (int t = 0; t < n; t += 8 * THREADS) {
            const int *const at = ids + t;
            int id[8];                                     // eight loads in flight; behind the last token that is read again
            if (t + 8 * THREADS <= n) {
#pragma unroll
                for (int i = 0; i < 8; ++i) id[i] = at[i * THREADS + threadIdx.x];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) id[i] = at[min(i * THREADS + (int)threadIdx.x, n - 1 - t)];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const unsigned row = place_from(id[i], (int)first);
                if (row < (unsigned)count && id[i] != padding) atomicOr(&bits[row >> 5], 1u << (row & 31));
            }
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
    const int log = lanes_log<GT>(c.dim), sub = threadIdx.x & ((1 << log) - 1);
    for (int r = threadIdx.x >> log; r < 256; r += 256 >> log)
        if (empty[r >> 6] >> (r & 63) & 1) clear_row<GT>(c, first + r, sub, 1 << log);
}

// ------------------------------------------------------------------ the sort
// Lanes of the wave with the same digit as this one, of those that have one.  Often these are few, or most of them the same: up to three digits are
// looked for one by one, and only if there are more, all bit by bit.
__device__ __forceinline__ unsigned long long same_digit(int d, int bits, bool valid)
{
    const unsigned long long all = __ballot(valid);
    unsigned long long left = all, m = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        if (!left) return m;
        const int one = __builtin_amdgcn_readlane(d, __builtin_ctzll(left));
        const unsigned long long equal = __ballot(valid && d == one);
        m = d == one ? equal : m;
        left &= ~equal;
    }
    if (!left) return m;
    m = all;
    for (int b = 0; b < bits; ++b) {
        const unsigned long long set = __ballot(d >> b & 1);
        m &= d >> b & 1 ? set : ~set;
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

// Up to NEAR tokens and RANGES ranges of rows: a workgroup owns `per` rows, reads all tokens, and so knows by itself how many positions are before those of
// its rows.  It counts its own, wave by wave (a wave has a sixteenth of the tokens), and puts them in their places.  Beside these, up to 256 workgroups
// clear (clear_unnamed): waiting and writing go together.
// One launch.
// Bound by every workgroup's reading of all tokens: 16384 into 32768 rows 16 us, 40001 into 50001 34, and 32 without a token that a third of them are.
// 16000 tokens, 4000 rows: 17 us; by one workgroup that sorted them in LDS while the others cleared 35.
template <int GT>
__global__ __launch_bounds__(1024) void k_sort_ranges(const int *__restrict__ ids, int n, int padding, int per, int bits, int ranges, int *__restrict__ keys_out,
                                                      int *__restrict__ at_out, int *__restrict__ joins, Clear c)
{
    constexpr int WAVES = 16, U = 8;                       // rounds of 64 tokens whose loads are in flight
    __shared__ int seen[WAVES][MOST_ROWS];
    __shared__ int part[WAVES], less[WAVES];
    if ((int)blockIdx.x >= ranges) {
        clear_unnamed<GT, 1024>(c, ids, n, padding, blockIdx.x - ranges, gridDim.x - ranges, reinterpret_cast<unsigned *>(&seen[0][0]));
        return;
    }
    if (blockIdx.x == 0 && threadIdx.x < 2) joins[threadIdx.x] = 0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = blockIdx.x * per, count = min(per, c.rows - first);
    const int rounds = (n + 1023) / 1024, begin = wave * rounds * 64;
    for (int d = threadIdx.x; d < WAVES * MOST_ROWS; d += 1024) (&seen[0][0])[d] = 0;
    __syncthreads();
    int before = 0;                                        // tokens of earlier rows
    unsigned long long active = 0;                         // rounds with tokens of this range
    static_assert(NEAR / 1024 <= 64, "a bit for each round");
    auto mine = [&](int id, int at) { return at < n && place_from(id, first) < (unsigned)count && id != padding; };
    // Few instructions for each token, most are of no concern here: what padding and the tokens that are read again behind the last one make of `before` is
    // taken off below.
    for (int r = 0; r < rounds; r += U) {
        const int *const at = ids + begin + 64 * r;
        int id[U];
        if (begin + 64 * (r + U) <= n) {
#pragma unroll
            for (int i = 0; i < U; ++i) id[i] = at[64 * i + lane];
        } else {
#pragma unroll
            for (int i = 0; i < U; ++i) id[i] = ids[min(begin + 64 * (r + i) + lane, n - 1)];
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (r + i >= rounds) break;
            before += (unsigned)id[i] < (unsigned)first;
            const int place = (int)place_from(id[i], first);
            if (__ballot((unsigned)place < (unsigned)count)) {                   // counts only: nothing waits for LDS
                active |= 1ull << (r + i);
                const bool is = mine(id[i], begin + 64 * (r + i) + lane);
                const unsigned long long same = same_digit(place, bits, is);
                if (is && !(same & ((1ull << lane) - 1))) atomicAdd(&seen[wave][place], __popcll(same));
            }
        }
    }
    const int over = begin + 64 * rounds - max(n, begin);  // places of this wave behind the last token
    if (over > 0 && (unsigned)ids[n - 1] < (unsigned)first) before -= over / 64 + (lane < over % 64);
    if ((unsigned)padding < (unsigned)first)
        for (int i = begin + lane; i < min(begin + 64 * rounds, n); i += 64) before -= ids[i] == padding;
#pragma unroll
    for (int d = 1; d < WAVE; d *= 2) before += __shfl_xor(before, d, WAVE);
    if (lane == 0) less[wave] = before;
    __syncthreads();
    int earlier = 0, own = 0;
    for (int w = 0; w < WAVES; ++w) earlier += less[w];
    if (threadIdx.x < MOST_ROWS) {
        int v[WAVES];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v[w] = seen[w][threadIdx.x];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            seen[w][threadIdx.x] = own;
            own += v[w];
        }
    }
    const int base = earlier + block_exclusive<1024>(own, part);
    if (threadIdx.x < MOST_ROWS) {
#pragma unroll
        for (int w = 0; w < WAVES; ++w) seen[w][threadIdx.x] += base;
    }
    if (threadIdx.x == 1023) part[0] = base;               // behind the last row of this range
    __syncthreads();
    while (active) {                                       // rounds in order, U of them at a time
        int at[U], id[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            at[i] = active ? begin + 64 * __builtin_ctzll(active) + lane : n;
            active &= active - 1;
            id[i] = ids[min(at[i], n - 1)];
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const bool is = mine(id[i], at[i]);
            if (!__ballot(is)) continue;
            const int to = place_in_wave((int)place_from(id[i], first), bits, is, lane, seen[wave]);
            if (is) {
                keys_out[to] = id[i];
                at_out[to] = at[i];
            }
        }
    }
    if ((int)blockIdx.x == ranges - 1)                     // positions that are in no row
        for (int i = part[0] + threadIdx.x; i < n; i += 1024) keys_out[i] = c.rows;
}

// Several workgroups: they count their digits, and then put their positions behind those of smaller digits and of earlier workgroups.
// FIRST: keys come from the tokens, and a position is its own place; workgroups behind the counting ones clear.
template <bool FIRST, int GT>
__global__ __launch_bounds__(256) void k_sort_count(const int *__restrict__ keys, int n, int padding, int shift, int bits, int blocks, int *__restrict__ count,
                                                    int *__restrict__ joins, Clear c)
{
    __shared__ int s[RANGE / 32];
    static_assert(RANGE / 32 >= 1 << MAX_BITS, "room for the counts");
    if (FIRST && (int)blockIdx.x >= blocks) {
        clear_unnamed<GT, 256>(c, keys, n, padding, blockIdx.x - blocks, gridDim.x - blocks, reinterpret_cast<unsigned *>(s));
        return;
    }
    if (FIRST && blockIdx.x == 0 && threadIdx.x < 2) joins[threadIdx.x] = 0;
    for (int d = threadIdx.x; d < 1 << bits; d += 256) s[d] = 0;
    __syncthreads();
    const int begin = blockIdx.x * SORT;
    for (int i = threadIdx.x; i < SORT && begin + i < n; i += 256) {
        const int k = FIRST ? key_of(keys, begin + i, c.rows, padding) : keys[begin + i];
        atomicAdd(&s[k >> shift & ((1 << bits) - 1)], 1);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < 1 << MAX_BITS; d += 256) {
        const int v = d < 1 << bits ? s[d] : 0;
        if (blocks <= BASES) count[((int)blockIdx.x << MAX_BITS) + d] = v;       // workgroup by workgroup: each of them reads all
        else if (d < 1 << bits) count[(int64_t)d * blocks + blockIdx.x] = v;     // digit by digit: to be scanned
    }
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
        static_assert(DIGITS == 2, "two counts to a load");
        int all[DIGITS] = {};
        for (int b = 0; b < blocks; b += 8) {
            int2 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = reinterpret_cast<const int2 *>(count)[(min(b + i, blocks - 1) << (MAX_BITS - 1)) + threadIdx.x];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool is = b + i < blocks, before = b + i < (int)blockIdx.x;
                all[0] += is ? v[i].x : 0;
                all[1] += is ? v[i].y : 0;
                base[0] += before ? v[i].x : 0;
                base[1] += before ? v[i].y : 0;
            }
        }
        const int sum = all[0] + all[1];
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
struct Grad {
    int n, rows, dim, accumulate, tile;
    const int *keys, *at;
    const void *dY;
    int64_t ldy;
    void *dE;
    int64_t lde;
    float factor;
    float *head, *tail;                                    // of each tile, dim: the part of a row that began before it, of one that goes on behind it
    int *joins;                                            // note_join
    bool aside;                                            // put_result
};

// Tiles with a row that begins in them and goes on behind them, in any order: two counts, those whose row has few parts from 2 on, the others from the end.
constexpr int MANY = 32;                                   // parts
__device__ __forceinline__ void note_join(const Grad &g, int tile, int row)
{
    const int64_t far = ((int64_t)tile + 1 + MANY) * g.tile;
    if (far < g.n && g.keys[far] == row) g.joins[2 + (g.n - 1) / g.tile - atomicAdd(g.joins + 1, 1)] = tile;
    else g.joins[2 + atomicAdd(g.joins, 1)] = tile;
}

template <int GT>
__device__ __forceinline__ void put_element(const Grad &g, int64_t at, float sum)
{
    const float v = g.factor * sum;
    store_as<GT>(g.dE, at, g.accumulate ? element<GT>(g.dE, at) + v : v);
}
// Four columns of row `row` of dE from column u.col on, without the first u.skip.
template <int GT>
__device__ __forceinline__ void put_row(const Grad &g, int row, Unit u, const float (&sum)[4])
{
    const int64_t at = row * g.lde + u.col;
    if (u.skip == 0) {
        float v[4];
        typename Bits<GT>::type *p = static_cast<typename Bits<GT>::type *>(g.dE) + at;
        if (g.accumulate) {
            Raw4<GT> r;
            load_raw<GT>(r, p);
            widen_raw<GT>(r, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += g.factor * sum[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = g.factor * sum[i];
        }
        store_row<GT>(p, v, g.aside);
    } else {
#pragma unroll
        for (int i = 1; i < 4; ++i)
            if (i >= u.skip) put_element<GT>(g, at + i, sum[i]);
    }
}

// One wave: the tile's positions, 256 J columns, four of each 256 to a lane.
template <int T, int GT, int J>
__device__ __forceinline__ void tile_sum(const Grad &g, int tile, int chunk, int lane)
{
    constexpr int U = 8;                                   // rows of dY in flight
    typedef typename Bits<T>::type B;
    const int p0 = tile * g.tile, count = min(g.tile, g.n - p0), p = min(p0 + lane, g.n - 1);
    const int key = g.keys[p], at = g.at[p];
    const int before = p0 > 0 ? g.keys[p0 - 1] : -1, behind = p0 + count < g.n ? g.keys[p0 + count] : -1;
    const int next = __shfl_down(key, 1);
    // positions behind which a row ends within the tile, and those that are in a row at all
    const bool last = lane == count - 1;
    const unsigned long long ends = __ballot(lane < count && (last || next != key));
    const int valid = __popcll(__ballot(lane < count && key < g.rows));
    bool mine[J];
    Unit u[J];
#pragma unroll
    for (int q = 0; q < J; ++q) {
        const int unit = (chunk * J + q) * 64 + lane;
        mine[q] = 4 * unit < g.dim;
        u[q] = unit_of<4>(mine[q] ? unit : 0, g.dim);
    }
    float sum[J][4] = {};
    for (int i = 0; i < valid; i += U) {
        Raw4<T> r[U][J];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const B *row = static_cast<const B *>(g.dY) + rl(at, min(i + j, valid - 1)) * g.ldy;
#pragma unroll
            for (int q = 0; q < J; ++q) load_raw<T>(r[j][q], row + u[q].col);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (i + j >= valid) break;
#pragma unroll
            for (int q = 0; q < J; ++q) {
                float v[4];
                widen_raw<T>(r[j][q], v);
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[q][k] += v[k];
            }
            if (ends >> (i + j) & 1) {
                const int row = rl(key, i + j);
                const bool began = row != before, goes_on = i + j == count - 1 && row == behind;
                if (began && goes_on && chunk == 0 && lane == 0) note_join(g, tile, row);
#pragma unroll
                for (int q = 0; q < J; ++q) {
                    if (mine[q]) {
                        if (began && !goes_on) {
                            put_row<GT>(g, row, u[q], sum[q]);
                        } else {                           // columns that two lanes have are the same
                            float *to = (began ? g.tail : g.head) + (int64_t)tile * g.dim + u[q].col;
                            *reinterpret_cast<v4f_e *>(to) = v4f{sum[q][0], sum[q][1], sum[q][2], sum[q][3]};
                        }
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum[q][k] = 0.0f;
                }
            }
        }
    }
}

// Rows of less than four columns: a wave per tile, a lane per column.
template <int T, int GT>
__device__ __forceinline__ void tile_sum_narrow(const Grad &g, int tile, int lane)
{
    const int p0 = tile * g.tile, p1 = min(p0 + g.tile, g.n);
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
        if (began && goes_on && lane == 0) note_join(g, tile, row);
        sum = 0.0f;
    }
}

template <int T, int GT, int J>
__global__ __launch_bounds__(256) void k_grad_sum(Grad g, int chunks, int64_t sums, int64_t all)
{
    __shared__ unsigned long long empty[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t b = blockIdx.x; b < all; b += gridDim.x) {
        const int64_t w = b * 4 + wave;
        if (b * 4 >= sums) clear_absent<GT>(Clear{g.dE, g.lde, g.rows, g.dim}, g.keys, g.n, (b - (sums + 3) / 4) * 256, empty);
        else if (w >= sums) continue;
        else if (g.dim < 4) tile_sum_narrow<T, GT>(g, (int)w, lane);
        else tile_sum<T, GT, J>(g, (int)(w / chunks), (int)(w % chunks), lane);
    }
}

// A row that begins in a tile and goes on behind it: its parts.  Few: a workgroup takes the tile and 2048 columns, a wave 256 of them; the parts from the second on
// in order, four loads in flight, and the first one last.  Many: the tile and 64 columns (with 256 columns to a workgroup, two of them took 34 us for 3.7 MB of parts,
// 54 GB/s each), 16 lanes take a 32nd of the parts, eight loads in flight, and their sums meet in LDS.
// (Without the lists, a workgroup to every tile and 256 columns took 25 us for 16384 tokens of 4096 columns, most to find nothing.)
constexpr int JOIN = 8;                                    // waves
struct Part {                                              // a lane's columns
    bool mine;
    Unit u;
};
__device__ __forceinline__ Part part_of(const Grad &g, int unit)
{
    Part p;
    p.mine = g.dim < 4 ? unit < g.dim : 4 * unit < g.dim;
    p.u = g.dim < 4 ? Unit{p.mine ? unit : 0, 0} : unit_of<4>(p.mine ? unit : 0, g.dim);
    return p;
}
__device__ __forceinline__ void add_parts(const Grad &g, const float *head, int more, float (&sum)[4])
{
    constexpr int U = 4;                                   // in flight
    if (g.dim < 4) {
        for (int i = 0; i < more; ++i) sum[0] += head[(int64_t)i * g.dim];
        return;
    }
    for (int i = 0; i < more; i += U) {
        Raw4<F32> r[U];
#pragma unroll
        for (int j = 0; j < U; ++j) load_raw<F32>(r[j], head + (int64_t)min(i + j, more - 1) * g.dim);
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] += i + j < more ? r[j].a[k] : 0.0f;
    }
}
template <int GT>
__device__ __forceinline__ void put_joined(const Grad &g, int tile, int row, const Part &p, float (&sum)[4])
{
    if (!p.mine) return;
    const float *const tail = g.tail + (int64_t)tile * g.dim + p.u.col;
    if (g.dim < 4) {
        put_element<GT>(g, row * g.lde + p.u.col, sum[0] + tail[0]);
    } else {
        const v4f v = *reinterpret_cast<const v4f_e *>(tail);
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] += v[k];
        put_row<GT>(g, row, p.u, sum);
    }
}
template <int GT>
__global__ __launch_bounds__(64 * JOIN) void k_grad_join(Grad g, int tiles, int groups, int strips)
{
    constexpr int U = 8;                                   // parts in flight for each lane
    __shared__ v4f meet[JOIN * 4][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t few = (int64_t)g.joins[0] * groups, all = few + (int64_t)g.joins[1] * strips;
    for (int64_t w = blockIdx.x; w < all; w += gridDim.x) {
        const bool many = w < all - few;                   // the long ones first
        const int64_t v = many ? w : w - (all - few);
        const int tile = many ? g.joins[2 + tiles - 1 - v / strips] : g.joins[2 + v / groups], row = g.keys[(tile + 1) * g.tile];
        int more = 0;                                      // tiles behind it that begin with the row
        for (;;) {
            const int t = tile + 1 + more + lane;
            const int same = __builtin_ctzll(~__ballot(t < tiles && g.keys[t < tiles ? t * g.tile : 0] == row) | (1ull << 63));
            more += same;                                  // at most 63 of a round
            if (same < 63) break;
        }
        const float *const heads = g.head + (int64_t)(tile + 1) * g.dim;
        if (!many) {
            const Part p = part_of(g, (int)(v % groups) * 64 * JOIN + wave * 64 + lane);
            float sum[4] = {};
            if (p.mine) add_parts(g, heads + p.u.col, more, sum);
            put_joined<GT>(g, tile, row, p, sum);
            continue;
        }
        const Part p = part_of(g, (int)(v % strips) * 16 + (lane & 15));
        const int each = (more + JOIN * 4 - 1) / (JOIN * 4), from = min((wave * 4 + (lane >> 4)) * each, more), to = min(from + each, more);
        v4f sum = {0, 0, 0, 0};
        if (p.mine) {
            const float *const head = heads + p.u.col;
            for (int i = from; i < to; i += U) {
                v4f part[U];
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    const float *const at = head + (int64_t)min(i + j, to - 1) * g.dim;
                    part[j] = g.dim < 4 ? v4f{*at, 0, 0, 0} : *reinterpret_cast<const v4f_e *>(at);
                }
#pragma unroll
                for (int j = 0; j < U; ++j) sum += i + j < to ? part[j] : v4f{0, 0, 0, 0};
            }
        }
        __syncthreads();                                   // the last sums have been read
        meet[wave * 4 + (lane >> 4)][lane & 15] = sum;
        __syncthreads();
        if (wave == 0 && lane < 16) {
            for (int o = 1; o < JOIN * 4; ++o) sum += meet[o][lane];
            float s4[4] = {sum[0], sum[1], sum[2], sum[3]};
            put_joined<GT>(g, tile, row, p, s4);
        }
    }
}

// ------------------------------------------------------------------ few tokens
// Up to SMALL tokens of 4 MB in all: one launch.  A workgroup owns rows and `width` of the columns, finds its tokens and their order as k_sort_ranges does, adds them
// up, a row to a wave (rows of more than LONG tokens: a sixteenth of them to a wave, whose sums meet in LDS), and clears the other rows.
// 512 tokens of 1024 columns, 8192 rows, f32: 11.8 us; by three launches 22.  In a trace 12.8, into 1024 rows 9.6, added to dE (nothing to clear) 10.2.
constexpr int LONG = 64;

template <int T, int GT>
__global__ __launch_bounds__(1024) void k_grad_few(Grad g, const int *__restrict__ ids, int padding, int per, int bits, int width)
{
    constexpr int WAVES = 16, U = 8;
    __shared__ int seen[WAVES][MOST_ROWS];
    __shared__ int key[SMALL], at[SMALL], start[SMALL + 1], part[WAVES];
    __shared__ unsigned long long present[MOST_ROWS / 64];
    __shared__ float meet[WAVES][4][64];
    typedef typename Bits<T>::type B;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = blockIdx.x * per, count = min(per, g.rows - first), col0 = blockIdx.y * width, cols = min(width, g.dim - col0);
    const int id = (int)threadIdx.x < g.n ? ids[threadIdx.x] : -1;
    for (int d = threadIdx.x; d < WAVES * MOST_ROWS; d += 1024) (&seen[0][0])[d] = 0;
    __syncthreads();
    const int place = (int)place_from(id, first);
    const bool mine = (unsigned)place < (unsigned)count && id != padding;
    int rank = 0;
    if (__ballot(mine)) rank = place_in_wave(place, bits, mine, lane, seen[wave]);
    __syncthreads();
    int own = 0;
    if (threadIdx.x < MOST_ROWS) {
        int v[WAVES];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v[w] = seen[w][threadIdx.x];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            seen[w][threadIdx.x] = own;
            own += v[w];
        }
        const unsigned long long m = __ballot(own > 0);
        if (lane == 0) present[wave] = m;
    }
    const int base = block_exclusive<1024>(own, part);
    const int nth = block_exclusive<1024>(own > 0, part);  // rows before this one that have tokens
    if (own > 0) start[nth] = base;
    if (threadIdx.x < MOST_ROWS) {
#pragma unroll
        for (int w = 0; w < WAVES; ++w) seen[w][threadIdx.x] += base;
    }
    if (threadIdx.x == 1023) {
        start[nth] = base;                                 // behind the last row
        part[0] = nth;
    }
    __syncthreads();
    const int segments = part[0];
    if (mine) {
        const int to = seen[wave][place] + rank;
        key[to] = id;
        at[to] = threadIdx.x;
    }
    __syncthreads();
    auto sum_up = [&](int from, int to, int col, float (&sum)[4]) {
        for (int i = from; i < to; i += U) {
            Raw4<T> r[U];
#pragma unroll
            for (int j = 0; j < U; ++j) load_raw<T>(r[j], static_cast<const B *>(g.dY) + at[min(i + j, to - 1)] * g.ldy + col);
#pragma unroll
            for (int j = 0; j < U; ++j) {
                float v[4];
                widen_raw<T>(r[j], v);
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[k] += i + j < to ? v[k] : 0.0f;
            }
        }
    };
    const int quads = (cols + 255) / 256;
    for (int i = wave; i < segments * quads; i += WAVES) {
        const int s = i / quads, from = start[s], to = start[s + 1], c = col0 + (i % quads * 64 + lane) * 4;
        if (to - from > LONG || c >= col0 + cols) continue;
        const int col = min(c, g.dim - 4);
        float sum[4] = {};
        sum_up(from, to, col, sum);
        put_row<GT>(g, key[from], Unit{col, c - col}, sum);
    }
    for (int i = 0; i < segments * quads; ++i) {
        const int s = i / quads, from = start[s], to = start[s + 1], c = col0 + (i % quads * 64 + lane) * 4;
        if (to - from <= LONG) continue;                   // (the same for all waves)
        const int each = (to - from + WAVES - 1) / WAVES, begin = from + wave * each, col = min(c, g.dim - 4);
        float sum[4] = {};
        sum_up(begin, min(begin + each, to), col, sum);
        __syncthreads();                                   // the last sums have been read
#pragma unroll
        for (int k = 0; k < 4; ++k) meet[wave][k][lane] = sum[k];
        __syncthreads();
        if (wave > 0 || c >= col0 + cols) continue;
        for (int o = 1; o < WAVES; ++o)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] += meet[o][k][lane];
        put_row<GT>(g, key[from], Unit{col, c - col}, sum);
    }
    if (!g.accumulate) {
        const Clear c = {static_cast<typename Bits<GT>::type *>(g.dE) + col0, g.lde, g.rows, cols};
        const int log = lanes_log<GT>(cols), sub = threadIdx.x & ((1 << log) - 1);
        for (int r = threadIdx.x >> log; r < count; r += 1024 >> log)
            if (!(present[r >> 6] >> (r & 63) & 1)) clear_row<GT>(c, first + r, sub, 1 << log);
    }
}

struct Space {
    int *keys[2], *at[2], *count, *scan, *joins;
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
    const int64_t blocks = (n + SORT - 1) / SORT, tiles = most_tiles(n, dim), counts = blocks << MAX_BITS;
    Space w;
    for (int i = 0; i < 2; ++i) {
        w.keys[i] = reinterpret_cast<int *>(take((size_t)n * 4));
        w.at[i] = reinterpret_cast<int *>(take((size_t)n * 4));
    }
    w.count = reinterpret_cast<int *>(take((size_t)counts * 4));
    w.scan = reinterpret_cast<int *>(take(scan_tmp_ints(counts) * 4));
    w.joins = reinterpret_cast<int *>(take((size_t)(tiles + 2) * 4));
    w.head = reinterpret_cast<float *>(take((size_t)tiles * (size_t)dim * 4));
    w.tail = reinterpret_cast<float *>(take((size_t)tiles * (size_t)dim * 4));
    w.bytes = used;
    return w;
}

unsigned at_most(int64_t blocks, int64_t most) { return (unsigned)(blocks < most ? blocks : most); }

// With up to NEAR tokens, rows without one are cleared beside the sort's first step, by workgroups that read all tokens; more tokens take these longer
// than the search in the sorted ones.
template <int T, int GT>
hipError_t run(int n, int rows, int dim, const int *ids, int padding, float factor, const void *dY, int64_t ldy, void *dE, int64_t lde, int accumulate,
               const Space &w, hipStream_t s)
{
    const Clear c = {dE, lde, rows, dim};
    const bool aside = (int64_t)rows * dim * (GT == F32 ? 4 : 2) >= ASIDE;
    const bool beside = !accumulate && n > 0 && n <= NEAR;
    const int *keys = ids, *at = nullptr;
    const Way way = way_of(n, rows, dim, T == F32 ? 4 : 2);
    if (way == ONE_LAUNCH) {
        // as many columns to a workgroup as leave about 512 of them
        const int quads = (dim + 255) / 256, split = quads < 4 ? quads : 4, width = (quads + split - 1) / split * 256, groups = (dim + width - 1) / width;
        int per = (rows * groups + 511) / 512, bits = 1;
        if (per > MOST_ROWS) per = MOST_ROWS;
        while ((per - 1) >> bits) ++bits;
        const Grad g = {n, rows, dim, accumulate, 0, nullptr, nullptr, dY, ldy, dE, lde, factor, nullptr, nullptr, nullptr, aside};
        PSK_LAUNCH((k_grad_few<T, GT>), dim3((rows + per - 1) / per, groups), dim3(1024), 0, s, g, ids, padding, per, bits, width);
        return take_launch_status();
    }
    int per = (rows + 255) / 256;
    if (per > MOST_ROWS) per = MOST_ROWS;
    if (way == BY_RANGES) {
        int bits = 1;
        while ((per - 1) >> bits) ++bits;
        const int ranges = (rows + per - 1) / per;
        PSK_LAUNCH((k_sort_ranges<GT>), dim3(ranges + (beside ? at_most(ranges, 256) : 0)), dim3(1024), 0, s, ids, n, padding, per, bits, ranges, w.keys[0], w.at[0], w.joins,
                   c);
        keys = w.keys[0];
        at = w.at[0];
    } else {
        const int blocks = (n + SORT - 1) / SORT;
        int bits = 1;
        while (rows >> bits) ++bits;                       // keys are 0 .. rows
        const int passes = (bits + MAX_BITS - 1) / MAX_BITS, digit = (bits + passes - 1) / passes;
        for (int pass = 0; n > 0 && pass < passes; ++pass) {
            const int shift = pass * digit;
            const unsigned clear = beside && pass == 0 ? at_most(((int64_t)rows + 3) / 4, 1024) : 0;
            if (pass == 0) PSK_LAUNCH((k_sort_count<true, GT>), dim3(blocks + clear), dim3(256), 0, s, keys, n, padding, shift, digit, blocks, w.count, w.joins, c);
            else PSK_LAUNCH((k_sort_count<false, GT>), dim3(blocks), dim3(256), 0, s, keys, n, padding, shift, digit, blocks, w.count, w.joins, c);
            const bool scan = way == BY_SCANNED_DIGITS;
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
    const Grad g = {n, rows, dim, accumulate, tile_of(n, dim), keys, at, dY, ldy, dE, lde, factor, w.head, w.tail, w.joins, aside};
    const int tiles = (n + g.tile - 1) / g.tile, j = quads_per_lane(dim), chunks = (dim + 256 * j - 1) / (256 * j), groups = (dim + 256 * JOIN - 1) / (256 * JOIN), strips = (dim + 63) / 64;
    const int64_t sums = (int64_t)tiles * chunks, all = (sums + 3) / 4 + (accumulate || beside ? 0 : ((int64_t)rows + 255) / 256);
    const auto sum = j == 1 ? k_grad_sum<T, GT, 1> : (j == 2 ? k_grad_sum<T, GT, 2> : k_grad_sum<T, GT, 3>);
    PSK_LAUNCH(sum, dim3(at_most(all, 65536)), dim3(256), 0, s, g, chunks, sums, all);
    if (tiles > 1) PSK_LAUNCH((k_grad_join<GT>), dim3(at_most((int64_t)tiles * groups, 1024)), dim3(64 * JOIN), 0, s, g, tiles, groups, strips);
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
