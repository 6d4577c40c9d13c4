// The embedding lookup (formulas: embed.h).  Bound by reading the rows of different tokens and writing Y.
//
// 16384 tokens of 131072 x 4096 bf16: 34 us, 5.6 TB/s; with stores that stay in the caches 44 (67 MB of Y 23.6 and 28.9, 17 MB 7.1 and 7.6; the call behind it,
// which reads Y, then takes as much longer).
#include "embed.h"

namespace psk {
namespace {

// 2^lanes_log lanes to a row, W columns to a lane.
template <int ET, int YT, int W>
__global__ __launch_bounds__(256) void k_embed(int n, int rows, int dim, int lanes_log, const int *__restrict__ ids, float factor, const void *E, int64_t lde,
                                               const float *__restrict__ scales, void *Y, int64_t ldy, bool aside)
{
    const int lanes = 1 << lanes_log, sub = threadIdx.x & (lanes - 1), units = (dim + W - 1) / W;
    const int64_t step = (int64_t)gridDim.x * (256 >> lanes_log);
    for (int64_t t = (int64_t)blockIdx.x * (256 >> lanes_log) + (threadIdx.x >> lanes_log); t < n; t += step) {
        const int id = ids[t];
        const bool none = (unsigned)id >= (unsigned)rows;
        const typename Bits<ET>::type *e = static_cast<const typename Bits<ET>::type *>(E) + (none ? 0 : id * lde);
        typename Bits<YT>::type *y = static_cast<typename Bits<YT>::type *>(Y) + t * ldy;
        float f = factor;
        if constexpr (ET == I8) f *= none ? 0.0f : scales[id];
        if (dim < W) {
            for (int k = sub; k < dim; k += lanes) store_as<YT>(Y, t * ldy + k, none ? 0.0f : element<ET>(e, k) * f);
            continue;
        }
        for (int u = sub; u < units; u += lanes) {
            const int k = unit_of<W>(u, dim).col;
            float v[W] = {};
            if (!none) {
                typename RawOf<ET, W>::type r;
                load_raw<ET>(r, e + k);
                widen_raw<ET>(r, v);
#pragma unroll
                for (int i = 0; i < W; ++i) v[i] *= f;
            }
            store_row<YT>(y + k, v, aside);
        }
    }
}

template <int ET, int YT>
hipError_t launch(int n, int rows, int dim, const int *ids, float factor, const void *E, int64_t lde, const float *scales, void *Y, int64_t ldy, hipStream_t s)
{
    constexpr int W = ET == F32 || YT == F32 ? 4 : 8;
    const int units = (dim + W - 1) / W;
    int log = 0;
    while (log < 8 && (1 << log) < units) ++log;
    const int64_t blocks = ((int64_t)n + (256 >> log) - 1) / (256 >> log);
    PSK_LAUNCH((k_embed<ET, YT, W>), dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s, n, rows, dim, log, ids, factor, E, lde, scales, Y, ldy,
               (int64_t)n * dim * (YT == F32 ? 4 : 2) >= ASIDE);
    return take_launch_status();
}

template <int ET>
hipError_t launch_y(int ytype, int n, int rows, int dim, const int *ids, float factor, const void *E, int64_t lde, const float *scales, void *Y, int64_t ldy,
                    hipStream_t s)
{
    const auto f = ytype == F32 ? launch<ET, F32> : (ytype == F16 ? launch<ET, F16> : launch<ET, BF16>);
    return f(n, rows, dim, ids, factor, E, lde, scales, Y, ldy, s);
}

}  // namespace

hipError_t launch_embed(int n, int rows, int dim, const int *ids, float factor, int etype, const void *E, int64_t lde, const float *scales, int ytype,
                        void *Y, int64_t ldy, hipStream_t s)
{
    const auto f = etype == F32 ? launch_y<F32> : (etype == F16 ? launch_y<F16> : (etype == BF16 ? launch_y<BF16> : launch_y<I8>));
    return f(ytype, n, rows, dim, ids, factor, E, lde, scales, Y, ldy, s);
}

}  // namespace psk
