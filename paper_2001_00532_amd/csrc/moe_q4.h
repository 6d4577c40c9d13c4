// The layer of a mixture of experts with 4-bit weights: which instance of the kernels in moe.h a call takes.
#pragma once
#include "moe.h"

namespace psk {
namespace {

template <int T, int S, int MOST, int P, int G1>
hipError_t launch_q4_down(const MoeCall &c, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s)
{
    typedef SpanQ4<T, 2, P, G1, S, true> UP;
    if (w2.shift == 5) return launch_most<UP, SpanQ4<BF16, 1, P, 1, S, true>, T, MOST>(c, w1, w3, w2, s);
    if (w2.shift == 6) return launch_most<UP, SpanQ4<BF16, 1, P, 2, S, true>, T, MOST>(c, w1, w3, w2, s);
    if (w2.shift == 7 || P == 1) return launch_most<UP, SpanQ4<BF16, 1, P, 4, S, true>, T, MOST>(c, w1, w3, w2, s);
    return launch_most<UP, SpanQ4<BF16, 1, P, 4 * P, S, true>, T, MOST>(c, w1, w3, w2, s);
}
template <int T, int S, int MOST, int P>
hipError_t launch_q4_up(const MoeCall &c, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s)
{
    if (w1.shift == 5) return launch_q4_down<T, S, MOST, P, 1>(c, w1, w3, w2, s);
    if (w1.shift == 6) return launch_q4_down<T, S, MOST, P, 2>(c, w1, w3, w2, s);
    if (w1.shift == 7 || P == 1) return launch_q4_down<T, S, MOST, P, 4>(c, w1, w3, w2, s);
    return launch_q4_down<T, S, MOST, P, 4 * P>(c, w1, w3, w2, s);
}
template <int T, int S>
hipError_t launch_q4(const MoeCall &c, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s)
{
    return c.n <= 4 ? launch_q4_up<T, S, 0, 2>(c, w1, w3, w2, s) : launch_q4_up<T, S, 1, 1>(c, w1, w3, w2, s);
}

}  // namespace

template <int T>
hipError_t launch_moe_q4_of(const MoeCall &c, int scale_type, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s)
{
    return scale_type == T ? launch_q4<T, T>(c, w1, w3, w2, s) : launch_q4<T, F32>(c, w1, w3, w2, s);
}

}  // namespace psk
