// The layer of a mixture of experts with 16-bit weights (moe.h).
#include "moe.h"

namespace psk {
namespace {

template <int T>
hipError_t launch_16(const MoeCall &c, const Weights16 &w1, const Weights16 &w3, const Weights16 &w2, hipStream_t s)
{
    return launch_layer<Span16<T, T, 2, 4>, Span16<T, BF16, 1, 4>, Span16<T, T, 2, 2>, Span16<T, BF16, 2, 2>, 2, T, NotKept>(c, w1, w3, w2, s);
}

}  // namespace

size_t moe_workspace_bytes(int64_t n, int64_t dim, int64_t inter, int64_t experts, int top_k)
{
    // a call with fewer tokens may take the other way: enough for both
    MoeCall c = {n, (int)dim, (int)inter, (int)experts, top_k, 0, nullptr, 0, nullptr, nullptr, nullptr, 0, nullptr};
    Call a;
    const size_t all = carve_moe(c, &a);
    c.n = n < FEW ? n : FEW;
    const size_t few = carve_moe(c, &a);
    return (all > few ? all : few) + 256;
}

hipError_t launch_moe_16(const MoeCall &c, int type, const void *W1, const void *W3, int64_t ld1, int64_t stride1, const void *W2, int64_t ld2,
                         int64_t stride2, hipStream_t s)
{
    const Weights16 w1 = {static_cast<const unsigned short *>(W1), ld1, stride1, c.inter, c.dim};
    const Weights16 w3 = {static_cast<const unsigned short *>(W3), ld1, stride1, c.inter, c.dim};
    const Weights16 w2 = {static_cast<const unsigned short *>(W2), ld2, stride2, c.dim, c.inter};
    return type == F16 ? launch_16<F16>(c, w1, w3, w2, s) : launch_16<BF16>(c, w1, w3, w2, s);
}

}  // namespace psk
