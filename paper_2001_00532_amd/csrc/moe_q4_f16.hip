// The layer of a mixture of experts with 4-bit weights, tokens of type f16.
#include "moe_q4.h"

namespace psk {
template hipError_t launch_moe_q4_of<F16>(const MoeCall &c, int scale_type, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s);
}
