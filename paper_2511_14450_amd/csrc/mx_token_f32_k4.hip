// Single tokens over caches of 8 and 4 bits: float rows, keys in 4 bits.
#include "mx_token.h"

namespace hyp {
template hipError_t mx_token<float, HYP_E2M1, HYP_E4M3>(const MxTokenCall &, hipStream_t);
template hipError_t mx_token<float, HYP_E2M1, HYP_E2M1>(const MxTokenCall &, hipStream_t);
}  // namespace hyp
