// Single tokens over caches of 8 and 4 bits: bf16 rows, keys in 4 bits.
#include "mx_token.h"

namespace hyp {
template hipError_t mx_token<bf16_t, HYP_E2M1, HYP_E4M3>(const MxTokenCall &, hipStream_t);
template hipError_t mx_token<bf16_t, HYP_E2M1, HYP_E2M1>(const MxTokenCall &, hipStream_t);
}  // namespace hyp
