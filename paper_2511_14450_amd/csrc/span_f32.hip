// Attention over a shared prefix and own keys, 32-bit floats.
#include "span_attention.h"

namespace hyp {
template hipError_t span_prompt<float>(const SpanCall &, bool, hipStream_t);
template hipError_t span_token<float>(const SpanCall &, bool, hipStream_t);
template hipError_t span_received<float>(const SpanCall &, bool, hipStream_t);
template hipError_t span_join<float>(const SpanCall &, hipStream_t);
}  // namespace hyp
