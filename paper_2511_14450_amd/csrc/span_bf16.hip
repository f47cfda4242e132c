// Attention over a shared prefix and own keys, bf16.
#include "span_attention.h"

namespace hyp {
template hipError_t span_prompt<bf16_t>(const SpanCall &, bool, hipStream_t);
template hipError_t span_token<bf16_t>(const SpanCall &, bool, hipStream_t);
template hipError_t span_received<bf16_t>(const SpanCall &, bool, hipStream_t);
template hipError_t span_join<bf16_t>(const SpanCall &, hipStream_t);
}  // namespace hyp
