// attention of one element type: lists of few queries
#include "attention_rows.h"

namespace stgn {
hipError_t attention_rows_f32(const AttnArgs& a, void* ws, hipStream_t s) { return attn::rows_of<float, false>(a, static_cast<float*>(ws), s); }
hipError_t attention_rows_grad_f32(const AttnArgs& a, void* ws, hipStream_t s) { return attn::rows_of<float, true>(a, static_cast<float*>(ws), s); }
}  // namespace stgn
