// attention of one element type: lists of few queries
#include "attention_rows.h"

namespace stgn {
hipError_t attention_rows_f16(const AttnArgs& a, void* ws, hipStream_t s) { return attn::rows_of<_Float16, false>(a, static_cast<float*>(ws), s); }
hipError_t attention_rows_grad_f16(const AttnArgs& a, void* ws, hipStream_t s) { return attn::rows_of<_Float16, true>(a, static_cast<float*>(ws), s); }
}  // namespace stgn
