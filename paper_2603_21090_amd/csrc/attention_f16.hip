// attention of one element type: lists of many queries (a file per type and kind: they compile beside each other)
#include "attention.h"

namespace stgn {
hipError_t attention_f16(const AttnArgs& a, hipStream_t s) { return attn::forward_of<_Float16>(a, s); }
hipError_t attention_grad_f16(const AttnArgs& a, hipStream_t s) { return attn::backward_of<_Float16>(a, s); }
}  // namespace stgn
