// attention of one element type: lists of many queries (a file per type and kind: they compile beside each other)
#include "attention.h"

namespace stgn {
hipError_t attention_f32(const AttnArgs& a, hipStream_t s) { return attn::forward_of<float>(a, s); }
hipError_t attention_grad_f32(const AttnArgs& a, hipStream_t s) { return attn::backward_of<float>(a, s); }
}  // namespace stgn
