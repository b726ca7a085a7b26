// attention of one element type: lists of many queries (a file per type and kind: they compile beside each other)
#include "attention.h"

namespace stgn {
size_t attention_bytes_bf16(const AttnArgs& a) { return attn::forward_bytes_of<__bf16>(a); }
size_t attention_grad_bytes_bf16(const AttnArgs& a) { return attn::backward_bytes_of<__bf16>(a); }
hipError_t attention_bf16(const AttnArgs& a, void* ws, hipStream_t s) { return attn::forward_of<__bf16>(a, ws, s); }
hipError_t attention_grad_bf16(const AttnArgs& a, void* ws, hipStream_t s) { return attn::backward_of<__bf16>(a, ws, s); }
}  // namespace stgn
