// dense products of one element type (a file per type: they compile beside each other)
#include "linear.h"

namespace stgn {
size_t linear_bytes_bf16(const LinearArgs& a) { return dense::part_bytes<__bf16>(a.rows, a.d_out, a.d_in, false, true); }
size_t linear_grad_bytes_bf16(const LinearGradArgs& a) { return dense::layout_of<__bf16>(a).total; }
hipError_t linear_bf16(const LinearArgs& a, void* ws, hipStream_t s) { return dense::forward<__bf16>(a, ws, s); }
hipError_t linear_grad_bf16(const LinearGradArgs& a, void* ws, hipStream_t s) { return dense::backward<__bf16>(a, ws, s); }
}  // namespace stgn
