// dense products of one element type (a file per type: they compile beside each other)
#include "linear.h"

namespace stgn {
size_t linear_bytes_f32(const LinearArgs& a) { return dense::part_bytes<float>(a.rows, a.d_out, a.d_in, false, true); }
size_t linear_grad_bytes_f32(const LinearGradArgs& a) { return dense::layout_of<float>(a).total; }
hipError_t linear_f32(const LinearArgs& a, void* ws, hipStream_t s) { return dense::forward<float>(a, ws, s); }
hipError_t linear_grad_f32(const LinearGradArgs& a, void* ws, hipStream_t s) { return dense::backward<float>(a, ws, s); }
}  // namespace stgn
