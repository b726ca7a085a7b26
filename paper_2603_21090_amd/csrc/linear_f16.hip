// dense products of one element type (a file per type: they compile beside each other)
#include "linear.h"

namespace stgn {
size_t linear_bytes_f16(const LinearArgs& a) { return dense::part_bytes<_Float16>(a.rows, a.d_out, a.d_in, false, true); }
size_t linear_grad_bytes_f16(const LinearGradArgs& a) { return dense::layout_of<_Float16>(a).total; }
hipError_t linear_f16(const LinearArgs& a, void* ws, hipStream_t s) { return dense::forward<_Float16>(a, ws, s); }
hipError_t linear_grad_f16(const LinearGradArgs& a, void* ws, hipStream_t s) { return dense::backward<_Float16>(a, ws, s); }
}  // namespace stgn
