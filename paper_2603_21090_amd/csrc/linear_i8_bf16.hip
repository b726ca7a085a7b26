// dense products of operands in 8 bits with outputs of one element type
#include "linear_i8.h"

namespace stgn {
hipError_t linear_i8_bf16(const Linear8Args& a, void* ws, hipStream_t s) { return dense8::forward<__bf16>(a, ws, s); }
}  // namespace stgn
