// the norm, its gradient and tensors in 8 bits, from one element type
#include "norm.h"

namespace stgn {
hipError_t rms_norm_f16(const NormArgs& a, hipStream_t s) { return a.q ? norm::rows_of<_Float16, norm::kNorm8>(a, s) : norm::rows_of<_Float16, norm::kNorm>(a, s); }
size_t rms_norm_grad_bytes_f16(const NormGradArgs& a) { return norm::grad_plan<_Float16>(a).total; }
hipError_t rms_norm_grad_f16(const NormGradArgs& a, void* ws, hipStream_t s) { return norm::backward<_Float16>(a, ws, s); }
hipError_t rows_in_8_f16(const NormArgs& a, hipStream_t s) { return norm::rows_of<_Float16, norm::kRows8>(a, s); }
hipError_t columns_in_8_f16(const ColumnsArgs& a, void* ws, hipStream_t s) { return norm::columns<_Float16>(a, ws, s); }
size_t columns_bytes_f16(const ColumnsArgs& a) { return norm::columns_bytes<_Float16>(a); }
}  // namespace stgn
