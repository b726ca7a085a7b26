// the norm, its gradient and tensors in 8 bits, from one element type
#include "norm.h"

namespace stgn {
hipError_t rms_norm_f32(const NormArgs& a, hipStream_t s) { return a.q ? norm::rows_of<float, norm::kNorm8>(a, s) : norm::rows_of<float, norm::kNorm>(a, s); }
size_t rms_norm_grad_bytes_f32(const NormGradArgs& a) { return norm::grad_plan<float>(a).total; }
hipError_t rms_norm_grad_f32(const NormGradArgs& a, void* ws, hipStream_t s) { return norm::backward<float>(a, ws, s); }
hipError_t rows_in_8_f32(const NormArgs& a, hipStream_t s) { return norm::rows_of<float, norm::kRows8>(a, s); }
hipError_t columns_in_8_f32(const ColumnsArgs& a, void* ws, hipStream_t s) { return norm::columns<float>(a, ws, s); }
size_t columns_bytes_f32(const ColumnsArgs& a) { return norm::columns_bytes<float>(a); }
}  // namespace stgn
