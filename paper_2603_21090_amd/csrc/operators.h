// The operators on the caller's own tensors (stgn_linear, stgn_attention and their gradients): what their entry points hand
// to the kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <tuple>

namespace stgn {

struct Strides { int64_t list, row, head; };                  // in elements; the numbers of one head lie side by side

struct AttnArgs {
  const void *q, *k, *v, *dout, *out;                         // dq, dk, dv: dense [lists, rows, heads, d]
  void *o, *dq, *dk, *dv;
  float* lse;                                                 // [lists, heads, q_len]
  float* delta;                                               // of the gradient: dout . out, laid out as lse
  const int *q_lens, *k_lens;                                 // [lists] or null: every list is q_len, k_len long
  Strides sq, sk, sv, so, sdo;
  int lists, q_len, k_len, heads, kv_heads, group, group_shift, d;                // group: query heads a key head; its logarithm or -1
  int causal, window;
  float scale;
};

struct LinearArgs {
  const void *x, *w, *bias, *residual;
  void *y, *pre;
  int64_t ld_x, ld_w, ld_res, ld_y, ld_pre;
  int rows, d_in, d_out, act;
};

struct LinearGradArgs {
  const void *dy, *x, *w, *pre;
  void *dx, *dw, *db;                                         // dense; null: not wanted
  int64_t ld_dy, ld_x, ld_w, ld_pre;
  int rows, d_in, d_out, act;
};

size_t linear_bytes(const LinearArgs& a, int dtype);
hipError_t launch_linear(const LinearArgs& a, int dtype, void* ws, hipStream_t s);

// a launch's own error, whatever an earlier call left behind
template <class... P, class... A>
inline hipError_t launch(void (*kernel)(P...), int64_t grid, int block, hipStream_t s, A... args) {
  std::tuple<P...> p(args...);
  return std::apply([&](auto&... x) {
    void* ptrs[] = {(void*)&x...};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((uint32_t)grid), dim3(block), ptrs, 0, s);
  }, p);
}

int fail_operator(int code, const char* why);                 // the message of stgn_last_error(NULL)

}  // namespace stgn
