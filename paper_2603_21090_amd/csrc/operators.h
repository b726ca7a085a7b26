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

// the norm of rows (with gain), rows in 8 bits (without), both
struct NormArgs {
  const void *x, *residual, *gain;
  void *h, *y;                                                // null: not wanted
  int8_t* q;
  float* scale;                                               // [rows]
  int64_t ld_x, ld_res, ld_h, ld_y, ld_q;
  int rows, width;
  double eps;
};

struct NormGradArgs {
  const void *dy, *h, *gain, *dh;
  void *dx, *dgain;                                           // null: not wanted
  int64_t ld_dy, ld_h, ld_dh, ld_dx;
  int rows, width;
  double eps;
};

// columns in 8 bits: x [rows x width], q [width x rows]
struct ColumnsArgs {
  const void* x;
  int8_t* q;
  float* scale;                                               // [width]
  int64_t ld_x, ld_q;
  int rows, width;
};

struct DropoutArgs {
  const void *x, *residual;
  void* y;
  const uint64_t* rng;                                        // seed, step
  int64_t ld_x, ld_res, ld_y;
  int rows, width;
  uint32_t border, site;                                      // numbers of 16 bits below the border are dropped
  float scale;                                                // of what is kept
};

struct Linear8Args {
  const int8_t *x, *w;                                        // [rows x d_in], [d_out x d_in]
  const float *x_scale, *w_scale;
  const void *bias, *residual;
  void* y;
  int64_t ld_x, ld_w, ld_res, ld_y;
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
