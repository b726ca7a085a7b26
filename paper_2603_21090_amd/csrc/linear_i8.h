// The dense product of operands in 8 bits, sums of 32-bit integers, on gfx950's matrix cores:
//
//   y = act(x_scale[m] w_scale[n] sum_k x[m][k] w[n][k] + bias[n]) + residual
//
// Both operands have k along their rows.  A workgroup owns BM x BN outputs; tiles of 128 bytes of k pass through LDS; accumulators hold the
// transposed tile, four neighbouring columns of one output row a lane.
#pragma once
#include "linear.h"

namespace stgn {
namespace dense8 {

using dense::up;

struct Product {
  const int8_t *l, *r;                                        // the weight (the output's columns), the rows
  int64_t ld_l, ld_r;
  int m, n, k;
  int k_per, splits;
  const float *r_scale, *l_scale;
  const void *bias, *residual;
  void* out;
  int64_t ld_res, ld_out;
  int act;
  int* part;                                                  // [splits, m, n] where splits > 1
};

constexpr int kBK = 128;

__device__ inline floatx4 scaled(const i32x4& s, float rs, const floatx4& ls) {
  floatx4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = (float)s[j] * rs * ls[j];
  return v;
}

template <class T>
__device__ inline void activate(int act, floatx4& v) {
  switch (act) {
    case dense::ACT_RELU: dense::activate<T, dense::ACT_RELU>(v); break;
    case dense::ACT_GELU: dense::activate<T, dense::ACT_GELU>(v); break;
    case dense::ACT_SILU: dense::activate<T, dense::ACT_SILU>(v); break;
    default: break;
  }
}

// scales, bias, activation, residual: four neighbouring outputs of row m
template <class T>
__device__ inline void finish4(const Product& a, int64_t m, int n, const i32x4& sum) {
  floatx4 v = scaled(sum, a.r_scale[m], load4(a.l_scale, n, a.n));
  if (a.bias) v += load4(static_cast<const T*>(a.bias), n, a.n);
  activate<T>(a.act, v);
  if (a.residual) v += load4(static_cast<const T*>(a.residual) + m * a.ld_res, n, a.n);
  store4(static_cast<T*>(a.out) + m * a.ld_out, n, a.n, v);
}

__device__ inline void store_sums(int* row, int n, int cols, const i32x4& v) {
  if (n + 4 <= cols) {
    *reinterpret_cast<u32x4_any*>(row + n) = __builtin_bit_cast(u32x4_any, v);
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (n + j < cols) row[n + j] = v[j];
  }
}
__device__ inline i32x4 load_sums(const int* row, int n, int cols) {
  if (n + 4 <= cols) return __builtin_bit_cast(i32x4, *reinterpret_cast<const u32x4_any*>(row + n));
  i32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (n + j < cols) v[j] = row[n + j];
  return v;
}

template <class T, int BM, int BN, int WM, int WN, int DEPTH>
__global__ __launch_bounds__(WM * WN * 64, BM * BN <= 64 * 64 ? 4 : 2) void product_kernel(Product a) {
  using El = Elem<int8_t>;
  constexpr int THREADS = WM * WN * 64, MB = BM / WM / 16, NB = BN / WN / 16, S = lds_stride<int8_t>(kBK);
  __shared__ __attribute__((aligned(16))) int8_t ls[BN * S], rs[BM * S];
  const int wave = threadIdx.x >> 6, wm = wave % WM * MB * 16, wn = wave / WM * NB * 16;
  const unsigned tm = (unsigned)(a.m + BM - 1) / BM, tn = (unsigned)(a.n + BN - 1) / BN;
  const int split = (int)(blockIdx.x / (tm * tn));
  int row, col;
  dense::tile_of(blockIdx.x % (tm * tn), tm, tn, row, col);
  const int m0 = row * BM, n0 = col * BN;
  const int kb = split * a.k_per, ke = min(a.k, kb + a.k_per);

  using MoveL = ProductMove<int8_t, BN, kBK, THREADS, true>;
  using MoveR = ProductMove<int8_t, BM, kBK, THREADS, true>;
  MoveL ml;
  MoveR mr;
  ml.start(a.l, a.ld_l, n0, a.n, kb, ke, a.k);
  mr.start(a.r, a.ld_r, m0, a.m, kb, ke, a.k);
  u32x4 rl[DEPTH][MoveL::NP], rr[DEPTH][MoveR::NP];
  i32x4 acc[NB][MB];
#pragma unroll
  for (int x = 0; x < NB; ++x)
#pragma unroll
    for (int y = 0; y < MB; ++y) acc[x][y] = i32x4{0, 0, 0, 0};
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (kb + d * kBK < ke) {
      ml.fetch(rl[d], kb + d * kBK);
      mr.fetch(rr[d], kb + d * kBK);
    }
  for (int kt = kb; kt < ke; kt += DEPTH * kBK) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int k = kt + d * kBK;
      if (k >= ke) break;
      __syncthreads();
      ml.store(ls, rl[d]);
      mr.store(rs, rr[d]);
      __syncthreads();
      if (k + DEPTH * kBK < ke) {
        ml.fetch(rl[d], k + DEPTH * kBK);
        mr.fetch(rr[d], k + DEPTH * kBK);
      }
#pragma unroll
      for (int s = 0; s < kBK; s += El::KF) {
        i32x4 lf[NB], rf[MB];
#pragma unroll
        for (int x = 0; x < NB; ++x) lf[x] = frag_rows(ls, S, wn + x * 16, s);
#pragma unroll
        for (int y = 0; y < MB; ++y) rf[y] = frag_rows(rs, S, wm + y * 16, s);
#pragma unroll
        for (int x = 0; x < NB; ++x)
#pragma unroll
          for (int y = 0; y < MB; ++y) acc[x][y] = El::mma(lf[x], rf[y], acc[x][y]);
      }
    }
  }
  const int lane = threadIdx.x & 63, nb = n0 + wn + 4 * (lane >> 4);
#pragma unroll
  for (int y = 0; y < MB; ++y) {
    __builtin_amdgcn_sched_barrier(0);
    const int64_t m = m0 + wm + y * 16 + (lane & 15);
    if (m >= a.m) continue;
#pragma unroll
    for (int x = 0; x < NB; ++x) {
      const int n = nb + x * 16;
      if (n >= a.n) continue;
      if (a.splits > 1) store_sums(a.part + (split * (int64_t)a.m + m) * a.n, n, a.n, acc[x][y]);
      else finish4<T>(a, m, n, acc[x][y]);
    }
  }
}

// Sums of the splits and the epilogue, four outputs a thread
template <class T>
__global__ __launch_bounds__(256) void join_kernel(Product a) {
  const int per_row = (a.n + 3) / 4;
  const int64_t total = (int64_t)a.m * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / per_row;
    const int n = (int)(i - m * per_row) * 4;
    i32x4 v = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) v += load_sums(a.part + ((int64_t)s * a.m + m) * a.n, n, a.n);
    finish4<T>(a, m, n, v);
  }
}

struct Plan { int bm, bn, splits, k_per; };

inline Plan plan_of(int64_t m, int64_t n, int64_t k) {
  Plan p{64, 64, 1, (int)up(k, kBK)};
  const int64_t tiles = ((m + 63) / 64) * ((n + 63) / 64);
  int64_t splits = tiles ? 1024 / tiles : 1;
  if (splits > k / (8 * kBK)) splits = k / (8 * kBK);
  if (splits < 1) splits = 1;
  p.k_per = (int)up((k + splits - 1) / splits, kBK);
  p.splits = (int)((k + p.k_per - 1) / p.k_per);
  return p;
}

inline size_t part_bytes(const Linear8Args& f) {
  const Plan p = plan_of(f.rows, f.d_out, f.d_in);
  return p.splits > 1 ? (size_t)p.splits * f.rows * f.d_out * sizeof(int) : 0;
}

template <class T>
hipError_t forward(const Linear8Args& f, void* ws, hipStream_t s) {
  Product a{};
  a.l = f.w; a.ld_l = f.ld_w; a.r = f.x; a.ld_r = f.ld_x;
  a.m = f.rows; a.n = f.d_out; a.k = f.d_in;
  a.r_scale = f.x_scale; a.l_scale = f.w_scale;
  a.bias = f.bias; a.residual = f.residual; a.ld_res = f.ld_res;
  a.out = f.y; a.ld_out = f.ld_y; a.act = f.act;
  const Plan p = plan_of(a.m, a.n, a.k);
  a.splits = p.splits;
  a.k_per = p.k_per;
  a.part = static_cast<int*>(ws);
  const int64_t grid = ((a.m + (int64_t)p.bm - 1) / p.bm) * ((a.n + (int64_t)p.bn - 1) / p.bn) * p.splits;
  const hipError_t e = launch(product_kernel<T, 64, 64, 2, 2, 3>, grid, 256, s, a);
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t blocks = ((int64_t)a.m * ((a.n + 3) / 4) + 255) / 256;
  return launch(join_kernel<T>, blocks < 4096 ? blocks : 4096, 256, s, a);
}

}  // namespace dense8
}  // namespace stgn
