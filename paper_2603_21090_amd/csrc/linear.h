// Dense products with their epilogue, and their gradients, on gfx950's matrix cores.
//
//   z = x W + b,  y = act(z) + r;     dz = dy act'(z),  dx = dz W^T,  dW = x^T dz,  db = column sums of dz
//
// One kernel does all three products, out[m][n] = sum_k L(n, k) R(m, k): a workgroup owns BM x BN outputs, both operands pass
// through LDS in tiles of BK elements of k, and the kernel is compiled for how each operand lies in memory: k along its rows
// (x in the forward product, both in dx) or rows per k (W in the forward product, both in dW; read from LDS transposed).
// Accumulators hold the transposed tile, four neighbouring columns of one output row a lane, so that bias, activation, residual
// and the stores are 8 or 16 bytes wide.
#pragma once
#include <math.h>

#include "operators.h"
#include "tile_ops.h"

namespace stgn {
namespace dense {

enum { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

__device__ inline float act_value(int act, float z) {
  switch (act) {
    case ACT_RELU: return z > 0.f ? z : 0.f;
    case ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678118654752440f));
    case ACT_SILU: return z / (1.f + expf(-z));
    default: return z;
  }
}
__device__ inline float act_slope(int act, float z) {
  switch (act) {
    case ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case ACT_GELU: return 0.5f * (1.f + erff(z * 0.70710678118654752440f)) + z * expf(-0.5f * z * z) * 0.39894228040143267794f;
    case ACT_SILU: { const float s = 1.f / (1.f + expf(-z)); return s * (1.f + z * (1.f - s)); }
    default: return 1.f;
  }
}

struct Product {
  const void *l, *r;                                          // L: the output's columns, R: its rows
  int64_t ld_l, ld_r;
  int m, n, k;
  int k_per, splits;                                          // elements of k a split sums, a multiple of BK
  const void *bias, *residual;
  void *out, *pre;
  int64_t ld_res, ld_out, ld_pre;
  int act;
  float* part;                                                // [splits, m, n] where splits > 1
};

// bias, activation, residual: four neighbouring outputs of row m
template <class T>
__device__ inline void finish4(const Product& a, int64_t m, int n, floatx4 v) {
  if (a.bias) v += load4(static_cast<const T*>(a.bias), n, a.n);
  if (a.pre) store4(static_cast<T*>(a.pre) + m * a.ld_pre, n, a.n, v);
  if (a.act != ACT_NONE) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = act_value(a.act, v[j]);
  }
  if (a.residual) v += load4(static_cast<const T*>(a.residual) + m * a.ld_res, n, a.n);
  store4(static_cast<T*>(a.out) + m * a.ld_out, n, a.n, v);
}

// Workgroup number -> output tile.  Consecutive workgroups go to the eight dies in turn: each die gets one run of tiles,
// and a run walks eight rows of tiles column by column, so that a die's L2 holds what its workgroups read.
__device__ inline void tile_of(unsigned id, unsigned tm, unsigned tn, int& row, int& col) {
  const unsigned n = tm * tn, die = id & 7u, q = n >> 3, rem = n & 7u;
  id = die * q + min(die, rem) + (id >> 3);
  const unsigned band = 8u * tn, b = id / band, left = min(8u, tm - b * 8u), in = id - b * band;
  row = (int)(b * 8u + in % left);
  col = (int)(in / left);
}

template <class T> constexpr int kTileK = 128 / (int)sizeof(T);    // 64 16-bit numbers, 32 floats: 128 bytes

template <class T, int BM, int BN, int WM, int WN, bool L_ROWS, bool R_ROWS>
__global__ __launch_bounds__(WM * WN * 64) void product_kernel(Product a) {
  using El = Elem<T>;
  constexpr int BK = kTileK<T>, THREADS = WM * WN * 64, MB = BM / WM / 16, NB = BN / WN / 16;
  constexpr int SL = lds_stride<T>(L_ROWS ? BK : BN), SR = lds_stride<T>(R_ROWS ? BK : BM);
  __shared__ __attribute__((aligned(16))) T ls[(L_ROWS ? BN : BK) * SL], rs[(R_ROWS ? BM : BK) * SR];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave % WM * MB * 16, wn = wave / WM * NB * 16;
  const unsigned tm = (unsigned)(a.m + BM - 1) / BM, tn = (unsigned)(a.n + BN - 1) / BN;
  const int split = (int)(blockIdx.x / (tm * tn));
  int row, col;
  tile_of(blockIdx.x % (tm * tn), tm, tn, row, col);
  const int m0 = row * BM, n0 = col * BN;
  const int kb = split * a.k_per, ke = min(a.k, kb + a.k_per);

  TileMove<T, L_ROWS ? BN : BK, L_ROWS ? BK : BN, THREADS> ml;
  TileMove<T, R_ROWS ? BM : BK, R_ROWS ? BK : BM, THREADS> mr;
  const T *lp = static_cast<const T*>(a.l), *rp = static_cast<const T*>(a.r);
  auto fetch = [&](int k) {
    if constexpr (L_ROWS) ml.fetch([&](int i) -> const T* { return n0 + i < a.n ? lp + (int64_t)(n0 + i) * a.ld_l + k : nullptr; }, ke - k);
    else ml.fetch([&](int i) -> const T* { return k + i < ke ? lp + (int64_t)(k + i) * a.ld_l + n0 : nullptr; }, a.n - n0);
    if constexpr (R_ROWS) mr.fetch([&](int i) -> const T* { return m0 + i < a.m ? rp + (int64_t)(m0 + i) * a.ld_r + k : nullptr; }, ke - k);
    else mr.fetch([&](int i) -> const T* { return k + i < ke ? rp + (int64_t)(k + i) * a.ld_r + m0 : nullptr; }, a.m - m0);
  };

  floatx4 acc[NB][MB];
#pragma unroll
  for (int x = 0; x < NB; ++x)
#pragma unroll
    for (int y = 0; y < MB; ++y) acc[x][y] = floatx4{0.f, 0.f, 0.f, 0.f};

  if (kb < ke) fetch(kb);
  for (int k = kb; k < ke; k += BK) {
    __syncthreads();
    ml.store(ls, SL);
    mr.store(rs, SR);
    __syncthreads();
    if (k + BK < ke) fetch(k + BK);
#pragma unroll
    for (int s = 0; s < BK; s += El::KF) {
      typename El::Frag lf[NB], rf[MB];
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        if constexpr (L_ROWS) lf[x] = frag_rows(ls, SL, wn + x * 16, s);
        else lf[x] = frag_cols<T, false>(ls, SL, s, wn + x * 16);
      }
#pragma unroll
      for (int y = 0; y < MB; ++y) {
        if constexpr (R_ROWS) rf[y] = frag_rows(rs, SR, wm + y * 16, s);
        else rf[y] = frag_cols<T, false>(rs, SR, s, wm + y * 16);
      }
#pragma unroll
      for (int x = 0; x < NB; ++x)
#pragma unroll
        for (int y = 0; y < MB; ++y) acc[x][y] = El::mma(lf[x], rf[y], acc[x][y]);
    }
  }

#pragma unroll
  for (int y = 0; y < MB; ++y) {
    const int m = m0 + wm + y * 16 + (lane & 15);
    if (m >= a.m) continue;
#pragma unroll
    for (int x = 0; x < NB; ++x) {
      const int n = n0 + wn + x * 16 + 4 * (lane >> 4);
      if (n >= a.n) continue;
      if (a.splits > 1) store4(a.part + ((int64_t)split * a.m + m) * a.n, n, a.n, acc[x][y]);
      else finish4<T>(a, m, n, acc[x][y]);
    }
  }
}

// sums of the splits, in their order, and the epilogue
template <class T>
__global__ __launch_bounds__(256) void join_kernel(Product a) {
  const int per_row = (a.n + 3) / 4;
  const int64_t total = (int64_t)a.m * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / per_row;
    const int n = (int)(i - m * per_row) * 4;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.splits; ++s) v += load4(a.part + ((int64_t)s * a.m + m) * a.n, n, a.n);
    finish4<T>(a, m, n, v);
  }
}

// dz = dy act'(z), rounded to T as the operand of the products that follow, and the sums of its columns over a workgroup's rows
template <class T>
__global__ __launch_bounds__(256) void dz_kernel(LinearGradArgs a, T* dz, int64_t ld_dz, float* sums, int rows_per) {
  __shared__ floatx4 wsum[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int cols = (a.d_out + 255) / 256, n = (int)(blockIdx.x % cols) * 256 + lane * 4, chunk = (int)(blockIdx.x / cols);
  const int64_t m1 = min((int64_t)a.rows, (int64_t)(chunk + 1) * rows_per);
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  if (n < a.d_out) {
    for (int64_t m = (int64_t)chunk * rows_per + wave; m < m1; m += 4) {
      floatx4 v = load4(static_cast<const T*>(a.dy) + m * a.ld_dy, n, a.d_out);
      if (dz) {
        const floatx4 z = load4(static_cast<const T*>(a.pre) + m * a.ld_pre, n, a.d_out);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= act_slope(a.act, z[j]);
        store4(dz + m * ld_dz, n, a.d_out, v);
      }
      acc += v;
    }
  }
  if (!sums) return;
  wsum[wave][lane] = acc;
  __syncthreads();
  if (wave == 0 && n < a.d_out) {
    const floatx4 v = (wsum[0][lane] + wsum[1][lane]) + (wsum[2][lane] + wsum[3][lane]);
    store4(sums + (int64_t)chunk * a.d_out, n, a.d_out, v);
  }
}

template <class T>
__global__ __launch_bounds__(256) void db_kernel(const float* sums, int chunks, int n, T* db) {
  __shared__ float wsum[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (int)blockIdx.x * 64 + lane;
  float acc = 0.f;
  if (c < n)
    for (int i = wave; i < chunks; i += 4) acc += sums[(int64_t)i * n + c];
  wsum[wave][lane] = acc;
  __syncthreads();
  if (wave == 0 && c < n) db[c] = (T)((wsum[0][lane] + wsum[1][lane]) + (wsum[2][lane] + wsum[3][lane]));
}

inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Plan { bool wide; int splits, k_per; };

// Large outputs take tiles of 128 x 128 (a wave 64 x 64), small ones 64 x 64.  Where the tiles leave the chip's 256 CUs idle and k
// is long, k is split: at least eight tiles of k a split, two workgroups a CU.
template <class T>
Plan plan_of(int64_t m, int64_t n, int64_t k) {
  constexpr int BK = kTileK<T>;
  Plan p;
  p.wide = ((m + 127) / 128) * ((n + 127) / 128) >= 256;
  const int64_t tile = p.wide ? 128 : 64, tiles = ((m + tile - 1) / tile) * ((n + tile - 1) / tile);
  int64_t splits = tiles ? 512 / tiles : 1;
  const int64_t most = k / (8 * BK);
  if (splits > most) splits = most;
  if (splits < 1) splits = 1;
  p.k_per = (int)up((k + splits - 1) / splits, BK);
  if (p.k_per < BK) p.k_per = BK;
  p.splits = (int)((k + p.k_per - 1) / p.k_per);
  if (p.splits < 1) p.splits = 1;
  return p;
}

template <class T>
size_t part_bytes(int64_t m, int64_t n, int64_t k) {
  const Plan p = plan_of<T>(m, n, k);
  return p.splits > 1 ? (size_t)p.splits * m * n * sizeof(float) : 0;
}

template <class T, bool L_ROWS, bool R_ROWS>
hipError_t product(Product a, void* part, hipStream_t s) {
  if (a.m == 0 || a.n == 0) return hipSuccess;
  const Plan p = plan_of<T>(a.m, a.n, a.k);
  a.splits = p.splits;
  a.k_per = p.k_per;
  a.part = static_cast<float*>(part);
  const int tile = p.wide ? 128 : 64;
  const int64_t grid = (int64_t)((a.m + tile - 1) / tile) * ((a.n + tile - 1) / tile) * p.splits;
  hipError_t e = p.wide ? launch(product_kernel<T, 128, 128, 2, 2, L_ROWS, R_ROWS>, grid, 256, s, a)
                        : launch(product_kernel<T, 64, 64, 2, 2, L_ROWS, R_ROWS>, grid, 256, s, a);
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t blocks = ((int64_t)a.m * ((a.n + 3) / 4) + 255) / 256;
  return launch(join_kernel<T>, blocks < 4096 ? blocks : 4096, 256, s, a);
}

template <class T>
hipError_t forward(const LinearArgs& f, void* ws, hipStream_t s) {
  Product a{};
  a.l = f.w; a.ld_l = f.ld_w; a.r = f.x; a.ld_r = f.ld_x;
  a.m = f.rows; a.n = f.d_out; a.k = f.d_in;
  a.bias = f.bias; a.residual = f.residual; a.ld_res = f.ld_res;
  a.out = f.y; a.ld_out = f.ld_y; a.pre = f.pre; a.ld_pre = f.ld_pre; a.act = f.act;
  return product<T, false, true>(a, ws, s);
}

// workspace of the gradient: dz | column sums | the splits' partial sums, of dx and then of dW
struct GradLayout { int64_t ld_dz; int chunks, rows_per; size_t sums, part, total; };
template <class T>
GradLayout layout_of(const LinearGradArgs& a) {
  GradLayout g;
  g.ld_dz = up(a.d_out, 16 / sizeof(T));
  const int64_t cols = (a.d_out + 255) / 256;
  int64_t chunks = (1024 + cols - 1) / cols;
  const int64_t most = (a.rows + 15) / 16;
  if (chunks > most) chunks = most;
  if (chunks < 1) chunks = 1;
  g.rows_per = (int)((a.rows + chunks - 1) / chunks);
  if (g.rows_per < 1) g.rows_per = 1;
  g.chunks = (int)chunks;
  g.sums = a.act != ACT_NONE ? (size_t)up((int64_t)a.rows * g.ld_dz * sizeof(T), 256) : 0;
  g.part = g.sums + (a.db ? (size_t)up((int64_t)g.chunks * a.d_out * sizeof(float), 256) : 0);
  const size_t px = a.dx ? part_bytes<T>(a.rows, a.d_in, a.d_out) : 0, pw = a.dw ? part_bytes<T>(a.d_in, a.d_out, a.rows) : 0;
  g.total = g.part + (px > pw ? px : pw);
  return g;
}

template <class T>
hipError_t backward(const LinearGradArgs& f, void* ws, hipStream_t s) {
  const GradLayout g = layout_of<T>(f);
  char* base = static_cast<char*>(ws);
  T* dz = f.act != ACT_NONE ? reinterpret_cast<T*>(base) : nullptr;
  float* sums = f.db ? reinterpret_cast<float*>(base + g.sums) : nullptr;
  hipError_t e = hipSuccess;
  if (dz || sums) {
    e = launch(dz_kernel<T>, (int64_t)g.chunks * ((f.d_out + 255) / 256), 256, s, f, dz, g.ld_dz, sums, g.rows_per);
    if (e == hipSuccess && sums) e = launch(db_kernel<T>, (f.d_out + 63) / 64, 256, s, (const float*)sums, g.chunks, f.d_out, static_cast<T*>(f.db));
  }
  const void* z = dz ? dz : f.dy;
  const int64_t ld_z = dz ? g.ld_dz : f.ld_dy;
  if (e == hipSuccess && f.dx) {
    Product a{};
    a.l = f.w; a.ld_l = f.ld_w; a.r = z; a.ld_r = ld_z;
    a.m = f.rows; a.n = f.d_in; a.k = f.d_out; a.out = f.dx; a.ld_out = f.d_in;
    e = product<T, true, true>(a, base + g.part, s);
  }
  if (e == hipSuccess && f.dw) {
    Product a{};
    a.l = z; a.ld_l = ld_z; a.r = f.x; a.ld_r = f.ld_x;
    a.m = f.d_in; a.n = f.d_out; a.k = f.rows; a.out = f.dw; a.ld_out = f.d_out;
    e = product<T, false, false>(a, base + g.part, s);
  }
  return e;
}

}  // namespace dense
}  // namespace stgn
