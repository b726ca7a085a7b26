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

// Phi(z), the normal distribution's share below z, and e^(-z^2/2).  16-bit types: Phi(-|z|) = poly(t) e^(-z^2/2) / 2, t = 1 / (1 + 0.3275911
// |z| / sqrt 2) (Abramowitz & Stegun 7.1.26, 1.5e-7 off at most; the tail keeps its size: 0.07 % off at -4).  erff takes several times
// the instructions on every output: 90 us more for 8,192 x 4,096 x 4,096 in bf16.
template <class T>
__device__ inline void normal_share(float z, float& share, float& bell) {
  if constexpr (sizeof(T) == 4) {
    share = 0.5f * (1.f + erff(z * 0.70710678118654752440f));
    bell = expf(-0.5f * z * z);
  } else {
    const float x = fabsf(z) * 0.70710678118654752440f, t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
    bell = __builtin_amdgcn_exp2f(-1.44269504088896340736f * x * x);
    const float poly = fmaf(fmaf(fmaf(fmaf(1.061405429f, t, -1.453152027f), t, 1.421413741f), t, -0.284496736f), t, 0.254829592f);
    const float tail = 0.5f * poly * t * bell;
    share = z < 0.f ? tail : 1.f - tail;
  }
}
// 1 / (1 + e^-z)
template <class T>
__device__ inline float logistic(float z) {
  if constexpr (sizeof(T) == 4) return 1.f / (1.f + expf(-z));
  else return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * z));
}

template <class T, int ACT>
__device__ inline float act_value(float z) {
  if constexpr (ACT == ACT_RELU) return z < 0.f ? 0.f : z;         // (a NaN stays one)
  if constexpr (ACT == ACT_GELU) {
    float share, bell;
    normal_share<T>(z, share, bell);
    return z * share;
  }
  if constexpr (ACT == ACT_SILU) return z * logistic<T>(z);
  return z;
}
template <class T>
__device__ inline float act_slope(int act, float z) {
  if (act == ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (act == ACT_GELU) {
    float share, bell;
    normal_share<T>(z, share, bell);
    return fmaf(z * 0.39894228040143267794f, bell, share);
  }
  const float s = logistic<T>(z);
  return s * fmaf(z, 1.f - s, 1.f);
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

template <class T, int ACT>
__device__ inline void activate(floatx4& v) {
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = act_value<T, ACT>(v[j]);
}

// bias, activation, residual: four neighbouring outputs of row m (one place in the code for all of them: `act` is the same for all)
template <class T>
__device__ inline void finish4(const Product& a, int64_t m, int n, floatx4 v) {
  if (a.bias) v += load4(static_cast<const T*>(a.bias), n, a.n);
  if (a.pre) store4(static_cast<T*>(a.pre) + m * a.ld_pre, n, a.n, v);
  switch (a.act) {
    case ACT_RELU: activate<T, ACT_RELU>(v); break;
    case ACT_GELU: activate<T, ACT_GELU>(v); break;
    case ACT_SILU: activate<T, ACT_SILU>(v); break;
    default: break;
  }
  if (a.residual) v += load4(static_cast<const T*>(a.residual) + m * a.ld_res, n, a.n);
  store4(static_cast<T*>(a.out) + m * a.ld_out, n, a.n, v);
}

// A wave's blocks of 16 x 16, from output (m0, n0): a split's sums, or the epilogue.  Sixteen rows at a time: the scheduler would have
// all rows' residuals in registers at once and spill the sums.
template <class T, int NB, int MB>
__device__ __forceinline__ void finish_tile(const Product& a, int split, int m0, int n0, floatx4 (&acc)[NB][MB]) {
  const int lane = threadIdx.x & 63, nb = n0 + 4 * (lane >> 4);
#pragma unroll
  for (int y = 0; y < MB; ++y) {
    __builtin_amdgcn_sched_barrier(0);
    const int64_t m = m0 + y * 16 + (lane & 15);
    if (m >= a.m) continue;
    auto each = [&](auto f) {
#pragma unroll
      for (int x = 0; x < NB; ++x)
        if (nb + x * 16 < a.n) f(nb + x * 16, acc[x][y]);
    };
    if (a.splits > 1) {
      each([&](int n, floatx4& v) { store4(a.part + (split * (int64_t)a.m + m) * a.n, n, a.n, v); });
      continue;
    }
    if (a.bias) each([&](int n, floatx4& v) { v += load4(static_cast<const T*>(a.bias), n, a.n); });
    if (a.pre) each([&](int n, floatx4& v) { store4(static_cast<T*>(a.pre) + m * a.ld_pre, n, a.n, v); });
    switch (a.act) {
      case ACT_RELU: each([&](int, floatx4& v) { activate<T, ACT_RELU>(v); }); break;
      case ACT_GELU: each([&](int, floatx4& v) { activate<T, ACT_GELU>(v); }); break;
      case ACT_SILU: each([&](int, floatx4& v) { activate<T, ACT_SILU>(v); }); break;
      default: break;
    }
    if (a.residual) each([&](int n, floatx4& v) { v += load4(static_cast<const T*>(a.residual) + m * a.ld_res, n, a.n); });
    each([&](int n, floatx4& v) { store4(static_cast<T*>(a.out) + m * a.ld_out, n, a.n, v); });
  }
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

// DEPTH tiles of k are on their way in registers while one is multiplied: where tiles are small and few, what a tile takes is the wait
// for memory (13 x 4,096 x 11,008 in bf16: 26.6 us with one, 19.9 with three).  Large ones have one on its way and two in LDS, so that a
// barrier a tile is enough.  Small tiles run four workgroups a CU: 128 registers.
template <class T, int BM, int BN, int WM, int WN, int DEPTH, bool L_ROWS, bool R_ROWS>
__global__ __launch_bounds__(WM * WN * 64, BM * BN <= 64 * 64 ? 4 : 2) void product_kernel(Product a) {
  using El = Elem<T>;
  constexpr int BK = kTileK<T>, THREADS = WM * WN * 64, MB = BM / WM / 16, NB = BN / WN / 16;
  constexpr int SL = lds_stride<T>(L_ROWS ? BK : BN), SR = lds_stride<T>(R_ROWS ? BK : BM);
  constexpr int BUFS = DEPTH == 1 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) T ls[BUFS][(L_ROWS ? BN : BK) * SL], rs[BUFS][(R_ROWS ? BM : BK) * SR];
  const int wave = threadIdx.x >> 6, wm = wave % WM * MB * 16, wn = wave / WM * NB * 16;
  const unsigned tm = (unsigned)(a.m + BM - 1) / BM, tn = (unsigned)(a.n + BN - 1) / BN;
  const int split = (int)(blockIdx.x / (tm * tn));
  int row, col;
  tile_of(blockIdx.x % (tm * tn), tm, tn, row, col);
  const int m0 = row * BM, n0 = col * BN;
  const int kb = split * a.k_per, ke = min(a.k, kb + a.k_per);

  using MoveL = ProductMove<T, BN, BK, THREADS, L_ROWS>;
  using MoveR = ProductMove<T, BM, BK, THREADS, R_ROWS>;
  MoveL ml;
  MoveR mr;
  ml.start(a.l, a.ld_l, n0, a.n, kb, ke, a.k);
  mr.start(a.r, a.ld_r, m0, a.m, kb, ke, a.k);
  u32x4 rl[DEPTH][MoveL::NP], rr[DEPTH][MoveR::NP];
  auto fetch = [&](int d, int k) {
    ml.fetch(rl[d], k);
    mr.fetch(rr[d], k);
  };

  floatx4 acc[NB][MB];
#pragma unroll
  for (int x = 0; x < NB; ++x)
#pragma unroll
    for (int y = 0; y < MB; ++y) acc[x][y] = floatx4{0.f, 0.f, 0.f, 0.f};

  auto multiply = [&](const T* l, const T* r) {
#pragma unroll
    for (int s = 0; s < BK; s += El::KF) {
      typename El::Frag lf[NB], rf[MB];
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        if constexpr (L_ROWS) lf[x] = frag_rows(l, SL, wn + x * 16, s);
        else lf[x] = frag_cols<T, false>(l, SL, s, wn + x * 16);
      }
#pragma unroll
      for (int y = 0; y < MB; ++y) {
        if constexpr (R_ROWS) rf[y] = frag_rows(r, SR, wm + y * 16, s);
        else rf[y] = frag_cols<T, false>(r, SR, s, wm + y * 16);
      }
#pragma unroll
      for (int x = 0; x < NB; ++x)
#pragma unroll
        for (int y = 0; y < MB; ++y) acc[x][y] = El::mma(lf[x], rf[y], acc[x][y]);
    }
  };
  if constexpr (DEPTH == 1) {                                 // two buffers in LDS, one barrier a tile
    if (kb < ke) {
      fetch(0, kb);
      ml.store(ls[0], rl[0]);
      mr.store(rs[0], rr[0]);
    }
    int buf = 0;
    for (int k = kb; k < ke; k += BK, buf ^= 1) {
      __syncthreads();
      const bool more = k + BK < ke;
      if (more) fetch(0, k + BK);
      multiply(ls[buf], rs[buf]);
      if (more) {
        ml.store(ls[buf ^ 1], rl[0]);
        mr.store(rs[buf ^ 1], rr[0]);
      }
    }
  } else {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (kb + d * BK < ke) fetch(d, kb + d * BK);
    for (int kt = kb; kt < ke; kt += DEPTH * BK) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        const int k = kt + d * BK;
        if (k >= ke) break;
        __syncthreads();
        ml.store(ls[0], rl[d]);
        mr.store(rs[0], rr[d]);
        __syncthreads();
        if (k + DEPTH * BK < ke) fetch(d, k + DEPTH * BK);
        multiply(ls[0], rs[0]);
      }
    }
  }
  finish_tile<T, NB, MB>(a, split, m0 + wm, n0 + wn, acc);
}

// The same for large outputs of 16-bit types: 256 x 256 outputs a workgroup of eight waves, each 64 rows x 128 columns, two tiles of
// k in LDS: one is multiplied while the next one is on its way through registers into the other, one barrier a tile.  Rows are not
// padded (two buffers of both operands are 128 KB); piece p (16 bytes) of row r lies at p ^ turn(r), which spreads what one read touches
// over the banks: eight rows of a fragment along k, four rows of a transposed one.  Rows and columns past the edge repeat the last
// ones and are not stored; k has whole tiles.
// The column side's fragments come in pairs: of 32 columns the first holds 8 q + 0 .. 3 (q = 0 .. 3) and the second 8 q + 4 .. 7, so that a
// lane's two accumulators are eight neighbouring outputs, and four lanes 64 bytes of a row.
template <class T, bool ROWS, bool PAIRS>
struct LargeMove {                                            // ROWS: [256 lines][64 of k], else [64 of k][256 lines]
  const T* at[4];
  u32x4 r[4];
  int64_t step;
  static __device__ inline int turn(int row) {
    if (PAIRS) return ROWS ? ((row >> 2) & 6) | ((row >> 1) & 1) : (row & 3) << 2;
    return ROWS ? row & 7 : ((row & 3) << 1) | (row & 8);
  }
  __device__ inline void start(const T* base, int64_t ld, int first, int lines, int k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = i * 512 + (int)threadIdx.x;
      if constexpr (ROWS) at[i] = base + (int64_t)min(first + p / 8, lines - 1) * ld + k + p % 8 * 8;
      else at[i] = base + (int64_t)(k + p / 32) * ld + min(first + p % 32 * 8, lines - 8);
    }
    step = ROWS ? 64 : 64 * ld;
  }
  __device__ inline void fetch() {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[i] = *reinterpret_cast<const u32x4_any*>(at[i]);
      at[i] += step;
    }
  }
  __device__ inline void store(T* tile) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = i * 512 + (int)threadIdx.x, row = ROWS ? p / 8 : p / 32, piece = ROWS ? p % 8 : p % 32;
      *reinterpret_cast<u32x4*>(tile + (p - piece + (piece ^ turn(row))) * 8) = r[i];
    }
  }
  // fragment of 16 lines from `line` (PAIRS: of a pair's 32 lines, the first's or the second's), elements k .. k + 31 of the tile
  static __device__ inline typename Elem<T>::Frag frag(const T* tile, int line, int k) {
    const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
    if constexpr (PAIRS) {
      const int pair = line & ~31, second = (line >> 4) & 1;
      if constexpr (ROWS) {
        const int r = 8 * (i >> 2) + 4 * second + (i & 3);
        return *reinterpret_cast<const typename Elem<T>::Frag*>(tile + (pair + r) * 64 + ((k / 8 + g) ^ turn(r)) * 8);
      } else {
        const int row = k + 8 * g + (i >> 2);
        const T* p = tile + row * 256 + ((pair / 8 + (i & 3)) ^ turn(row)) * 8 + 4 * second;
        return join_transposed<T>(read_transposed(p), read_transposed(p + 4 * 256));
      }
    } else if constexpr (ROWS) {
      return *reinterpret_cast<const typename Elem<T>::Frag*>(tile + (line + i) * 64 + ((k / 8 + g) ^ turn(i)) * 8);
    } else {
      const int row = k + 8 * g + (i >> 2);                   // and four further on: the same turn
      const T* p = tile + row * 256 + ((line / 8 + ((i & 3) >> 1)) ^ turn(row)) * 8 + (i & 1) * 4;
      return join_transposed<T>(read_transposed(p), read_transposed(p + 4 * 256));
    }
  }
};

template <class T, bool L_ROWS, bool R_ROWS>
__global__ __launch_bounds__(512) void large_product_kernel(Product a) {
  constexpr int BK = 64, NB = 8, MB = 4, TILE = 256 * BK;
  __shared__ __attribute__((aligned(16))) T ls[2][TILE], rs[2][TILE];
  const int wave = threadIdx.x >> 6, wm = wave % 4 * 64, wn = wave / 4 * 128;
  const unsigned tm = (unsigned)(a.m + 255) / 256, tn = (unsigned)(a.n + 255) / 256;
  int row, col;
  tile_of(blockIdx.x, tm, tn, row, col);
  const int m0 = row * 256, n0 = col * 256, tiles = a.k / BK;

  LargeMove<T, L_ROWS, true> ml;
  LargeMove<T, R_ROWS, false> mr;
  ml.start(static_cast<const T*>(a.l), a.ld_l, n0, a.n, 0);
  mr.start(static_cast<const T*>(a.r), a.ld_r, m0, a.m, 0);
  floatx4 acc[NB][MB];
#pragma unroll
  for (int x = 0; x < NB; ++x)
#pragma unroll
    for (int y = 0; y < MB; ++y) acc[x][y] = floatx4{0.f, 0.f, 0.f, 0.f};

  if (tiles > 0) {
    ml.fetch();
    mr.fetch();
    ml.store(ls[0]);
    mr.store(rs[0]);
  }
  for (int t = 0; t < tiles; ++t) {
    __syncthreads();                                          // tile t is there, and nobody reads the other buffer any more
    const bool more = t + 1 < tiles;
    if (more) {
      ml.fetch();
      mr.fetch();
    }
    const T *l = ls[t & 1], *r = rs[t & 1];
#pragma unroll
    for (int s = 0; s < BK; s += 32) {
      typename Elem<T>::Frag lf[NB], rf[MB];
#pragma unroll
      for (int y = 0; y < MB; ++y) rf[y] = mr.frag(r, wm + y * 16, s);
#pragma unroll
      for (int x = 0; x < NB; ++x) lf[x] = ml.frag(l, wn + x * 16, s);
#pragma unroll
      for (int x = 0; x < NB; ++x)
#pragma unroll
        for (int y = 0; y < MB; ++y) acc[x][y] = Elem<T>::mma(lf[x], rf[y], acc[x][y]);
    }
    if (more) {
      ml.store(ls[(t + 1) & 1]);
      mr.store(rs[(t + 1) & 1]);
    }
  }

  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int y = 0; y < MB; ++y) {
    __builtin_amdgcn_sched_barrier(0);
    const int64_t m = m0 + wm + y * 16 + (lane & 15);
    if (m >= a.m) continue;
    auto each = [&](auto f) {
#pragma unroll
      for (int x = 0; x < NB; x += 2) {
        const int n = n0 + wn + x * 16 + 8 * (lane >> 4);
        if (n < a.n) f(n, acc[x][y], acc[x + 1][y]);
      }
    };
    if (a.bias) each([&](int n, floatx4& u, floatx4& v) { add8(static_cast<const T*>(a.bias), n, a.n, u, v); });
    if (a.pre) each([&](int n, floatx4& u, floatx4& v) { store8(static_cast<T*>(a.pre) + m * a.ld_pre, n, a.n, u, v); });
    switch (a.act) {
      case ACT_RELU: each([&](int, floatx4& u, floatx4& v) { activate<T, ACT_RELU>(u); activate<T, ACT_RELU>(v); }); break;
      case ACT_GELU: each([&](int, floatx4& u, floatx4& v) { activate<T, ACT_GELU>(u); activate<T, ACT_GELU>(v); }); break;
      case ACT_SILU: each([&](int, floatx4& u, floatx4& v) { activate<T, ACT_SILU>(u); activate<T, ACT_SILU>(v); }); break;
      default: break;
    }
    if (a.residual) each([&](int n, floatx4& u, floatx4& v) { add8(static_cast<const T*>(a.residual) + m * a.ld_res, n, a.n, u, v); });
    each([&](int n, floatx4& u, floatx4& v) { store8(static_cast<T*>(a.out) + m * a.ld_out, n, a.n, u, v); });
  }
}

// Sums of the splits, in their order, and the epilogue: four outputs a thread, or where the splits are many four outputs a lane, the four
// waves taking every fourth split.
constexpr int kManySplits = 12;
template <class T>
__global__ __launch_bounds__(256) void join_kernel(Product a) {
  __shared__ floatx4 part[4][64];
  const bool many = a.splits >= kManySplits;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per_row = (a.n + 3) / 4;
  const int64_t total = (int64_t)a.m * per_row, step = (int64_t)gridDim.x * (many ? 64 : 256);
  for (int64_t at = (int64_t)blockIdx.x * (many ? 64 : 256); at < total; at += step) {
    const int64_t i = at + (many ? lane : (int)threadIdx.x);
    const int64_t m = i / per_row;
    const int n = (int)(i - m * per_row) * 4;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    if (i < total) {
#pragma unroll 4
      for (int s = many ? wave : 0; s < a.splits; s += many ? 4 : 1) v += load4(a.part + ((int64_t)s * a.m + m) * a.n, n, a.n);
    }
    if (many) {
      __syncthreads();
      part[wave][lane] = v;
      __syncthreads();
      if (wave) continue;
      v = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
    }
    if (i < total) finish4<T>(a, m, n, v);
  }
}

// dz = dy act'(z), rounded to T as the operand of the products that follow (8,192 x 4,096 x 4,096 in bf16, against 64 bits: 0.0023 off in the norm,
// 0.0017 with a dz of 32 bits, which would take both products twice or on the fp32 units), and the sums of its unrounded columns over a workgroup's
// rows
template <class T>
__global__ __launch_bounds__(256) void dz_kernel(LinearGradArgs a, T* dz, int64_t ld_dz, float* sums, int rows_per) {
  __shared__ floatx4 wsum[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int cols = (a.d_out + 255) / 256, n = (int)(blockIdx.x % cols) * 256 + lane * 4, chunk = (int)(blockIdx.x / cols);
  const int64_t m1 = min((int64_t)a.rows, (int64_t)(chunk + 1) * rows_per);
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  if (n < a.d_out) {
    constexpr int U = 4;                                      // rows requested at once
    for (int64_t m = (int64_t)chunk * rows_per + wave; m < m1; m += 4 * U) {
      floatx4 v[U], z[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        v[u] = z[u] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (m + 4 * u >= m1) continue;
        v[u] = load4(static_cast<const T*>(a.dy) + (m + 4 * u) * a.ld_dy, n, a.d_out);
        if (dz) z[u] = load4(static_cast<const T*>(a.pre) + (m + 4 * u) * a.ld_pre, n, a.d_out);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (m + 4 * u >= m1) continue;
        if (dz) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[u][j] *= act_slope<T>(a.act, z[u][j]);
          store4(dz + (m + 4 * u) * ld_dz, n, a.d_out, v[u]);
        }
        acc += v[u];
      }
    }
  }
  if (!a.db) return;
  wsum[wave][lane] = acc;
  __syncthreads();
  if (wave == 0 && n < a.d_out) {
    const floatx4 v = (wsum[0][lane] + wsum[1][lane]) + (wsum[2][lane] + wsum[3][lane]);
    if (rows_per >= a.rows) store4(static_cast<T*>(a.db), n, a.d_out, v);       // all rows: no second launch
    else store4(sums + (int64_t)chunk * a.d_out, n, a.d_out, v);
  }
}

template <class T>
__global__ __launch_bounds__(1024) void db_kernel(const float* sums, int chunks, int n, T* db) {
  __shared__ float wsum[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (int)blockIdx.x * 64 + lane;
  float acc = 0.f;
  if (c < n) {
#pragma unroll 8
    for (int i = wave; i < chunks; i += 16) acc += sums[(int64_t)i * n + c];
  }
  wsum[wave][lane] = acc;
  __syncthreads();
  if (wave == 0 && c < n) {
#pragma unroll
    for (int w = 1; w < 16; ++w) acc += wsum[w][lane];
    db[c] = (T)acc;
  }
}

inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Plan { int bm, bn, splits, k_per; };

// Tiles of a product:
//   256 x 256  16-bit types, 256 such tiles or more, k of whole tiles (one at least: dW of no rows has none and reads nothing), rows per k
//              of whole pieces of 16 bytes
//   128 x 128, 112, 96, 64   256 such tiles or more that pad m by no more than a quarter over 64 rows; the width that pads n least (fp32, whose products are the bound: 40,000 x 372 x 200 97 us in
//              tiles of 128 columns, 87 in 112; 16-bit: 64 columns where n has no more, or 128 would pad a quarter more)
//              The same with k split, eight tiles of k a split at least, where that makes 384 workgroups or more.
//   64 x 64    everything smaller, k split while there are fewer than 1,024 workgroups, eight tiles of k a split at least: joining takes 4 to 8
//              us, a tile of k 0.4 to 0.8 (bf16 1,500 x 1,000 x 800 in one split 14.5 us, in three of five tiles 20.0; 700 x 2,000 x 1,500 in one
//              30.0, in three of eleven 22.7).
//   32 x 32    fp32 where those are fewer than 256: a wave's 32 x 32 outputs of 200 terms are 3 us of matrix instructions.
template <class T>
Plan plan_of(int64_t m, int64_t n, int64_t k, bool l_rows, bool r_rows) {
  constexpr int BK = kTileK<T>;
  const auto tiles_of = [&](int64_t bm, int64_t bn) { return ((m + bm - 1) / bm) * ((n + bn - 1) / bn); };
  const bool whole = sizeof(T) == 2 && k > 0 && k % 64 == 0 && (l_rows || n % 8 == 0) && (r_rows || m % 8 == 0);
  Plan p{256, 256, 1, (int)up(k < BK ? BK : k, BK)};
  if (whole && tiles_of(256, 256) >= 256) return p;
  p.bm = 128;
  p.bn = 128;
  if (sizeof(T) == 4) {
    for (int w : {112, 96, 64})
      if (up(n, w) < up(n, p.bn)) p.bn = w;
  } else if (up(n, 64) * 5 <= up(n, 128) * 4) {
    p.bn = 64;
  }
  const auto split = [&](int64_t workgroups, int64_t least) {
    const int64_t tiles = tiles_of(p.bm, p.bn);
    int64_t splits = tiles ? workgroups / tiles : 1;
    if (splits > k / (least * BK)) splits = k / (least * BK);
    if (splits < 1) splits = 1;
    p.k_per = (int)up((k + splits - 1) / splits, BK);
    if (p.k_per < BK) p.k_per = BK;
    p.splits = (int)((k + p.k_per - 1) / p.k_per);
    if (p.splits < 1) p.splits = 1;
  };
  if (up(m, 128) * 4 <= up(m, 64) * 5) {
    if (tiles_of(p.bm, p.bn) >= 256) return p;
    if (tiles_of(p.bm, p.bn) * (k / (8 * BK)) >= 384) {
      split(512, 8);
      return p;
    }
  }
  p.bm = p.bn = 64;
  split(1024, 8);
  if (sizeof(T) == 4 && tiles_of(64, 64) * p.splits < 256) {
    p.bm = p.bn = 32;
    split(1024, 8);
  }
  return p;
}

template <class T>
size_t part_bytes(int64_t m, int64_t n, int64_t k, bool l_rows, bool r_rows) {
  const Plan p = plan_of<T>(m, n, k, l_rows, r_rows);
  return p.splits > 1 ? (size_t)p.splits * m * n * sizeof(float) : 0;
}

template <class T, bool L_ROWS, bool R_ROWS>
hipError_t product(Product a, void* part, hipStream_t s) {
  if (a.m == 0 || a.n == 0) return hipSuccess;
  const Plan p = plan_of<T>(a.m, a.n, a.k, L_ROWS, R_ROWS);
  a.splits = p.splits;
  a.k_per = p.k_per;
  a.part = static_cast<float*>(part);
  const int64_t grid = ((a.m + (int64_t)p.bm - 1) / p.bm) * ((a.n + (int64_t)p.bn - 1) / p.bn) * p.splits;
  hipError_t e = hipErrorInvalidValue;
  if constexpr (sizeof(T) == 2) {
    if (p.bm == 256) e = launch(large_product_kernel<T, L_ROWS, R_ROWS>, grid, 512, s, a);
    else if (p.bn == 128) e = launch(product_kernel<T, 128, 128, 2, 2, 1, L_ROWS, R_ROWS>, grid, 256, s, a);
    else if (p.bm == 128) e = launch(product_kernel<T, 128, 64, 4, 1, 2, L_ROWS, R_ROWS>, grid, 256, s, a);
  } else {
    if (p.bm == 32) e = launch(product_kernel<T, 32, 32, 2, 2, 3, L_ROWS, R_ROWS>, grid, 256, s, a);
    else if (p.bn == 128) e = launch(product_kernel<T, 128, 128, 2, 2, 1, L_ROWS, R_ROWS>, grid, 256, s, a);
    else if (p.bn == 112) e = launch(product_kernel<T, 128, 112, 4, 1, 1, L_ROWS, R_ROWS>, grid, 256, s, a);
    else if (p.bn == 96) e = launch(product_kernel<T, 128, 96, 4, 1, 1, L_ROWS, R_ROWS>, grid, 256, s, a);
    else if (p.bm == 128) e = launch(product_kernel<T, 128, 64, 4, 1, 1, L_ROWS, R_ROWS>, grid, 256, s, a);
  }
  if (p.bm == 64) e = launch(product_kernel<T, 64, 64, 2, 2, 3, L_ROWS, R_ROWS>, grid, 256, s, a);
  if (e != hipSuccess || p.splits == 1) return e;
  const int per = p.splits >= kManySplits ? 64 : 256;
  const int64_t blocks = ((int64_t)a.m * ((a.n + 3) / 4) + per - 1) / per;
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
  const int64_t most = a.rows <= 64 ? 1 : (a.rows + 15) / 16;
  if (chunks > most) chunks = most;
  if (chunks < 1) chunks = 1;
  g.rows_per = (int)((a.rows + chunks - 1) / chunks);
  if (g.rows_per < 1) g.rows_per = 1;
  g.chunks = (int)chunks;
  g.sums = a.act != ACT_NONE ? (size_t)up((int64_t)a.rows * g.ld_dz * sizeof(T), 256) : 0;
  g.part = g.sums + (a.db && g.chunks > 1 ? (size_t)up((int64_t)g.chunks * a.d_out * sizeof(float), 256) : 0);
  const size_t px = a.dx ? part_bytes<T>(a.rows, a.d_in, a.d_out, true, true) : 0, pw = a.dw ? part_bytes<T>(a.d_in, a.d_out, a.rows, false, false) : 0;
  g.total = g.part + (px > pw ? px : pw);
  return g;
}

template <class T>
hipError_t backward(const LinearGradArgs& f, void* ws, hipStream_t s) {
  const GradLayout g = layout_of<T>(f);
  char* base = static_cast<char*>(ws);
  T* dz = f.act != ACT_NONE ? reinterpret_cast<T*>(base) : nullptr;
  float* sums = f.db && g.chunks > 1 ? reinterpret_cast<float*>(base + g.sums) : nullptr;
  hipError_t e = hipSuccess;
  if (dz || f.db) {
    e = launch(dz_kernel<T>, (int64_t)g.chunks * ((f.d_out + 255) / 256), 256, s, f, dz, g.ld_dz, sums, g.rows_per);
    if (e == hipSuccess && sums) e = launch(db_kernel<T>, (f.d_out + 63) / 64, 1024, s, (const float*)sums, g.chunks, f.d_out, static_cast<T*>(f.db));
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
