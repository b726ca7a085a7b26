// The dense product of operands in 8 bits, sums of 32-bit integers, on gfx950's matrix cores:
//
//   y = act(x_scale[m] w_scale[n] sum_k x[m][k] w[n][k] + bias[n]) + residual
//
// Both operands have k along their rows, so every fragment is 16 neighbouring bytes.  Accumulators hold the transposed tile, four neighbouring columns
// of one output row a lane.  Kernels:
//   fragments  operands go from memory into the matrix instructions without LDS, eight waves share k and add up at the end: for few rows or small outputs,
//              where what counts is one latency instead of one for each tile of k
//   64 x 64    tiles through registers into LDS, any alignment, k split where tiles are few
//   128 x 128  the same, and as a variant whose tiles go from memory into LDS directly, for operands in whole pieces of 16 bytes
//   in turns   256 x 256 and 128 x 128, directly too: two groups of four waves, one multiplying while the other reads
#pragma once
#include <utility>

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

// ---- fragments straight from memory

// The last `count` of a piece's 16 bytes, zeros in front (0 and less: none; 16 and more: all)
__device__ inline i32x4 last_bytes(const i32x4& v, int count) {
  i32x4 r;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int first = 16 - count - 4 * d;                     // of the word's bytes
    r[d] = first <= 0 ? v[d] : first >= 4 ? 0 : (int)((uint32_t)v[d] & (0xFFFFFFFFu << 8 * first));
  }
  return r;
}
// A piece of a row at k: past the row's whole pieces its last 16 bytes, which both operands read alike; of the rows' side what was there before is
// taken out by last_bytes
__device__ inline i32x4 piece_at(const int8_t* row, int k, int total) {
  if (total < 16) return __builtin_bit_cast(i32x4, load16<int8_t, kShort>(row, k == 0 ? total : 0));
  return __builtin_bit_cast(i32x4, *reinterpret_cast<const u32x4_any*>(row + min(k, total - 16)));
}

// 16 MB rows and 16 NB columns a workgroup; eight waves take 128 bytes of k each in turn, four of their turns are on their way at once (4 x 4,096 x 4,096: 5.9
// us, 2.9 TB/s of weights with the launch, and 11 in tiles of 64 x 64 with 8 splits and their joining; 1,024 x 1,024 x 1,024: 8.3 and 12)
template <class T, int MB, int NB>
__global__ __launch_bounds__(512) void fragments_kernel(Product a) {
  constexpr int WAVES = 8, DEPTH = MB + NB > 6 ? 2 : 4;
  __shared__ i32x4 part[WAVES][MB * NB][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, g = lane >> 4;
  const unsigned tm = (unsigned)(a.m + 16 * MB - 1) / (16 * MB), tn = (unsigned)(a.n + 16 * NB - 1) / (16 * NB);
  int row, col;
  dense::tile_of(blockIdx.x, tm, tn, row, col);
  const int m0 = row * 16 * MB, n0 = col * 16 * NB;
  const int8_t *l[NB], *r[MB];
#pragma unroll
  for (int x = 0; x < NB; ++x) l[x] = a.l + (int64_t)min(n0 + x * 16 + i16, a.n - 1) * a.ld_l;
#pragma unroll
  for (int y = 0; y < MB; ++y) r[y] = a.r + (int64_t)min(m0 + y * 16 + i16, a.m - 1) * a.ld_r;
  i32x4 lf[DEPTH][2][NB], rf[DEPTH][2][MB], acc[NB][MB];
#pragma unroll
  for (int x = 0; x < NB; ++x)
#pragma unroll
    for (int y = 0; y < MB; ++y) acc[x][y] = i32x4{0, 0, 0, 0};
  auto fetch = [&](int d, int k0) {
    if (k0 + kBK <= a.k) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int k = k0 + s * 64 + g * 16;
#pragma unroll
        for (int x = 0; x < NB; ++x) lf[d][s][x] = __builtin_bit_cast(i32x4, *reinterpret_cast<const u32x4_any*>(l[x] + k));
#pragma unroll
        for (int y = 0; y < MB; ++y) rf[d][s][y] = __builtin_bit_cast(i32x4, *reinterpret_cast<const u32x4_any*>(r[y] + k));
      }
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int k = k0 + s * 64 + g * 16;
#pragma unroll
        for (int x = 0; x < NB; ++x) lf[d][s][x] = piece_at(l[x], k, a.k);
#pragma unroll
        for (int y = 0; y < MB; ++y) rf[d][s][y] = a.k < 16 ? piece_at(r[y], k, a.k) : last_bytes(piece_at(r[y], k, a.k), a.k - k);
      }
    }
  };
  constexpr int STEP = WAVES * kBK;
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (wave * kBK + d * STEP < a.k) fetch(d, wave * kBK + d * STEP);
  for (int kt = wave * kBK; kt < a.k; kt += DEPTH * STEP) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int k = kt + d * STEP;
      if (k >= a.k) break;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int x = 0; x < NB; ++x)
#pragma unroll
          for (int y = 0; y < MB; ++y) acc[x][y] = Elem<int8_t>::mma(lf[d][s][x], rf[d][s][y], acc[x][y]);
      if (k + DEPTH * STEP < a.k) fetch(d, k + DEPTH * STEP);
    }
  }
#pragma unroll
  for (int x = 0; x < NB; ++x)
#pragma unroll
    for (int y = 0; y < MB; ++y) part[wave][x * MB + y][lane] = acc[x][y];
  __syncthreads();
  for (int b = wave; b < MB * NB; b += WAVES) {
    i32x4 sum = part[0][b][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += part[w][b][lane];
    const int m = m0 + b % MB * 16 + i16, n = n0 + b / MB * 16 + 4 * g;
    if (m < a.m && n < a.n) finish4<T>(a, m, n, sum);
  }
}

// ---- tiles through registers

// DEPTH tiles of k are on their way in registers while one is multiplied; with one, two are in LDS and a barrier a tile is enough (as in the kernel of
// other types: where tiles are small and few, what a tile takes is the wait for memory).
template <class T, int BM, int BN, int WM, int WN, int DEPTH>
__global__ __launch_bounds__(WM * WN * 64, BM * BN <= 64 * 64 ? 4 : 2) void product_kernel(Product a) {
  using El = Elem<int8_t>;
  constexpr int THREADS = WM * WN * 64, MB = BM / WM / 16, NB = BN / WN / 16, S = lds_stride<int8_t>(kBK), BUFS = DEPTH == 1 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) int8_t ls[BUFS][BN * S], rs[BUFS][BM * S];
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
  auto fetch = [&](int d, int k) {
    ml.fetch(rl[d], k);
    mr.fetch(rr[d], k);
  };
  auto multiply = [&](const int8_t* l, const int8_t* r) {
#pragma unroll
    for (int s = 0; s < kBK; s += El::KF) {
      i32x4 lf[NB], rf[MB];
#pragma unroll
      for (int x = 0; x < NB; ++x) lf[x] = frag_rows(l, S, wn + x * 16, s);
#pragma unroll
      for (int y = 0; y < MB; ++y) rf[y] = frag_rows(r, S, wm + y * 16, s);
#pragma unroll
      for (int x = 0; x < NB; ++x)
#pragma unroll
        for (int y = 0; y < MB; ++y) acc[x][y] = El::mma(lf[x], rf[y], acc[x][y]);
    }
  };
  if constexpr (DEPTH == 1) {
    if (kb < ke) {
      fetch(0, kb);
      ml.store(ls[0], rl[0]);
      mr.store(rs[0], rr[0]);
    }
    int buf = 0;
    for (int k = kb; k < ke; k += kBK, buf ^= 1) {
      __syncthreads();
      const bool more = k + kBK < ke;
      if (more) fetch(0, k + kBK);
      multiply(ls[buf], rs[buf]);
      if (more) {
        ml.store(ls[buf ^ 1], rl[0]);
        mr.store(rs[buf ^ 1], rr[0]);
      }
    }
  } else {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (kb + d * kBK < ke) fetch(d, kb + d * kBK);
    for (int kt = kb; kt < ke; kt += DEPTH * kBK) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        const int k = kt + d * kBK;
        if (k >= ke) break;
        __syncthreads();
        ml.store(ls[0], rl[d]);
        mr.store(rs[0], rr[d]);
        __syncthreads();
        if (k + DEPTH * kBK < ke) fetch(d, k + DEPTH * kBK);
        multiply(ls[0], rs[0]);
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

// ---- tiles from memory into LDS directly

// 16 bytes a lane from base + off into the wave's 1,024 bytes of LDS from `lds` on, lane after lane.  No register receives anything; the compiler does not
// know that a load is on its way, wait_loads waits for it.
__device__ inline void load_lds(const int8_t* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
template <int N>                                              // until N of this wave's latest loads are on their way at most
__device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ inline void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// a barrier that waits for no load: what a wave needs to have finished, it waits for itself in front
__device__ inline void meet_here() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
__device__ inline uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }

// LDS rows hold BK bytes of k unpadded; piece p of row r lies at p ^ turn(r).  LDS gives 256 bytes a cycle to sixteen lanes of a 16-byte read, and those are lanes 0 .. 3 and
// 12 .. 15 of one lane group with 4 .. 11 of the next: rows i of 0 .. 3 and 12 .. 15 at piece p and of 4 .. 11 at p ^ 1.  With these turns they lie in
// sixteen different places of 256 bytes (counted: no conflicts; with the row's number as its turn every read of 64-byte rows took two cycles).  The column side's
// fragments come in pairs: of 32 columns the first holds 8 q + 0 .. 3 (q = 0 .. 3) and the second 8 q + 4 .. 7, so that a lane's two accumulators are
// eight neighbouring outputs.
template <int BK, bool PAIRS>
struct Direct {
  static constexpr int PIECES = BK / 16;
  static __device__ inline int turn(int r) {
    if (BK == 64) {
      const int q = PAIRS ? r >> 3 : r >> 2;
      return ((q ^ q >> 1) & 1) << 1 | (q >> 1 & 1);
    }
    return PAIRS ? ((r >> 2) & 6) | ((r >> 1) & 1) : (r >> 1) & 7;
  }
  // offset of this lane's piece of the wave's load number i from the tile's first row on, and which piece of the tile's k it is
  static __device__ inline int row_of(int load) { return load * (64 / PIECES) + (int)(threadIdx.x & 63) / PIECES; }
  static __device__ inline int piece_of(int row) { return ((int)threadIdx.x & (PIECES - 1)) ^ turn(row); }
  static __device__ inline i32x4 frag(const int8_t* tile, int line, int k) {
    const int lane = threadIdx.x & 63, i = lane & 15;
    const int r = PAIRS ? (line & ~31) + 8 * (i >> 2) + ((line >> 2) & 4) + (i & 3) : line + i;
    return *reinterpret_cast<const i32x4*>(tile + r * BK + ((k / 16 + (lane >> 4)) ^ turn(r)) * 16);
  }
};

// Loads of one operand's tiles of LINES rows, LOADS a wave: rows past the matrix's last repeat it; past k (TAIL: k may end inside a tile) the row's last
// piece is repeated
template <int BK, bool PAIRS, int LINES, int WAVES, bool TAIL>
struct DirectMove {
  using D = Direct<BK, PAIRS>;
  static constexpr int LOADS = LINES * BK / 1024 / WAVES;
  const int8_t* base;                                         // the tile's first row at its k
  uint32_t off[LOADS];
  __device__ inline void start(const int8_t* matrix, int64_t ld, int first, int lines, int k, int wave) {
    base = matrix + (int64_t)first * ld + k;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int r = D::row_of(wave * LOADS + i);
      off[i] = (uint32_t)(min(first + r, lines - 1) - first) * (uint32_t)ld + D::piece_of(r) * 16;
    }
  }
  // left: bytes of k from this tile on, a multiple of 16
  __device__ inline void issue(uint32_t lds, int wave, int left) {
    const uint32_t to = lds + wave * LOADS * 1024;
    if (!TAIL || left >= BK) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) load_lds(base, off[i], to + i * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int past = D::piece_of(D::row_of(wave * LOADS + i)) * 16 + 16 - left;
        load_lds(base, off[i] - max(past, 0), to + i * 1024);
      }
    }
    base += BK;
  }
};

// Eight neighbouring outputs of row m; `residual`: theirs, where all eight are there and the type has 16 bits
template <class T>
__device__ inline void finish8(const Product& a, int64_t m, int n, float rs, const i32x4& s, const i32x4& t, const u32x4& residual) {
  const bool both = n + 4 < a.n;
  floatx4 u = scaled(s, rs, load4(a.l_scale, n, a.n)), v = {0.f, 0.f, 0.f, 0.f};
  if (both) v = scaled(t, rs, load4(a.l_scale, n + 4, a.n));
  auto add = [&](const T* row) {
    if constexpr (sizeof(T) == 2) {
      add8(row, n, a.n, u, v);
    } else {
      u += load4(row, n, a.n);
      if (both) v += load4(row, n + 4, a.n);
    }
  };
  if (a.bias) add(static_cast<const T*>(a.bias));
  activate<T>(a.act, u);
  activate<T>(a.act, v);
  if (a.residual) {
    if (sizeof(T) == 2 && n + 8 <= a.n) {
      if constexpr (sizeof(T) == 2) {
        const typename Elem<T>::Frag f = __builtin_bit_cast(typename Elem<T>::Frag, residual);
#pragma unroll
        for (int j = 0; j < 4; ++j) { u[j] += (float)f[j]; v[j] += (float)f[j + 4]; }
      }
    } else {
      add(static_cast<const T*>(a.residual) + m * a.ld_res);
    }
  }
  T* out = static_cast<T*>(a.out) + m * a.ld_out;
  if constexpr (sizeof(T) == 2) {
    store8(out, n, a.n, u, v);
  } else {
    store4(out, n, a.n, u);
    if (both) store4(out, n + 4, a.n, v);
  }
}

// A wave's blocks from output (m0, n0), columns in pairs of blocks.  The residual of sixteen rows is on its way while the sixteen rows before are finished.
template <class T, int NB, int MB>
__device__ __forceinline__ void finish_pairs(const Product& a, int split, int m0, int n0, i32x4 (&acc)[NB][MB]) {
  const int lane = threadIdx.x & 63, first = n0 + 8 * (lane >> 4);
  u32x4 ahead[2][NB / 2];
  auto ask = [&](int y) {
    const int64_t m = m0 + y * 16 + (lane & 15);
#pragma unroll
    for (int x = 0; x < NB / 2; ++x) {
      ahead[y & 1][x] = u32x4{0, 0, 0, 0};
      if (sizeof(T) == 2 && a.residual && a.splits == 1 && m < a.m && first + x * 32 + 8 <= a.n)
        ahead[y & 1][x] = *reinterpret_cast<const u32x4_any*>(static_cast<const T*>(a.residual) + m * a.ld_res + first + x * 32);
    }
  };
  ask(0);
#pragma unroll
  for (int y = 0; y < MB; ++y) {
    if (y + 1 < MB) ask(y + 1);
    __builtin_amdgcn_sched_barrier(0);
    const int64_t m = m0 + y * 16 + (lane & 15);
    if (m >= a.m) continue;
    const float rs = a.r_scale[m];
#pragma unroll
    for (int x = 0; x < NB; x += 2) {
      const int n = first + x * 16;
      if (n >= a.n) continue;
      if (a.splits > 1) {
        int* row = a.part + (split * (int64_t)a.m + m) * a.n;
        store_sums(row, n, a.n, acc[x][y]);
        if (n + 4 < a.n) store_sums(row, n + 4, a.n, acc[x + 1][y]);
      } else {
        finish8<T>(a, m, n, rs, acc[x][y], acc[x + 1][y], ahead[y & 1][x / 2]);
      }
    }
  }
}

// 128 x 128 outputs a workgroup of four waves, two tiles of 128 bytes of k in LDS, one barrier a tile; two workgroups a CU, so that one's epilogue
// runs beside the other's products
template <class T>
__global__ __launch_bounds__(256, 2) void direct_kernel(Product a) {
  constexpr int MB = 4, NB = 4, TILE = 128 * kBK;
  __shared__ __attribute__((aligned(16))) int8_t lds[4 * TILE];           // tile of the columns | of the rows, twice
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
  const unsigned tm = (unsigned)(a.m + 127) / 128, tn = (unsigned)(a.n + 127) / 128;
  const int split = (int)(blockIdx.x / (tm * tn));
  int row, col;
  dense::tile_of(blockIdx.x % (tm * tn), tm, tn, row, col);
  const int m0 = row * 128, n0 = col * 128;
  const int kb = split * a.k_per, ke = min(a.k, kb + a.k_per);
  DirectMove<kBK, true, 128, 4, true> ml;
  DirectMove<kBK, false, 128, 4, true> mr;
  ml.start(a.l, a.ld_l, n0, a.n, kb, wave);
  mr.start(a.r, a.ld_r, m0, a.m, kb, wave);
  const uint32_t to = lds_address(lds);
  i32x4 acc[NB][MB];
#pragma unroll
  for (int x = 0; x < NB; ++x)
#pragma unroll
    for (int y = 0; y < MB; ++y) acc[x][y] = i32x4{0, 0, 0, 0};
  if (kb < ke) {
    ml.issue(to, wave, ke - kb);
    mr.issue(to + TILE, wave, ke - kb);
  }
  int buf = 0;
  for (int k = kb; k < ke; k += kBK, buf ^= 1) {
    wait_loads<0>();
    wait_lds();
    meet_here();                                              // the tile is there, and nobody reads the other buffer any more
    if (k + kBK < ke) {
      ml.issue(to + (buf ^ 1) * 2 * TILE, wave, ke - k - kBK);
      mr.issue(to + (buf ^ 1) * 2 * TILE + TILE, wave, ke - k - kBK);
    }
    const int8_t *l = lds + buf * 2 * TILE, *r = l + TILE;
#pragma unroll
    for (int s = 0; s < kBK; s += 64) {
      i32x4 lf[NB], rf[MB];
#pragma unroll
      for (int y = 0; y < MB; ++y) rf[y] = Direct<kBK, false>::frag(r, wm + y * 16, s);
#pragma unroll
      for (int x = 0; x < NB; ++x) lf[x] = Direct<kBK, true>::frag(l, wn + x * 16, s);
      if (k + kBK > ke) {                                     // (uniform) past k: zeros on the rows' side
#pragma unroll
        for (int y = 0; y < MB; ++y) rf[y] = k + s + (lane >> 4) * 16 < ke ? rf[y] : i32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int x = 0; x < NB; ++x)
#pragma unroll
        for (int y = 0; y < MB; ++y) acc[x][y] = Elem<int8_t>::mma(lf[x], rf[y], acc[x][y]);
    }
  }
  finish_pairs<T, NB, MB>(a, split, m0 + wm, n0 + wn, acc);
}

// until `tiles` of this wave's latest tiles of LOADS loads are on their way at most
template <int LOADS, int MOST>
__device__ inline void wait_tiles(int tiles) {
  if constexpr (MOST == 0) {
    wait_loads<0>();
  } else {
    if (tiles >= MOST) wait_loads<LOADS * MOST>();
    else wait_tiles<LOADS, MOST - 1>(tiles);
  }
}

// BM x BN outputs a workgroup of eight waves, BUFS tiles of 64 bytes of k in LDS.  Two groups of four waves, one of each on every SIMD, half a step
// apart: while one group multiplies, the other reads its next fragments and asks for a tile BUFS - 1 steps on, so that the matrix pipe has work all the
// time.
//  - A tile is read by either group after the barrier behind which both have waited for their own loads of it: the wait for tile t + 1 is in
//    front of the barrier that ends a group's reading of tile t.
//  - A buffer is written again (the loads of tile t + BUFS - 1) after the barrier behind which both groups have their fragments of tile t - 1 in registers.
// Group 1 waits once more in front of the loop, group 0 behind it: both pass the same number of barriers.  k is whole tiles (a last tile that k may end in
// cost 6 us of 146 at 8,192 x 4,096 x 4,096).
template <class T, int BM, int BN, int WM, int WN, int BUFS>
__global__ __launch_bounds__(512) void turns_kernel(Product a) {
  constexpr int BK = 64, MB = BM / WM / 16, NB = BN / WN / 16, LT = BN * BK, TILE = (BM + BN) * BK, LOADS = TILE / 1024 / 8;
  static_assert(WM * WN == 8, "eight waves");
  __shared__ __attribute__((aligned(16))) int8_t lds[BUFS * TILE];        // the columns' tile | the rows' tile, BUFS times
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wm = wave % WM * MB * 16, wn = wave / WM * NB * 16;
  const unsigned tm = (unsigned)(a.m + BM - 1) / BM, tn = (unsigned)(a.n + BN - 1) / BN;
  const int split = (int)(blockIdx.x / (tm * tn));
  int row, col;
  dense::tile_of(blockIdx.x % (tm * tn), tm, tn, row, col);
  const int m0 = row * BM, n0 = col * BN, kb = split * a.k_per, tiles = (min(a.k, kb + a.k_per) - kb) / BK;
  DirectMove<BK, true, BN, 8, false> ml;
  DirectMove<BK, false, BM, 8, false> mr;
  static_assert(decltype(ml)::LOADS + decltype(mr)::LOADS == LOADS, "loads of a tile and wave");
  ml.start(a.l, a.ld_l, n0, a.n, kb, wave);
  mr.start(a.r, a.ld_r, m0, a.m, kb, wave);
  const uint32_t to = lds_address(lds);
  auto issue = [&](int buf) {
    ml.issue(to + buf * TILE, wave, BK);
    mr.issue(to + buf * TILE + LT, wave, BK);
  };
  i32x4 acc[NB][MB];
#pragma unroll
  for (int x = 0; x < NB; ++x)
#pragma unroll
    for (int y = 0; y < MB; ++y) acc[x][y] = i32x4{0, 0, 0, 0};
  for (int t = 0; t < BUFS - 1 && t < tiles; ++t) issue(t);
  wait_tiles<LOADS, BUFS - 2>(tiles - 1);
  meet_here();
  if (wave >= 4) meet_here();
  int buf = 0;
  for (int t = 0; t < tiles; ++t) {
    const int8_t *l = lds + buf * TILE, *r = l + LT;
    i32x4 lf[NB], rf[MB];
#pragma unroll
    for (int y = 0; y < MB; ++y) rf[y] = Direct<BK, false>::frag(r, wm + y * 16, 0);
#pragma unroll
    for (int x = 0; x < NB; ++x) lf[x] = Direct<BK, true>::frag(l, wn + x * 16, 0);
    if (t + BUFS - 1 < tiles) {
      issue(buf == 0 ? BUFS - 1 : buf - 1);
      wait_loads<LOADS*(BUFS - 2)>();
    } else {
      wait_tiles<LOADS, BUFS - 2>(tiles - 2 - t);
    }
    wait_lds();
    meet_here();
#pragma unroll
    for (int x = 0; x < NB; ++x)
#pragma unroll
      for (int y = 0; y < MB; ++y) acc[x][y] = Elem<int8_t>::mma(lf[x], rf[y], acc[x][y]);
    meet_here();
    buf = buf == BUFS - 1 ? 0 : buf + 1;
  }
  if (wave < 4) meet_here();
  finish_pairs<T, NB, MB>(a, split, m0 + wm, n0 + wn, acc);
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

enum Kind { kFragments, kSmall, kMiddle, kDirect, kTurns, kLarge };
struct Plan { Kind kind; int splits, k_per, mb, nb; };         // mb, nb: blocks of 16 rows and columns (fragments)

// Operands in whole pieces of 16 bytes, whose tiles' offsets are 32-bit numbers
inline bool whole_pieces(const Linear8Args& f) {
  return f.d_in % 16 == 0 && f.ld_x % 16 == 0 && f.ld_w % 16 == 0 && f.ld_x < (1 << 23) && f.ld_w < (1 << 23) &&
         reinterpret_cast<uintptr_t>(f.x) % 16 == 0 && reinterpret_cast<uintptr_t>(f.w) % 16 == 0;
}

// Which kernel, by the number of tiles and the length of their sums (us, bf16 outputs with the full epilogue; each pair is the two sides of a rule):
//   fragments  the smallest tile that makes 256 workgroups at most (500 x 500 x 500: 32 x 32 4.0, 32 x 16 4.1, 32 x 64 4.5; 16 x 11,008 x 4,096: 32 x 64 13.3, 16 x 16 14.6) and
//              reads 400 KB of operands a workgroup at most (256 x 2,048 x 4,096, 393 KB: 14.5, in 128 x 128 16.6; 128 x 4,096 x 8,192, 786 KB: 25.5 and
//              20.4), with up to 16 rows 1 MB; rows that no 16 bytes align cost it three times that: 64 KB (100 x 1,000 x 999, 48 KB: 5.8, in 64 x 64 8.4;
//              1,000 x 257 x 1,999, 192 KB: 15.9 and 13.5)
//   256 x 256  whole tiles of 64 of k, long sums, and tiles that fill the 256 CUs' rounds to nine tenths: 8,192 x 4,096 x 4,096 153, in 128 x 128 182;
//              2,048 x 8,192 x 4,096 95 and 104; but 5,000 x 4,096 x 4,096 (320 tiles) 141 and 130
//   128 x 128  from 2^32 multiplications on (padded) where tiles go into LDS directly: 512 x 4,096 x 4,096 24.1, in 64 x 64 31.5; 16,384 x 256 x 1,024 17.7 and
//              19.3; but 512 x 4,096 x 1,024 16.8 and 14.2; k split to make a workgroup for every CU (200 x 4,096 x 4,096 in one 26.5, in four 18.6);
//              by eight waves in turns where a CU has one workgroup at most or little to sum (2,048 x 2,048 x 2,048 20.1, by four waves 22.1; 4,096 x 8,192 x 256
//              66 and 70; but 16,384 x 1,024 x 1,024 50 and 47)
//              from 2^34 on through registers: 1,024 x 4,096 x 4,096 42 and 47; but 4,000 x 1,000 x 1,000 28 and 20
//   64 x 64    everything smaller, k split while there are fewer than 1,024 workgroups, eight tiles of k a split at least, four where there are few workgroups
//              (70 x 64 x 8,192 in 8 splits 12.6, in 16 9.1)
inline Plan plan_of(int64_t m, int64_t n, int64_t k, bool whole) {
  const auto tiles_of = [&](int64_t b) { return ((m + b - 1) / b) * ((n + b - 1) / b); };
  Plan p{kFragments, 1, (int)up(k, kBK), 0, 0};
  const int64_t most = !whole ? 64 << 10 : m <= 16 ? 1 << 20 : 400 << 10;
  for (const auto& b : {std::pair<int, int>{1, 1}, {2, 1}, {2, 2}, {2, 4}, {4, 4}}) {
    p.mb = b.first;
    p.nb = b.second;
    if (((m + 16 * p.mb - 1) / (16 * p.mb)) * ((n + 16 * p.nb - 1) / (16 * p.nb)) > 256) continue;
    if (16 * (p.mb + p.nb) * k <= most) return p;
    break;
  }
  const auto split = [&](int64_t tiles, int64_t workgroups, int64_t least) {
    int64_t splits = workgroups / tiles;
    if (splits > k / (least * kBK)) splits = k / (least * kBK);
    if (splits < 1) splits = 1;
    p.k_per = (int)up((k + splits - 1) / splits, kBK);
    p.splits = (int)((k + p.k_per - 1) / p.k_per);
  };
  const int64_t large = tiles_of(256), middle = tiles_of(128), small = tiles_of(64), rounds = (large + 255) / 256;
  if (whole && k % 64 == 0 && k >= 1024 && large * 10 >= rounds * 256 * 9) {
    p.kind = kLarge;
  } else if (whole && middle * k >= 1 << 18) {
    p.kind = kDirect;
    split(middle, 256, 8);
    if (k % 64 == 0 && p.splits == 1 && (middle <= 256 || k <= 512)) p.kind = kTurns;
  } else if (middle * k >= 1 << 20 && middle >= 256) {
    p.kind = kMiddle;
  } else {
    p.kind = kSmall;
    split(small, 1024, small * (k / (8 * kBK)) < 64 ? 4 : 8);
  }
  return p;
}

inline size_t part_bytes(const Linear8Args& f) {
  if (f.rows == 0) return 0;                                  // (a plan has a tile at least)
  // (the pointers' alignment is not known where the workspace is asked for: enough for either)
  const Plan p = plan_of(f.rows, f.d_out, f.d_in, true), q = plan_of(f.rows, f.d_out, f.d_in, false);
  const int splits = p.splits > q.splits ? p.splits : q.splits;
  return splits > 1 ? (size_t)splits * f.rows * f.d_out * sizeof(int) : 0;
}

template <class T>
hipError_t run(Product a, const Plan& p, void* ws, hipStream_t s) {
  a.splits = p.splits;
  a.k_per = p.k_per;
  a.part = static_cast<int*>(ws);
  const auto grid = [&](int64_t b) { return ((a.m + b - 1) / b) * ((a.n + b - 1) / b) * p.splits; };
  hipError_t e = hipErrorInvalidValue;
  switch (p.kind) {
    case kFragments: {
      const int64_t n = ((a.m + 16 * p.mb - 1) / (16 * p.mb)) * (int64_t)((a.n + 16 * p.nb - 1) / (16 * p.nb));
      if (p.mb == 1) return launch(fragments_kernel<T, 1, 1>, n, 512, s, a);
      if (p.mb == 4) return launch(fragments_kernel<T, 4, 4>, n, 512, s, a);
      if (p.nb == 1) return launch(fragments_kernel<T, 2, 1>, n, 512, s, a);
      if (p.nb == 2) return launch(fragments_kernel<T, 2, 2>, n, 512, s, a);
      return launch(fragments_kernel<T, 2, 4>, n, 512, s, a);
    }
    case kSmall: e = launch(product_kernel<T, 64, 64, 2, 2, 3>, grid(64), 256, s, a); break;
    case kMiddle: e = launch(product_kernel<T, 128, 128, 2, 2, 1>, grid(128), 256, s, a); break;
    case kDirect: e = launch(direct_kernel<T>, grid(128), 256, s, a); break;
    case kTurns: return launch(turns_kernel<T, 128, 128, 2, 4, 5>, grid(128), 512, s, a);
    case kLarge: return launch(turns_kernel<T, 256, 256, 4, 2, 4>, grid(256), 512, s, a);
  }
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t blocks = ((int64_t)a.m * ((a.n + 3) / 4) + 255) / 256;
  return launch(join_kernel<T>, blocks < 4096 ? blocks : 4096, 256, s, a);
}

template <class T>
hipError_t forward(const Linear8Args& f, void* ws, hipStream_t s) {
  Product a{};
  a.l = f.w; a.ld_l = f.ld_w; a.r = f.x; a.ld_r = f.ld_x;
  a.m = f.rows; a.n = f.d_out; a.k = f.d_in;
  a.r_scale = f.x_scale; a.l_scale = f.w_scale;
  a.bias = f.bias; a.residual = f.residual; a.ld_res = f.ld_res;
  a.out = f.y; a.ld_out = f.ld_y; a.act = f.act;
  return run<T>(a, plan_of(a.m, a.n, a.k, whole_pieces(f)), ws, s);
}

}  // namespace dense8
}  // namespace stgn
