// The dense product of operands in 8 bits, sums of 32-bit integers, on gfx950's matrix cores:
//
//   y = act(x_scale[m] w_scale[n] sum_k x[m][k] w[n][k] + bias[n]) + residual
//
// Both operands have k along their rows, so every fragment is 16 neighbouring bytes.  Accumulators hold the transposed tile, four neighbouring columns
// of one output row a lane.  Kernels:
//   fragments  operands go from memory into the matrix instructions without LDS, eight waves share k and add up at the end: for few rows or small outputs,
//              where what counts is one latency instead of one for each tile of k
//   64 x 64    tiles through registers into LDS, any alignment, k split where tiles are few
//   128 x 128  tiles from memory into LDS directly, for operands in whole pieces of 16 bytes, or laid out so first
//   256 x 256  directly too, in turns: two groups of four waves, one multiplying while the other reads
// Sizes in these comments are rows x columns x k.  Figures are us of kernels with bf16 outputs, bias, gelu and residual, launched one after the other from a program in C++, up to
// four sets of operands and outputs in turn; where two are given for one size, both are of one run, and another run's or card's are up to a tenth off.  Through the binding,
// where a result takes the place of the one before it, the same kernels take less (8,192 x 4,096 x 4,096 141 us, 155 here).
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

// Four neighbouring numbers of a row as they lie in memory, those that it has
template <class T>
__device__ inline typename Elem<T>::Four ask4(const T* row, int n, int cols) {
  using Bits = std::conditional_t<sizeof(T) == 4, u32x4_any, u32x2_any>;
  if (n + 4 <= cols) return __builtin_bit_cast(typename Elem<T>::Four, *reinterpret_cast<const Bits*>(row + n));
  typename Elem<T>::Four f;
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] = n + j < cols ? row[n + j] : (T)0.f;
  return f;
}
// What four neighbouring outputs of row m take beside their sums: scales, bias, activation, residual.  Asked for in front of the sums, so that their latency and
// that of the operands are one.
template <class T>
struct Ends {
  typename Elem<T>::Four bias, residual;
  floatx4 ls;
  float rs;
  __device__ inline void ask(const Product& a, int64_t m, int n) {
    rs = a.r_scale[m];
    ls = __builtin_bit_cast(floatx4, ask4(a.l_scale, n, a.n));
    if (a.bias) bias = ask4(static_cast<const T*>(a.bias), n, a.n);
    if (a.residual) residual = ask4(static_cast<const T*>(a.residual) + m * a.ld_res, n, a.n);
  }
  __device__ inline void finish(const Product& a, int64_t m, int n, const i32x4& sum) const {
    floatx4 v = scaled(sum, rs, ls);
    if (a.bias) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += (float)bias[j];
    }
    activate<T>(a.act, v);
    if (a.residual) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += (float)residual[j];
    }
    store4(static_cast<T*>(a.out) + m * a.ld_out, n, a.n, v);
  }
};

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

// 16 MB rows and 16 NB columns a workgroup; eight waves take 128 bytes of k each in turn, four of their turns are on their way at once (4 x 4,096 x 4,096: 5.7
// us, 2.9 TB/s of weights with the launch, and 9.6 in tiles of 64 x 64 with 8 splits and their joining; 1,024 x 1,024 x 1,024: 7.9 and 8.3)
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
  constexpr int STEP = WAVES * kBK, MINE = (MB * NB + WAVES - 1) / WAVES;
  Ends<T> ends[MINE];                                         // of this wave's blocks of the joined sums
  auto place = [&](int i, int& m, int& n) {
    const int b = wave + i * WAVES;
    m = m0 + b % MB * 16 + i16;
    n = n0 + b / MB * 16 + 4 * g;
    return b < MB * NB && m < a.m && n < a.n;
  };
  auto ask = [&] {
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      int m, n;
      if (place(i, m, n)) ends[i].ask(a, m, n);
    }
  };
  constexpr bool EARLY = (MB + NB) * DEPTH < 24;              // (registers)
  if (EARLY) ask();
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
  if (!EARLY) ask();
#pragma unroll
  for (int x = 0; x < NB; ++x)
#pragma unroll
    for (int y = 0; y < MB; ++y) part[wave][x * MB + y][lane] = acc[x][y];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < MINE; ++i) {
    const int b = wave + i * WAVES;
    int m, n;
    if (!place(i, m, n)) continue;
    i32x4 sum = part[0][b][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += part[w][b][lane];
    ends[i].finish(a, m, n, sum);
  }
}

// ---- tiles through registers

// 64 x 64 outputs a workgroup, any alignment.  HALVES = 1: four waves, all of k, three tiles of 128 bytes of k on their way in registers while one is multiplied.  HALVES
// = 2, for few workgroups, where what a tile takes is a wait: eight waves, tiles of 256 bytes, either half of the waves takes one half and at the end finishes
// one half of the rows (1,531 x 777 x 1,027: 13.2 us, by four waves 14.9; 500 x 1,027 x 900 8.7 and 11.3; but 6,000 x 500 x 1,001 20.6 and 17.2).
template <class T, int HALVES>
__global__ __launch_bounds__(HALVES * 256, 4) void product_kernel(Product a) {
  using El = Elem<int8_t>;
  constexpr int BM = 64, BN = 64, BK = HALVES * kBK, THREADS = HALVES * 256, MB = 2, NB = 2, DEPTH = HALVES == 1 ? 3 : 1, S = lds_stride<int8_t>(BK);
  constexpr bool SPLITS = HALVES == 2;                        // (few tiles; more of them are enough without)
  __shared__ __attribute__((aligned(16))) int8_t ls[BN * S], rs[BM * S];
  const int wave = threadIdx.x >> 6, half = wave >> 2, wm = wave % 2 * MB * 16, wn = wave / 2 % 2 * NB * 16;
  const unsigned tm = (unsigned)(a.m + BM - 1) / BM, tn = (unsigned)(a.n + BN - 1) / BN;
  const int split = SPLITS ? (int)(blockIdx.x / (tm * tn)) : 0;
  int row, col;
  dense::tile_of(SPLITS ? blockIdx.x % (tm * tn) : blockIdx.x, tm, tn, row, col);
  const int m0 = row * BM, n0 = col * BN;
  const int kb = SPLITS ? split * a.k_per : 0, ke = SPLITS ? min(a.k, kb + a.k_per) : a.k;

  using MoveL = ProductMove<int8_t, BN, BK, THREADS, true>;
  using MoveR = ProductMove<int8_t, BM, BK, THREADS, true>;
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
  auto multiply = [&] {
#pragma unroll
    for (int i = 0; i < kBK; i += El::KF) {
      const int s = half * kBK + i;
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
  };
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (kb + d * BK < ke) fetch(d, kb + d * BK);
  for (int kt = kb; kt < ke; kt += DEPTH * BK) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int k = kt + d * BK;
      if (k >= ke) break;
      __syncthreads();
      ml.store(ls, rl[d]);
      mr.store(rs, rr[d]);
      __syncthreads();
      if (k + DEPTH * BK < ke) fetch(d, k + DEPTH * BK);
      multiply();
    }
  }
  const int lane = threadIdx.x & 63, m = m0 + wm + (lane & 15), n = n0 + wn + 4 * (lane >> 4);
  constexpr int ROWS = MB / HALVES;                           // blocks of sixteen rows that this wave finishes
  Ends<T> ends[ROWS][NB];
  auto line = [&](int y) { return m + (HALVES == 1 ? y : half) * 16; };
#pragma unroll
  for (int y = 0; y < ROWS; ++y)
#pragma unroll
    for (int x = 0; x < NB; ++x)
      if ((!SPLITS || a.splits == 1) && line(y) < a.m && n + x * 16 < a.n) ends[y][x].ask(a, line(y), n + x * 16);
  if constexpr (HALVES == 2) {
    __shared__ i32x4 part[8][NB][64];
#pragma unroll
    for (int x = 0; x < NB; ++x) part[wave][x][lane] = half ? acc[x][0] : acc[x][1];
    __syncthreads();
#pragma unroll
    for (int x = 0; x < NB; ++x) acc[x][0] = (half ? acc[x][1] : acc[x][0]) + part[wave ^ 4][x][lane];
  }
#pragma unroll
  for (int y = 0; y < ROWS; ++y) {
#pragma unroll
    for (int x = 0; x < NB; ++x) {
      if (line(y) >= a.m || n + x * 16 >= a.n) continue;
      if (SPLITS && a.splits > 1) store_sums(a.part + (split * (int64_t)a.m + line(y)) * a.n, n + x * 16, a.n, acc[x][y]);
      else ends[y][x].finish(a, line(y), n + x * 16, acc[x][y]);
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

// eight neighbouring outputs as they lie in memory
template <class T>
struct Eight {
  u32x4 p[sizeof(T) / 2];
  __device__ inline Eight() {}
  __device__ inline Eight(const floatx4& u, const floatx4& v) {
    if constexpr (sizeof(T) == 2) {
      typename Elem<T>::Frag f;
#pragma unroll
      for (int j = 0; j < 4; ++j) { f[j] = (T)u[j]; f[j + 4] = (T)v[j]; }
      p[0] = __builtin_bit_cast(u32x4, f);
    } else {
      p[0] = __builtin_bit_cast(u32x4, u);
      p[1] = __builtin_bit_cast(u32x4, v);
    }
  }
  __device__ inline void load(const T* from) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) p[i] = reinterpret_cast<const u32x4_any*>(from)[i];
  }
  __device__ inline void store(T* to) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<u32x4_any*>(to)[i] = p[i];
  }
  __device__ inline void add(floatx4& u, floatx4& v) const {
    if constexpr (sizeof(T) == 2) {
      const typename Elem<T>::Frag f = __builtin_bit_cast(typename Elem<T>::Frag, p[0]);
#pragma unroll
      for (int j = 0; j < 4; ++j) { u[j] += (float)f[j]; v[j] += (float)f[j + 4]; }
    } else {
      u += __builtin_bit_cast(floatx4, p[0]);
      v += __builtin_bit_cast(floatx4, p[1]);
    }
  }
};

// The epilogue of a wave's blocks from output (m0, n0), columns in pairs of blocks, for outputs of eight columns and more; of the eights that the output has
// in part nothing is stored.  What the columns' side takes is asked for once, and the residual of sixteen rows is on its way while the sixteen rows before are
// finished: a wait for a load is also one for the stores in front of it (eights that each waited for their own loads: 8,192 x 4,096 x 4,096 with gelu
// and residual 174, so 157; 16,384 x 1,024 x 1,024 47 and 37).  Rows and columns past the output's are computed from its last ones.
template <class T, int ACT, bool WHOLE, int NB, int MB>
__device__ __forceinline__ void finish_eights(const Product& a, int m0, int n0, i32x4 (&acc)[NB][MB]) {
  constexpr int XS = sizeof(T) == 4 && NB == 8 ? 1 : NB / 2;  // eights at a time (registers)
  const int lane = threadIdx.x & 63, m = m0 + (lane & 15), first = n0 + 8 * (lane >> 4);
#pragma unroll
  for (int x0 = 0; x0 < NB / 2; x0 += XS) {
    Eight<T> res[2][XS], bias[XS];
    floatx4 ls[XS][2];
    float rs[MB];
    auto column = [&](int x) { return WHOLE ? first + (x0 + x) * 32 : min(first + (x0 + x) * 32, a.n - 8); };
    auto row = [&](int y) { return (int64_t)(WHOLE ? m + y * 16 : min(m + y * 16, a.m - 1)); };
    auto ask = [&](int y) {
#pragma unroll
      for (int x = 0; x < XS; ++x) res[y & 1][x].load(static_cast<const T*>(a.residual) + row(y) * a.ld_res + column(x));
    };
    if (a.residual) ask(0);
#pragma unroll
    for (int x = 0; x < XS; ++x) {
#pragma unroll
      for (int h = 0; h < 2; ++h) ls[x][h] = __builtin_bit_cast(floatx4, *reinterpret_cast<const u32x4_any*>(a.l_scale + column(x) + h * 4));
      if (a.bias) bias[x].load(static_cast<const T*>(a.bias) + column(x));
    }
#pragma unroll
    for (int y = 0; y < MB; ++y) rs[y] = a.r_scale[row(y)];
#pragma unroll
    for (int y = 0; y < MB; ++y) {
      if (a.residual && y + 1 < MB) ask(y + 1);
#pragma unroll
      for (int x = 0; x < XS; ++x) {
        __builtin_amdgcn_sched_barrier(0);
        floatx4 u = scaled(acc[2 * (x0 + x)][y], rs[y], ls[x][0]), v = scaled(acc[2 * (x0 + x) + 1][y], rs[y], ls[x][1]);
        if (a.bias) bias[x].add(u, v);
        dense::activate<T, ACT>(u);
        dense::activate<T, ACT>(v);
        if (a.residual) res[y & 1][x].add(u, v);
        const int n = first + (x0 + x) * 32;
        if (WHOLE || (m + y * 16 < a.m && n + 8 <= a.n)) Eight<T>(u, v).store(static_cast<T*>(a.out) + (m + y * 16) * a.ld_out + n);
      }
    }
  }
}

// ... of the eight that the output has in part: the 1 .. 7 columns from `part` on, which lanes of one group hold in one pair of blocks.  All lanes load, from
// the output's last row where theirs is past it, so that nothing waits before everything is asked for (1,300 x 1,903 x 1,600: one after the other 24.6 us, so 22.8)
template <class T, int NB, int MB>
__device__ __forceinline__ void finish_part(const Product& a, int m0, int n0, i32x4 (&acc)[NB][MB], int part) {
  const int lane = threadIdx.x & 63, m = m0 + (lane & 15), count = a.n - part;
  i32x4 sums[2][MB];
#pragma unroll
  for (int x = 0; x < NB; x += 2) {
    if ((part - n0) / 32 != x / 2) continue;                  // (uniform)
#pragma unroll
    for (int y = 0; y < MB; ++y) {
      sums[0][y] = acc[x][y];
      sums[1][y] = acc[x + 1][y];
    }
  }
  float ls[7], rs[MB];
  T bias[7], res[MB][7];
#pragma unroll
  for (int j = 0; j < 7; ++j) {
    if (j >= count) continue;
    ls[j] = a.l_scale[part + j];
    if (a.bias) bias[j] = static_cast<const T*>(a.bias)[part + j];
  }
#pragma unroll
  for (int y = 0; y < MB; ++y) {
    const int64_t row = min(m + y * 16, a.m - 1);
    rs[y] = a.r_scale[row];
    if (!a.residual) continue;
#pragma unroll
    for (int j = 0; j < 7; ++j)
      if (j < count) res[y][j] = static_cast<const T*>(a.residual)[row * a.ld_res + part + j];
  }
  const bool mine = (part - n0) % 32 / 8 == lane >> 4;
#pragma unroll
  for (int y = 0; y < MB; ++y) {
    floatx4 v[2];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j / 4][j % 4] = j < 7 && j < count ? (float)sums[j / 4][y][j % 4] * rs[y] * ls[j < 7 ? j : 0] + (a.bias ? (float)bias[j < 7 ? j : 0] : 0.f) : 0.f;
    activate<T>(a.act, v[0]);
    activate<T>(a.act, v[1]);
    if (!mine || m + y * 16 >= a.m) continue;
    T* out = static_cast<T*>(a.out) + (m + y * 16) * a.ld_out + part;
#pragma unroll
    for (int j = 0; j < 7; ++j)
      if (j < count) out[j] = (T)(v[j / 4][j % 4] + (a.residual ? (float)res[y][j] : 0.f));
  }
}

// ... all of it (for outputs of eight columns and more), or with SPLITS a split's sums
template <class T, bool SPLITS, int NB, int MB>
__device__ __forceinline__ void finish_pairs(const Product& a, int split, int m0, int n0, i32x4 (&acc)[NB][MB]) {
  auto eights = [&](auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    switch (a.act) {
      case dense::ACT_RELU: finish_eights<T, dense::ACT_RELU, WHOLE>(a, m0, n0, acc); break;
      case dense::ACT_GELU: finish_eights<T, dense::ACT_GELU, WHOLE>(a, m0, n0, acc); break;
      case dense::ACT_SILU: finish_eights<T, dense::ACT_SILU, WHOLE>(a, m0, n0, acc); break;
      default: finish_eights<T, dense::ACT_NONE, WHOLE>(a, m0, n0, acc); break;
    }
  };
  if (m0 >= a.m || n0 >= a.n) return;
  if (SPLITS && a.splits > 1) {
    const int lane = threadIdx.x & 63, m = m0 + (lane & 15), n = n0 + 8 * (lane >> 4);
#pragma unroll
    for (int y = 0; y < MB; ++y)
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        const int c = n + x / 2 * 32 + x % 2 * 4;
        if (m + y * 16 < a.m && c < a.n) store_sums(a.part + (split * (int64_t)a.m + m + y * 16) * a.n, c, a.n, acc[x][y]);
      }
    return;
  }
  if (m0 + MB * 16 <= a.m && n0 + NB * 16 <= a.n) return eights(std::true_type());
  eights(std::false_type());
  const int part = a.n / 8 * 8;
  if (part < a.n && part < n0 + NB * 16) finish_part<T>(a, m0, n0, acc, part);
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
  finish_pairs<T, true>(a, split, m0 + wm, n0 + wn, acc);
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

// 256 x 256 outputs a workgroup of eight waves, four tiles of 64 bytes of k in LDS.  Two groups of four waves, one of each on every SIMD, half a step
// apart: while one group multiplies, the other reads its next fragments and asks for a tile three steps on, so that the matrix pipe has work all the
// time.
//  - A tile is read by either group after the barrier behind which both have waited for their own loads of it: the wait for tile t + 1 is in
//    front of the barrier that ends a group's reading of tile t.
//  - A buffer is written again (the loads of tile t + 3) after the barrier behind which both groups have their fragments of tile t - 1 in registers.
// Group 1 waits once more in front of the loop, group 0 behind it: both pass the same number of barriers.  k is whole tiles (a last tile that k may end in
// cost 6 us of 146 at 8,192 x 4,096 x 4,096).
template <class T>
__global__ __launch_bounds__(512) void turns_kernel(Product a) {
  constexpr int BM = 256, BN = 256, WM = 4, WN = 2, BUFS = 4, BK = 64, MB = BM / WM / 16, NB = BN / WN / 16, LT = BN * BK, TILE = (BM + BN) * BK, LOADS = TILE / 1024 / 8;
  __shared__ __attribute__((aligned(16))) int8_t lds[BUFS * TILE];        // the columns' tile | the rows' tile, BUFS times
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wm = wave % WM * MB * 16, wn = wave / WM * NB * 16;
  const unsigned tm = (unsigned)(a.m + BM - 1) / BM, tn = (unsigned)(a.n + BN - 1) / BN;
  int row, col;
  dense::tile_of(blockIdx.x, tm, tn, row, col);
  const int m0 = row * BM, n0 = col * BN, tiles = a.k / BK;
  DirectMove<BK, true, BN, 8, false> ml;
  DirectMove<BK, false, BM, 8, false> mr;
  static_assert(decltype(ml)::LOADS + decltype(mr)::LOADS == LOADS, "loads of a tile and wave");
  ml.start(a.l, a.ld_l, n0, a.n, 0, wave);
  mr.start(a.r, a.ld_r, m0, a.m, 0, wave);
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
  finish_pairs<T, false>(a, 0, m0 + wm, n0 + wn, acc);
}

// Sums of the splits and the epilogue, four outputs a thread
template <class T>
__global__ __launch_bounds__(256) void join_kernel(Product a) {
  const int per_row = (a.n + 3) / 4;
  const int64_t total = (int64_t)a.m * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / per_row;
    const int n = (int)(i - m * per_row) * 4;
    Ends<T> ends;
    ends.ask(a, m, n);
    i32x4 v = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) v += load_sums(a.part + ((int64_t)s * a.m + m) * a.n, n, a.n);
    ends.finish(a, m, n, v);
  }
}

// Operands whose rows no 16 bytes align, laid out again: rows of a.k bytes apart, zeros behind the row's own `k`.  A piece of 16 bytes a thread.
struct Unaligned { const int8_t* from; int8_t* to; int64_t ld; int rows; };
template <class T>
__global__ __launch_bounds__(256) void align_kernel(Unaligned x, Unaligned w, int k, int k_out) {
  const int pieces = k_out / 16;
  const int64_t total = ((int64_t)x.rows + w.rows) * pieces;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t line = i / pieces;
    const int at = (int)(i - line * pieces) * 16;
    const bool of_x = line < x.rows;
    const int64_t row = of_x ? line : line - x.rows;
    const int8_t* from = (of_x ? x.from + row * x.ld : w.from + row * w.ld) + at;
    u32x4 v = {0, 0, 0, 0};
    if (at < k) v = load16<T, kWide>(from, k - at);          // (k > 16)
    *reinterpret_cast<u32x4*>((of_x ? x.to : w.to) + row * k_out + at) = v;
  }
}

enum Kind { kFragments, kSmall, kSmall2, kDirect, kLarge };
struct Plan { Kind kind; int splits, k_per, mb, nb, aligned; };      // mb, nb: blocks of 16 rows and columns (fragments); aligned: bytes of k in operands that are laid out again

// Operands in whole pieces of 16 bytes, whose tiles' offsets are 32-bit numbers: by their sizes, and by where they lie too
inline bool whole_rows(const Linear8Args& f) {
  return f.d_in % 16 == 0 && f.ld_x % 16 == 0 && f.ld_w % 16 == 0 && f.ld_x < (1 << 23) && f.ld_w < (1 << 23);
}
inline bool whole_pieces(const Linear8Args& f) {
  return whole_rows(f) && reinterpret_cast<uintptr_t>(f.x) % 16 == 0 && reinterpret_cast<uintptr_t>(f.w) % 16 == 0;
}

// Which kernel, by the number of tiles and the length of their sums (each pair is the two sides of a rule, of one run):
//   fragments  the smallest tile that makes 256 workgroups at most (500 x 500 x 500: 32 x 32 3.9, 32 x 16 4.9, 32 x 64 4.4; 16 x 11,008 x 4,096: 32 x 64 12.9, 16 x 16 15.2) and
//              reads 400 KB of operands a workgroup at most (256 x 2,048 x 4,096, 393 KB: 14.4, in 128 x 128 15.9; 128 x 4,096 x 8,192, 786 KB: 24.7 and
//              19.8), with up to 16 rows 1 MB; rows that no 16 bytes align cost it three times that: 64 KB (100 x 1,000 x 999, 48 KB: 5.6, in 64 x 64 8.2;
//              1,000 x 257 x 1,999, 192 KB: 15.9 and 12.1)
//   256 x 256  whole tiles of 64 of k, long sums, more than 128 rows and columns, and tiles that fill the 256 CUs' rounds to nine tenths: 8,192 x 4,096 x 4,096 155, in 128 x 128
//              171; 2,048 x 8,192 x 4,096 80 and 90; but 5,000 x 4,096 x 4,096 (320 tiles) 120 and 108, 4,096 x 8,192 x 256 54.6 and 52.0, 65,000 x 128 x 1,024 30.7 and 26.3
//   128 x 128  from 64 rows and columns on: from 2^31 multiplications on (padded) where more than 512 tiles of 64 x 64 would be made, from 2^32 on with fewer: 8,192 x 512 x 512
//              10.0, in 64 x 64 12.8; 1,536 x 1,536 x 1,536 14.2 and 17.7; but 512 x 4,096 x 1,024 11.4 and 10.8; 50,000 x 48 x 1,024 17.4 and 15.9; from 1.5 x 2^32 on for columns that are
//              no eights (2,000 x 2,001 x 2,000 23.2 and 27.1; 1,300 x 1,903 x 1,600 22.8 and 19.1); k split to make a workgroup for every CU (200 x 4,096 x 4,096 in one 25.1, in
//              four 18.1)
//   64 x 64    everything smaller; by eight waves with up to 512 tiles, k split to make up to 512 workgroups of 512 bytes of k at least (64 x 8,192 x 8,191 in four 27.3,
//              in two 33.4, in eight 31.2; 1,000 x 257 x 1,999 in three 12.1, in one 15.6)
// Rows that 16 bytes do not align are laid out again where that makes one of the larger kernels possible, with 192 tiles of 128 x 128 and more and 128 rows and
// columns (8,192 x 4,096 x 4,095: 165, in 64 x 64 as they are 462; 4,000 x 1,000 x 1,001 18.5 and 21.0; 50,000 x 128 x 1,001 36 and 43; but 6,000 x 500 x 1,001, 188 tiles,
// 20.6 and 17.2; 100,000 x 64 x 4,095 279 and 156).
inline Plan plan_of(int64_t m, int64_t n, int64_t k, bool whole, bool align) {
  const auto tiles_of = [&](int64_t b) { return ((m + b - 1) / b) * ((n + b - 1) / b); };
  Plan p{kFragments, 1, (int)up(k, kBK), 0, 0, 0};
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
  if (!whole && align && k > 16 && middle >= 192 && m >= 128 && n >= 128) {
    Plan q = plan_of(m, n, up(k, 64), true, false);
    q.aligned = (int)up(k, 64);
    if (q.kind >= kDirect) return q;
  }
  const int64_t least = n % 8 ? 3 << 17 : small > 512 ? 1 << 17 : 1 << 18;
  if (whole && m > 128 && n > 128 && k % 64 == 0 && k >= 1024 && large * 10 >= rounds * 256 * 9) {
    p.kind = kLarge;
  } else if (whole && m >= 64 && n >= 64 && middle * k >= least) {
    p.kind = kDirect;
    split(middle, 256, 8);
  } else {
    p.kind = small > 512 ? kSmall : kSmall2;
    if (p.kind == kSmall2) split(small, 512, 4);
  }
  return p;
}

// Workspace: operands laid out again, then the sums of splits
inline size_t aligned_bytes(const Plan& p, int64_t m, int64_t n) { return (size_t)up((m + n) * p.aligned, 256); }
inline size_t part_bytes(const Linear8Args& f) {
  if (f.rows == 0) return 0;                                  // (a plan has a tile at least)
  const auto bytes = [&](const Plan& p) {
    return aligned_bytes(p, f.rows, f.d_out) + (p.splits > 1 ? (size_t)p.splits * f.rows * f.d_out * sizeof(int) : 0);
  };
  // (where the operands lie is not known when the workspace is asked for: enough for either)
  const bool whole = whole_rows(f);
  const size_t any = bytes(plan_of(f.rows, f.d_out, f.d_in, false, !whole)), best = whole ? bytes(plan_of(f.rows, f.d_out, f.d_in, true, false)) : 0;
  return any > best ? any : best;
}

template <class T>
hipError_t run(Product a, const Plan& p, void* ws, hipStream_t s) {
  a.splits = p.splits;
  a.k_per = p.k_per;
  a.part = reinterpret_cast<int*>(static_cast<char*>(ws) + aligned_bytes(p, a.m, a.n));
  const auto grid = [&](int64_t b) { return ((a.m + b - 1) / b) * ((a.n + b - 1) / b) * p.splits; };
  hipError_t e = hipErrorInvalidValue;
  if (p.aligned) {
    int8_t* to = static_cast<int8_t*>(ws);
    const Unaligned x{a.r, to, a.ld_r, a.m}, w{a.l, to + (int64_t)a.m * p.aligned, a.ld_l, a.n};
    const int64_t blocks = (((int64_t)a.m + a.n) * (p.aligned / 16) + 255) / 256;
    if ((e = launch(align_kernel<int8_t>, blocks < 8192 ? blocks : 8192, 256, s, x, w, a.k, p.aligned)) != hipSuccess) return e;
    a.r = x.to; a.l = w.to; a.ld_r = a.ld_l = a.k = p.aligned;
  }
  switch (p.kind) {
    case kFragments: {
      const int64_t n = ((a.m + 16 * p.mb - 1) / (16 * p.mb)) * (int64_t)((a.n + 16 * p.nb - 1) / (16 * p.nb));
      if (p.mb == 1) return launch(fragments_kernel<T, 1, 1>, n, 512, s, a);
      if (p.mb == 4) return launch(fragments_kernel<T, 4, 4>, n, 512, s, a);
      if (p.nb == 1) return launch(fragments_kernel<T, 2, 1>, n, 512, s, a);
      if (p.nb == 2) return launch(fragments_kernel<T, 2, 2>, n, 512, s, a);
      return launch(fragments_kernel<T, 2, 4>, n, 512, s, a);
    }
    case kSmall: return launch(product_kernel<T, 1>, grid(64), 256, s, a);
    case kSmall2: e = launch(product_kernel<T, 2>, grid(64), 512, s, a); break;
    case kDirect: e = launch(direct_kernel<T>, grid(128), 256, s, a); break;
    case kLarge: return launch(turns_kernel<T>, grid(256), 512, s, a);
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
  return run<T>(a, plan_of(a.m, a.n, a.k, whole_pieces(f), !whole_rows(f)), ws, s);
}

}  // namespace dense8
}  // namespace stgn
