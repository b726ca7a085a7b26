// The root-mean-square norm of rows with the residual's addition, its gradient, and rows or columns in 8 bits with scales.
//
//   h = x + residual,  r = 1 / sqrt(mean h^2 + eps),  y = h r g;       scale = max |y| / 127,  q = y 127 / max |y| to the nearest whole number
//   dx = r (g dy - h r mean(r g dy h)) + dh,                            dg = column sums of dy h r
//
// Bytes bound all of it: a row is read once and stays in its lanes' registers between its sums and its outputs.  LANES lanes hold a row, 8 to 32
// numbers each (by_width): 16 lanes (sixteen rows a workgroup, whose sums take four steps within a wave) to 1,024 (one row); longer rows are
// read again.
// The sum of squares is a sum of 64 bits: r, and with it a number in 8 bits whose value lies next to a border, then does not hang on the
// order of the sum, and no magnitude of 32 bits overflows it.
// Figures are of kernels launched one after the other from a program in C++, three sets of inputs and outputs in turn; where two are given for one size, both
// are of one run, and another run's or card's are up to a tenth off.  Through the binding, where a result takes the place of the one before it, the same kernels take less (the norm of
// 16,384 x 4,096 in bf16 44 us, 50 here).
#pragma once
#include <math.h>

#include "operators.h"
#include "tile_ops.h"

namespace stgn {
namespace norm {

template <class T> constexpr int kE = Elem<T>::E;

template <class T>
__device__ inline void unpack(const u32x4& r, float (&v)[kE<T>]) {
  const typename Elem<T>::Frag f = __builtin_bit_cast(typename Elem<T>::Frag, r);
#pragma unroll
  for (int j = 0; j < kE<T>; ++j) v[j] = (float)f[j];
}
template <class T>
__device__ inline void store_piece(T* row, int c, int width, const float (&v)[kE<T>]) {
  if constexpr (kE<T> == 4) store4(row, c, width, floatx4{v[0], v[1], v[2], v[3]});
  else store8(row, c, width, floatx4{v[0], v[1], v[2], v[3]}, floatx4{v[4], v[5], v[6], v[7]});
}
// a piece of a row, read so that no other lane's elements are touched (where a row may be written in place while others are still read)
template <class T>
__device__ inline u32x4 load_own(const T* row, int c, int width) {
  return c + kE<T> <= width ? load16<T, kWhole>(row + c, kE<T>) : load16<T, kShort>(row + c, width - c);
}

// The piece at column c as it is asked for, and as it is used: a row that ends with a part of a piece is read from its last 16 bytes, which are moved down when they
// are used (behind the load, the move would wait for it: 20,000 x 2,100 in bf16 181 us of gradient, 81 so)
template <class T>
__device__ inline u32x4 ask_piece(const T* row, int c, int width, RowEnd end) {
  if (c >= width) return u32x4{0, 0, 0, 0};
  if (end == kShort) return load16<T, kShort>(row + c, width - c);
  return *reinterpret_cast<const u32x4_any*>(row + c - max(c + kE<T> - width, 0));
}
template <class T>
__device__ inline u32x4 settle(const u32x4& v, int c, int width, RowEnd end) {
  const int early = c + kE<T> - width;
  if (end == kWide && early > 0 && early < kE<T>) return moved_down<T>(v, early * (int)sizeof(T));
  return v;
}

// the low bytes of four numbers
__device__ inline uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(b, a, 0x0C0C0400u) | __builtin_amdgcn_perm(d, c, 0x04000C0Cu);
}
// Whether none of the wave's lanes has piece i of its row (of 16 lanes a row, every wave has every piece)
template <int LANES, int E>
__device__ inline bool without(int i, int width) {
  if (LANES < 64) return false;
  const int first = LANES > 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x & (LANES - 1)) : 0;
  return (first + i * LANES) * E >= width;
}

template <int E>
__device__ inline void store_bytes(int8_t* row, int c, int width, const uint32_t (&q)[E]) {
  uint32_t w[E / 4];
#pragma unroll
  for (int i = 0; i < E / 4; ++i) w[i] = low_bytes(q[4 * i], q[4 * i + 1], q[4 * i + 2], q[4 * i + 3]);
  if (c + E <= width) {
    if constexpr (E == 4) *reinterpret_cast<u32_any*>(row + c) = w[0];
    else *reinterpret_cast<u32x2_any*>(row + c) = u32x2_any{w[0], w[1]};
  } else {
#pragma unroll
    for (int j = 0; j < E - 1; ++j)
      if (c + j < width) row[c + j] = (int8_t)q[j];
  }
}

// y 127 / top to the nearest whole number, halves to the even one; up = 127 / top in 64 bits.  The product is off by 2^-45 at most.  A quotient of
// numbers of 24 bits that is no half is 2^-34 or more away from one, so rounding it to multiples of 2^-40 first makes halves exact and
// moves nothing across one: q is the definition's number for every y and top.
// The number is the low byte.  up = 0 in rows with an infinity or a NaN: all their numbers are 0, a NaN's low byte being 0 too (fp32 has 23 bits of its payload,
// the high ones in fp64).
__device__ inline uint32_t to_eight(float y, double up) {
  constexpr double kSnap = 6144.0, kWhole52 = 6755399441055744.0;        // 1.5 x 2^12, 1.5 x 2^52
  const double t = ((double)y * up + kSnap) - kSnap;
  return (uint32_t)__builtin_bit_cast(uint64_t, t + kWhole52);
}
// of the bits of a row's largest magnitude; a row with an infinity or a NaN has scale NaN and zeros, so that what is computed from it shows them
__device__ inline float scale_of(uint32_t top) { return top >= 0x7F800000u ? __builtin_nanf("") : (float)((double)__builtin_bit_cast(float, top) / 127.0); }
__device__ inline double up_of(uint32_t top) {
  return top == 0u || top >= 0x7F800000u ? 0.0 : 127.0 / (double)__builtin_bit_cast(float, top);
}
__device__ inline uint32_t magnitude(float y) { return __builtin_bit_cast(uint32_t, y) & 0x7FFFFFFFu; }

__device__ inline float inverse_root(double sum, int width, double eps) {
  const double r = 1.0 / sqrt(sum / width + eps);
  return r > 3.4028234663852886e38 ? 3.4028234663852886e38f : (float)r;          // (rows of zeros with eps = 0 stay zeros)
}

// h r g in fp32.  (fp16: left to itself, the compiler takes the last product and the rounding to fp16 as one where nothing else needs the fp32 value, and y
// would have other bits beside 8-bit outputs than without them.)
template <class T>
__device__ inline float normed(float h, float r, float g) {
  float y = h * r * g;
  if constexpr (std::is_same<T, _Float16>::value) asm("" : "+v"(y));
  return y;
}

// every lane's value from N lanes further on within its sixteen, round about
template <int N, class V>
__device__ inline V rotated(V v) {
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x120 + N, 0xF, 0xF, true));
  } else {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    i32x2 w = __builtin_bit_cast(i32x2, v);
    w[0] = __builtin_amdgcn_mov_dpp(w[0], 0x120 + N, 0xF, 0xF, true);
    w[1] = __builtin_amdgcn_mov_dpp(w[1], 0x120 + N, 0xF, 0xF, true);
    return __builtin_bit_cast(V, w);
  }
}
// Value of all LANES lanes that hold a row, the same bits in each; `at`: LDS for rows that lie in several waves, which nobody else uses between one barrier of
// the workgroup and the next
template <int LANES, class V, class F>
__device__ inline V across(V v, V* at, F f) {
  v = f(v, rotated<8>(v));
  v = f(v, rotated<4>(v));
  v = f(v, rotated<2>(v));
  v = f(v, rotated<1>(v));
  if constexpr (LANES >= 64) {
    v = f(v, (V)__shfl_xor(v, 16));
    v = f(v, (V)__shfl_xor(v, 32));
  }
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    v = at[0];
#pragma unroll
    for (int w = 1; w < LANES / 64; ++w) v = f(v, at[w]);
  }
  return v;
}
template <int LANES>
__device__ inline double sum_across(double v, double* at) { return across<LANES>(v, at, [](double a, double b) { return a + b; }); }
template <int LANES>
__device__ inline uint32_t top_across(uint32_t v, uint32_t* at) { return across<LANES>(v, at, [](uint32_t a, uint32_t b) { return a > b ? a : b; }); }

constexpr int block_of(int lanes) { return lanes < 256 ? 256 : lanes; }

enum Kind { kNorm, kNorm8, kRows8 };                          // y; 8 bits of y (and y); 8 bits of x

// Rows whose pieces stay in registers.  All of a row is read before any of it is written: outputs may lie where the inputs do.  A workgroup walks down the rows: the
// gain is read once, and the next row is on its way while one is summed and written (bf16, a workgroup for every row or four and so: 30,000 x 1,027 56 us and 34,
// 30,000 x 2,000 57 and 47, 16,384 x 4,096 in 8 bits 63 and 48, the norm alone 50 and 50).
template <class T, int LANES, int NP, Kind KIND>
__global__ __launch_bounds__(block_of(LANES), LANES == 512 ? 4 : 1) void rows_kernel(NormArgs a) {
  constexpr int E = kE<T>, PER = block_of(LANES) / LANES;
  __shared__ double sums[LANES > 64 ? LANES / 64 : 1];
  __shared__ uint32_t tops[LANES > 64 ? LANES / 64 : 1];
  const int lane = (int)threadIdx.x % LANES;
  const RowEnd end = row_end<T>(a.width);
  constexpr bool AHEAD = LANES < 1024 || NP * E <= 16;        // (32 numbers a lane of 1,024 leave no registers for another row)
  u32x4 rx[NP], rr[NP], rg[NP];
  auto ask = [&](int64_t row) {
    const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
    const T* res = a.residual ? static_cast<const T*>(a.residual) + row * a.ld_res : nullptr;
#pragma unroll
    for (int i = 0; i < NP; ++i) rx[i] = ask_piece(x, (lane + i * LANES) * E, a.width, end);
    if (res) {
#pragma unroll
      for (int i = 0; i < NP; ++i) rr[i] = ask_piece(res, (lane + i * LANES) * E, a.width, end);
    }
  };
  const int64_t step = (int64_t)gridDim.x * PER;
  int64_t row = (int64_t)blockIdx.x * PER + (int)threadIdx.x / LANES;
  if (AHEAD && row < a.rows) ask(row);
  if constexpr (KIND != kRows8) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (lane + i * LANES) * E;
      rg[i] = c < a.width ? load_own(static_cast<const T*>(a.gain), c, a.width) : u32x4{0, 0, 0, 0};
    }
  }
  for (; row < a.rows; row += step) {
    if (!AHEAD) ask(row);
    float v[NP][E];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (lane + i * LANES) * E;
      unpack<T>(settle<T>(rx[i], c, a.width, end), v[i]);
      if (a.residual) {
        float u[E];
        unpack<T>(settle<T>(rr[i], c, a.width, end), u);
#pragma unroll
        for (int j = 0; j < E; ++j) v[i][j] += u[j];
      }
    }
    if (AHEAD && row + step < a.rows) ask(row + step);
    if constexpr (KIND != kRows8) {
      double sum = 0.0;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        if (without<LANES, E>(i, a.width)) continue;
#pragma unroll
        for (int j = 0; j < E; ++j) sum = fma((double)v[i][j], (double)v[i][j], sum);
      }
      const float r = inverse_root(sum_across<LANES>(sum, sums), a.width, a.eps);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = (lane + i * LANES) * E;
        if (c >= a.width) continue;
        if (a.h) store_piece(static_cast<T*>(a.h) + row * a.ld_h, c, a.width, v[i]);
        float g[E];
        unpack<T>(rg[i], g);
#pragma unroll
        for (int j = 0; j < E; ++j) v[i][j] = normed<T>(v[i][j], r, g[j]);
        if (KIND == kNorm || a.y) store_piece(static_cast<T*>(a.y) + row * a.ld_y, c, a.width, v[i]);
      }
    }
    if constexpr (KIND != kNorm) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) top = max(top, magnitude(v[i][j]));          // (past the row: zeros)
      top = top_across<LANES>(top, tops);
      const double up = up_of(top);
      if (lane == 0) a.scale[row] = scale_of(top);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = (lane + i * LANES) * E;
        if (c >= a.width) continue;
        uint32_t q[E];
#pragma unroll
        for (int j = 0; j < E; ++j) q[j] = to_eight(v[i][j], up);
        store_bytes<E>(a.q + row * a.ld_q, c, a.width, q);
      }
    }
    if constexpr (LANES > 64) __syncthreads();                // (the sums' LDS, where the workgroup has another row)
  }
}

// Rows longer than 1,024 lanes hold: read once a sum and once for the outputs.  A workgroup a row: as many rows as there are CUs keep the card busy, fewer do not (bf16, 64 rows of 2^20
// numbers 210 us, one 158).
template <class T, Kind KIND>
__global__ __launch_bounds__(1024) void long_rows_kernel(NormArgs a) {
  constexpr int E = kE<T>, LANES = 1024;
  __shared__ double sums[LANES / 64];
  __shared__ uint32_t tops[LANES / 64];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
    const T* res = a.residual ? static_cast<const T*>(a.residual) + row * a.ld_res : nullptr;
    auto each = [&](auto f) {
      for (int c = (int)threadIdx.x * E; c < a.width; c += LANES * E) {
        float v[E], u[E];
        unpack<T>(load_own(x, c, a.width), v);
        if (res) {
          unpack<T>(load_own(res, c, a.width), u);
#pragma unroll
          for (int j = 0; j < E; ++j) v[j] += u[j];
        }
        f(c, v);
      }
    };
    float r = 1.f;
    if constexpr (KIND != kRows8) {
      double sum = 0.0;
      each([&](int, float (&v)[E]) {
#pragma unroll
        for (int j = 0; j < E; ++j) sum = fma((double)v[j], (double)v[j], sum);
      });
      r = inverse_root(sum_across<LANES>(sum, sums), a.width, a.eps);
    }
    auto norm = [&](int c, float (&v)[E]) {
      if constexpr (KIND != kRows8) {
        float g[E];
        unpack<T>(load_own(static_cast<const T*>(a.gain), c, a.width), g);
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = normed<T>(v[j], r, g[j]);
      }
    };
    uint32_t top = 0;
    if constexpr (KIND != kNorm) {
      each([&](int c, float (&v)[E]) {
        norm(c, v);
#pragma unroll
        for (int j = 0; j < E; ++j) top = max(top, c + j < a.width ? magnitude(v[j]) : 0u);
      });
      top = top_across<LANES>(top, tops);
      if (threadIdx.x == 0) a.scale[row] = scale_of(top);
    }
    const double up = up_of(top);
    each([&](int c, float (&v)[E]) {
      if (a.h) store_piece(static_cast<T*>(a.h) + row * a.ld_h, c, a.width, v);
      norm(c, v);
      if (KIND != kRows8 && (KIND == kNorm || a.y)) store_piece(static_cast<T*>(a.y) + row * a.ld_y, c, a.width, v);
      if constexpr (KIND != kNorm) {
        uint32_t q[E];
#pragma unroll
        for (int j = 0; j < E; ++j) q[j] = to_eight(v[j], up);
        store_bytes<E>(a.q + row * a.ld_q, c, a.width, q);
      }
    });
    __syncthreads();
  }
}

constexpr int64_t kMostBlocks = 1 << 20;                      // of a launch; more rows go round again

// f(lanes, pieces) for the fewest lanes that hold a row with 16 numbers each, or longer() where none do.  A SIMD has four waves of such norms (three in fp32) and three of
// their gradients (two in fp32).  32 numbers a lane for the widest rows, some of whose kernels spill (up to 24 registers), and for 16-bit rows of 1,025 to
// 2,048: two waves a SIMD, but a row is one wave's and no sum goes through LDS (30,000 x 1,027 34 us, by 256 lanes of 8 numbers 40 with their best number of workgroups;
// in 8 bits 41 and 50, its gradient 62 and 77; 30,000 x 2,000 47 and 49, 47 and 56, 79 and 84).  GRAD: 512 lanes at most there, whose registers hold what the gradient
// keeps of 32 numbers (1,024 lanes of 16, half the registers each, spill: 4,096 x 16,384 in bf16 192 us, 118 so).
template <class T, bool GRAD, class F, class L>
hipError_t by_width(int width, F f, L longer) {
#define STGN_HOLDS(lanes, numbers) \
  if (width <= lanes * numbers) return f(std::integral_constant<int, lanes>(), std::integral_constant<int, numbers / kE<T>>());
  STGN_HOLDS(16, 8)
  STGN_HOLDS(16, 16)
  STGN_HOLDS(64, 8)
  STGN_HOLDS(64, 16)
  if constexpr (kE<T> == 8) {
    STGN_HOLDS(64, 32)
  } else {
    STGN_HOLDS(256, 8)
  }
  STGN_HOLDS(256, 16)
  STGN_HOLDS(512, 16)
  if constexpr (GRAD) {
    STGN_HOLDS(512, 32)
  } else {
    STGN_HOLDS(1024, 16)
    if constexpr (kE<T> == 8) {
      STGN_HOLDS(1024, 32)
    }
  }
#undef STGN_HOLDS
  return longer();
}

inline int64_t blocks_for(int64_t rows, int lanes) {
  const int per = block_of(lanes) / lanes;
  const int64_t n = (rows + per - 1) / per;
  return n < kMostBlocks ? n : kMostBlocks;
}

template <class T, Kind KIND>
hipError_t rows_of(const NormArgs& a, hipStream_t s) {
  return by_width<T, false>(
      a.width,
      [&](auto lanes, auto pieces) {
        constexpr int L = decltype(lanes)::value, N = decltype(pieces)::value;
        int64_t blocks = blocks_for(a.rows, L);
        // 1,024 workgroups walk down the rows, 512 of 512 lanes, 256 of 1,024: as many as the CUs hold at once of kernels with four waves a SIMD, of which some have more and some
        // fewer (bf16, us with half as many, these, half as many again: 16,384 x 4,096 48, 50, 52, in 8 bits 64, 48, 49; 30,000 x 1,027 31, 34, 35, in 8 bits 40, 41, 43; 200,000 x 64 22, 18, 17).  With a
        // residual, whose four streams keep memory busy anyhow, a workgroup a row (16,384 x 4,096 91 us, 100 walking, 30,000 x 2,000 85 and 95; but 30,000 x 1,027, whose rows
        // no 16 bytes align, 70 and 57).
        const int64_t most = L <= 256 ? 1024 : L == 512 ? 512 : 256;
        if (!(KIND == kNorm && a.residual) && blocks > most) blocks = most;
        return launch(rows_kernel<T, L, N, KIND>, blocks, block_of(L), s, a);
      },
      [&]() { return launch(long_rows_kernel<T, KIND>, a.rows < kMostBlocks ? a.rows : kMostBlocks, 1024, s, a); });
}

// ---- gradient

// r, and r mean(g dy h): dx = r (g dy - (h r) back), whose factors neither overflow nor vanish where h is large or small
struct Back { float r, back; };
__device__ inline Back back_of(double squares, double dots, int width, double eps) {
  Back b;
  b.r = inverse_root(squares, width, eps);
  b.back = (float)((double)b.r * (dots / width));
  return b;
}

// A workgroup walks down the rows and keeps the gain's gradient of its rows in registers: one partial sum a column and workgroup.  These sums are of 32 bits, as 64 would take
// 16 to 32 registers more, and the parts are added up in 64: in fp32 dgain of 40,000 x 200 is 1.1e-7 off in the norm and 0.7e-7 where all of a column is added in 64 bits, of
// 1,000,000 x 200 2.1e-7 and 0.6e-7; in 16 bits the result's own rounding hides it.
template <class T, int LANES, int NP>
__global__ __launch_bounds__(block_of(LANES)) void grad_kernel(NormGradArgs a, float* part) {
  constexpr int E = kE<T>, PER = block_of(LANES) / LANES;
  __shared__ double sums[2][LANES > 64 ? LANES / 64 : 1];
  __shared__ float fold[PER > 1 ? PER : 1][PER > 1 ? LANES * NP * E : 1];
  const int lane = (int)threadIdx.x % LANES;
  const RowEnd end = row_end<T>(a.width);
  float acc[NP][E];
  u32x4 rg[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (lane + i * LANES) * E;
    rg[i] = c < a.width ? load_own(static_cast<const T*>(a.gain), c, a.width) : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < E; ++j) acc[i][j] = 0.f;
  }
  constexpr bool AHEAD = NP < 8;                              // (32 numbers of fp32 a lane leave no registers for another row)
  u32x4 rh[NP], ry[NP], rd[NP], next_h[NP], next_y[NP];
  auto ask = [&](u32x4(&to)[NP], const void* matrix, int64_t ld, int64_t row) {
    const T* p = static_cast<const T*>(matrix) + row * ld;
#pragma unroll
    for (int i = 0; i < NP; ++i) to[i] = ask_piece(p, (lane + i * LANES) * E, a.width, end);
  };
#pragma unroll
  for (int i = 0; i < NP; ++i) rd[i] = u32x4{0, 0, 0, 0};
  const int64_t step = (int64_t)gridDim.x * PER;
  int64_t row = (int64_t)blockIdx.x * PER + (int)threadIdx.x / LANES;
  if (AHEAD && row < a.rows) {
    ask(next_h, a.h, a.ld_h, row);
    ask(next_y, a.dy, a.ld_dy, row);
  }
  for (; row < a.rows; row += step) {
    if (!AHEAD) {
      ask(next_h, a.h, a.ld_h, row);
      ask(next_y, a.dy, a.ld_dy, row);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (lane + i * LANES) * E;
      rh[i] = settle<T>(next_h[i], c, a.width, end);
      ry[i] = settle<T>(next_y[i], c, a.width, end);
    }
    if (a.dh) ask(rd, a.dh, a.ld_dh, row);
    if (AHEAD && row + step < a.rows) {
      ask(next_h, a.h, a.ld_h, row + step);
      ask(next_y, a.dy, a.ld_dy, row + step);
    }
    double squares = 0.0, dots = 0.0;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (without<LANES, E>(i, a.width)) continue;
      float hv[E], yv[E], gv[E];
      unpack<T>(rh[i], hv);
      unpack<T>(ry[i], yv);
      unpack<T>(rg[i], gv);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        squares = fma((double)hv[j], (double)hv[j], squares);
        dots = fma((double)(yv[j] * gv[j]), (double)hv[j], dots);
      }
    }
    squares = sum_across<LANES>(squares, sums[0]);
    dots = sum_across<LANES>(dots, sums[1]);
    const Back b = back_of(squares, dots, a.width, a.eps);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (lane + i * LANES) * E;
      if (without<LANES, E>(i, a.width)) continue;
      float hv[E], yv[E], gv[E], dv[E];
      unpack<T>(rh[i], hv);
      unpack<T>(ry[i], yv);
      unpack<T>(rg[i], gv);
      unpack<T>(settle<T>(rd[i], c, a.width, end), dv);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const float unit = hv[j] * b.r;
        acc[i][j] = fmaf(yv[j], unit, acc[i][j]);
        dv[j] = fmaf(b.r, fmaf(-unit, b.back, yv[j] * gv[j]), dv[j]);
      }
      if (a.dx && c < a.width) store_piece(static_cast<T*>(a.dx) + row * a.ld_dx, c, a.width, dv);
    }
    if constexpr (LANES > 64) __syncthreads();
  }
  if (!a.dgain) return;
  if constexpr (PER > 1) {
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int j = 0; j < E; ++j) fold[threadIdx.x / LANES][(lane + i * LANES) * E + j] = acc[i][j];
    __syncthreads();
    for (int c = (int)threadIdx.x; c < a.width; c += (int)blockDim.x) {
      float v = fold[0][c];
#pragma unroll
      for (int p = 1; p < PER; ++p) v += fold[p][c];
      if (gridDim.x > 1) part[(int64_t)blockIdx.x * a.width + c] = v;
      else static_cast<T*>(a.dgain)[c] = (T)v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (lane + i * LANES) * E;
      if (c >= a.width) continue;
      if (gridDim.x > 1) {
#pragma unroll
        for (int j = 0; j < E; j += 4)
          if (c + j < a.width) store4(part + (int64_t)blockIdx.x * a.width, c + j, a.width, floatx4{acc[i][j], acc[i][j + 1], acc[i][j + 2], acc[i][j + 3]});
      } else {
        store_piece(static_cast<T*>(a.dgain), c, a.width, acc[i]);
      }
    }
  }
}

// Rows longer than the lanes hold: dx, and r of every row for the gain's gradient behind it
template <class T>
__global__ __launch_bounds__(1024) void long_grad_kernel(NormGradArgs a, float* r) {
  constexpr int E = kE<T>, LANES = 1024;
  __shared__ double sums[2][LANES / 64];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* h = static_cast<const T*>(a.h) + row * a.ld_h;
    const T* dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
    const T* dh = a.dh ? static_cast<const T*>(a.dh) + row * a.ld_dh : nullptr;
    auto each = [&](auto f) {
      for (int c = (int)threadIdx.x * E; c < a.width; c += LANES * E) {
        float hv[E], t[E], g[E];
        unpack<T>(load_own(h, c, a.width), hv);
        unpack<T>(load_own(dy, c, a.width), t);
        unpack<T>(load_own(static_cast<const T*>(a.gain), c, a.width), g);
#pragma unroll
        for (int j = 0; j < E; ++j) t[j] *= g[j];
        f(c, hv, t);
      }
    };
    double squares = 0.0, dots = 0.0;
    each([&](int, float (&hv)[E], float (&t)[E]) {
#pragma unroll
      for (int j = 0; j < E; ++j) {
        squares = fma((double)hv[j], (double)hv[j], squares);
        dots = fma((double)t[j], (double)hv[j], dots);
      }
    });
    squares = sum_across<LANES>(squares, sums[0]);
    dots = sum_across<LANES>(dots, sums[1]);
    const Back b = back_of(squares, dots, a.width, a.eps);
    if (a.dgain && threadIdx.x == 0) r[row] = b.r;
    __syncthreads();                                          // (the sums' LDS)
    if (!a.dx) continue;
    each([&](int c, float (&hv)[E], float (&t)[E]) {
      float dv[E];
      unpack<T>(dh ? load_own(dh, c, a.width) : u32x4{0, 0, 0, 0}, dv);
#pragma unroll
      for (int j = 0; j < E; ++j) dv[j] = fmaf(b.r, fmaf(-hv[j] * b.r, b.back, t[j]), dv[j]);
      store_piece(static_cast<T*>(a.dx) + row * a.ld_dx, c, a.width, dv);
    });
  }
}
// ... the sums of 256 columns over a chunk of rows.  h r first, whose magnitude is the root of the width at most: dy h may be past what 32 bits hold where dy h r is not
template <class T>
__global__ __launch_bounds__(256) void long_gain_kernel(NormGradArgs a, const float* r, float* part, int rows_per) {
  __shared__ floatx4 wsum[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int cols = (a.width + 255) / 256, n = (int)(blockIdx.x % cols) * 256 + lane * 4;
  const int64_t chunk = blockIdx.x / cols, m1 = min((int64_t)a.rows, (chunk + 1) * rows_per);
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  if (n < a.width) {
#pragma unroll 4
    for (int64_t m = chunk * rows_per + wave; m < m1; m += 4)
      acc += load4(static_cast<const T*>(a.dy) + m * a.ld_dy, n, a.width) * (load4(static_cast<const T*>(a.h) + m * a.ld_h, n, a.width) * r[m]);
  }
  wsum[wave][lane] = acc;
  __syncthreads();
  if (wave == 0 && n < a.width)
    store4(part + chunk * a.width, n, a.width, (wsum[0][lane] + wsum[1][lane]) + (wsum[2][lane] + wsum[3][lane]));
}

// The partial sums of sixteen columns a workgroup, in their order but for 64 runs that are added at the end (in 64 bits: as many as the partial sums are, their
// order then costs no bit)
template <class T>
__global__ __launch_bounds__(1024) void gain_kernel(const float* part, int parts, int width, T* dgain) {
  __shared__ double wsum[16][16];
  const int column = threadIdx.x & 15, c = (int)blockIdx.x * 16 + column;
  double acc = 0.0;
  if (c < width) {
#pragma unroll 8
    for (int i = (int)threadIdx.x >> 4; i < parts; i += 64) acc += (double)part[(int64_t)i * width + c];
  }
  acc += __shfl_xor(acc, 16);
  acc += __shfl_xor(acc, 32);
  if ((threadIdx.x & 63) < 16) wsum[threadIdx.x >> 6][column] = acc;
  __syncthreads();
  if (threadIdx.x < 16 && c < width) {
    acc = wsum[0][column];
#pragma unroll
    for (int w = 1; w < 16; ++w) acc += wsum[w][column];
    dgain[c] = (T)(float)acc;
  }
}

inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// parts: partial sums a column; of long rows: chunks of rows, and r of every row in front of the sums
struct GradPlan { int64_t blocks; int parts, rows_per; size_t sums, total; bool is_long; };
template <class T>
GradPlan grad_plan(const NormGradArgs& a) {
  GradPlan p{};
  by_width<T, true>(
      a.width,
      [&](auto lanes, auto pieces) {
        constexpr int L = decltype(lanes)::value;
        p.blocks = blocks_for(a.rows, L);
        // As many workgroups as the CUs hold at once, each of which has its partial sums (16 numbers a lane in fp32, 32, rows of 16 lanes and full ones of 256: two a CU;
        // us, bf16: 51,480 x 777 with 512 workgroups 79, 768 71, 1,024 92; 78,125 x 512 73, 64, 66; 9,765 x 4,096 66, 68, 79)
        constexpr int NUMBERS = decltype(pieces)::value * kE<T>;
        const bool two = NUMBERS > 16 || (NUMBERS == 16 && (sizeof(T) == 4 || L == 16 || (L == 256 && a.width * 4 >= L * NUMBERS * 3)));
        const int64_t most = L > 256 ? 256 : two ? 512 : NUMBERS == 16 ? 768 : 1024;
        if (a.dgain && p.blocks > most) p.blocks = most;
        p.parts = (int)p.blocks;
        return hipSuccess;
      },
      [&]() {
        p.is_long = true;
        p.blocks = a.rows < kMostBlocks ? a.rows : kMostBlocks;
        const int64_t chunks = a.rows < 64 ? 1 : a.rows < 64 * 64 ? a.rows / 64 : 64;
        p.rows_per = (int)((a.rows + chunks - 1) / chunks);
        if (p.rows_per < 1) p.rows_per = 1;
        p.parts = (int)((a.rows + p.rows_per - 1) / p.rows_per);
        return hipSuccess;
      });
  if (a.dgain) {
    p.sums = p.is_long ? (size_t)up((int64_t)a.rows * sizeof(float), 256) : 0;
    p.total = p.sums + (p.parts > 1 || p.is_long ? (size_t)p.parts * a.width * sizeof(float) : 0);
  }
  return p;
}

template <class T>
hipError_t backward(const NormGradArgs& a, void* ws, hipStream_t s) {
  const GradPlan p = grad_plan<T>(a);
  float* part = ws ? reinterpret_cast<float*>(static_cast<char*>(ws) + p.sums) : nullptr;
  hipError_t e = hipSuccess;
  if (p.blocks > 0)
    e = by_width<T, true>(
        a.width,
        [&](auto lanes, auto pieces) {
          constexpr int L = decltype(lanes)::value, N = decltype(pieces)::value;
          return launch(grad_kernel<T, L, N>, p.blocks, block_of(L), s, a, part);
        },
        [&]() {
          hipError_t f = launch(long_grad_kernel<T>, p.blocks, 1024, s, a, static_cast<float*>(ws));
          if (f == hipSuccess && a.dgain)
            f = launch(long_gain_kernel<T>, (int64_t)p.parts * ((a.width + 255) / 256), 256, s, a, (const float*)ws, part, p.rows_per);
          return f;
        });
  if (e == hipSuccess && a.dgain && (p.parts != 1 || p.is_long))
    e = launch(gain_kernel<T>, (a.width + 15) / 16, 1024, s, (const float*)part, p.parts, a.width, static_cast<T*>(a.dgain));
  return e;
}

// ---- columns in 8 bits: largest magnitudes of a piece's columns a lane over chunks of rows, then tiles turned over through LDS

template <class T>
__global__ __launch_bounds__(1024) void column_tops_kernel(ColumnsArgs a, uint32_t* tops, int rows_per) {
  constexpr int E = kE<T>, WIDE = 64 * E;                     // columns a workgroup, a piece a lane
  __shared__ uint32_t wtop[16][WIDE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int cols = (a.width + WIDE - 1) / WIDE, n0 = (int)(blockIdx.x % cols) * WIDE, n = n0 + lane * E;
  const int64_t chunk = blockIdx.x / cols, m1 = min((int64_t)a.rows, (chunk + 1) * rows_per);
  uint32_t top[E];
#pragma unroll
  for (int j = 0; j < E; ++j) top[j] = 0;
  if (n < a.width) {
#pragma unroll 8
    for (int64_t m = chunk * rows_per + wave; m < m1; m += 16) {
      float v[E];
      unpack<T>(load_own(static_cast<const T*>(a.x) + m * a.ld_x, n, a.width), v);
#pragma unroll
      for (int j = 0; j < E; ++j) top[j] = max(top[j], magnitude(v[j]));
    }
  }
#pragma unroll
  for (int j = 0; j < E; ++j) wtop[wave][lane * E + j] = top[j];
  __syncthreads();
  const int c = (int)threadIdx.x;
  if (c < WIDE && n0 + c < a.width) {
    uint32_t t = wtop[0][c];
#pragma unroll
    for (int w = 1; w < 16; ++w) t = max(t, wtop[w][c]);
    tops[chunk * a.width + n0 + c] = t;
  }
}

constexpr int kTileRows = 128, kTileCols = 64;

// 16 bytes of a column, those of them that it has
__device__ inline void store_line(int8_t* to, const int8_t* from, int left) {
  if (left >= 16) {
    *reinterpret_cast<u32x4_any*>(to) = *reinterpret_cast<const u32x4*>(from);
  } else {
    for (int j = 0; j < left; ++j) to[j] = from[j];
  }
}

template <class T>
__global__ __launch_bounds__(256) void columns_kernel(ColumnsArgs a, const uint32_t* tops, int chunks) {
  constexpr int E = kE<T>, STRIDE = kTileRows + 16, ACROSS = kTileCols / E, ITEMS = kTileRows / 4 * ACROSS / 256;
  __shared__ uint32_t part[4][kTileCols], top[kTileCols];
  __shared__ __attribute__((aligned(16))) int8_t tile[kTileCols * STRIDE];
  const int tiles_n = (a.width + kTileCols - 1) / kTileCols;
  const int n0 = (int)(blockIdx.x % tiles_n) * kTileCols;
  const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * kTileRows;
  u32x4 raw[ITEMS][4];                                        // four rows of a piece; on their way while the columns' maxima are found
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int at = i * 256 + (int)threadIdx.x, c = n0 + at % ACROSS * E;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t m = m0 + at / ACROSS * 4 + u;
      raw[i][u] = m < a.rows && c < a.width ? load_own(static_cast<const T*>(a.x) + m * a.ld_x, c, a.width) : u32x4{0, 0, 0, 0};
    }
  }
  {
    const int c = threadIdx.x & 63, from = threadIdx.x >> 6;
    uint32_t t = 0;
    if (n0 + c < a.width) {
#pragma unroll 8
      for (int i = from; i < chunks; i += 4) t = max(t, tops[(int64_t)i * a.width + n0 + c]);
    }
    part[from][c] = t;
    __syncthreads();
    if (from == 0) {
      t = max(max(part[0][c], part[1][c]), max(part[2][c], part[3][c]));
      top[c] = t;
      if (m0 == 0 && n0 + c < a.width) a.scale[n0 + c] = scale_of(t);
    }
    __syncthreads();
  }
  // a word of four rows' bytes in each of the piece's columns
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int at = i * 256 + (int)threadIdx.x, piece = at % ACROSS, quad = at / ACROSS;
    float v[4][E];
#pragma unroll
    for (int u = 0; u < 4; ++u) unpack<T>(raw[i][u], v[u]);
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const double by = up_of(top[piece * E + j]);
      *reinterpret_cast<uint32_t*>(tile + (piece * E + j) * STRIDE + quad * 4) =
          low_bytes(to_eight(v[0][j], by), to_eight(v[1][j], by), to_eight(v[2][j], by), to_eight(v[3][j], by));
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kTileCols * (kTileRows / 16); i += 256) {
    const int c = i / (kTileRows / 16), at = i % (kTileRows / 16) * 16;
    if (n0 + c >= a.width || m0 + at >= a.rows) continue;
    store_line(a.q + (int64_t)(n0 + c) * a.ld_q + m0 + at, tile + c * STRIDE + at, (int)(a.rows - m0 - at));
  }
}

// Up to 1,024 rows: a workgroup has its 64 columns whole, in registers, and one launch without a workspace does both (bf16, 256 x 1,024: 5.0 us, two launches 6.8; 1,024 x
// 8,192 10.8 and 12.3; 1,000 x 1,000 9.2 and 8.7, and the host's share is half)
constexpr int kOneRows = 1024;

template <class T>
__global__ __launch_bounds__(1024) void whole_columns_kernel(ColumnsArgs a) {
  constexpr int E = kE<T>, STRIDE = kOneRows + 16, ACROSS = kTileCols / E, ITEMS = kOneRows / 4 * ACROSS / 1024;
  __shared__ uint32_t top[kTileCols];
  __shared__ __attribute__((aligned(16))) int8_t tile[kTileCols * STRIDE];
  const int n0 = (int)blockIdx.x * kTileCols, piece = (int)threadIdx.x % ACROSS, c = n0 + piece * E;
  if (threadIdx.x < kTileCols) top[threadIdx.x] = 0;
  auto row_of = [&](int i) { return (i * 1024 + (int)threadIdx.x) / ACROSS * 4; };
  u32x4 raw[ITEMS][4];
  uint32_t mine[E];
#pragma unroll
  for (int j = 0; j < E; ++j) mine[j] = 0;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int m = row_of(i) + u;
      raw[i][u] = m < a.rows && c < a.width ? load_own(static_cast<const T*>(a.x) + m * a.ld_x, c, a.width) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float v[E];
      unpack<T>(raw[i][u], v);
#pragma unroll
      for (int j = 0; j < E; ++j) mine[j] = max(mine[j], magnitude(v[j]));
    }
#pragma unroll
  for (int j = 0; j < E; ++j)
#pragma unroll
    for (int d = ACROSS; d < 64; d *= 2) mine[j] = max(mine[j], (uint32_t)__shfl_xor((int)mine[j], d));
  __syncthreads();
  if ((threadIdx.x & 63) < ACROSS) {
#pragma unroll
    for (int j = 0; j < E; ++j) atomicMax(&top[piece * E + j], mine[j]);
  }
  __syncthreads();
  if (threadIdx.x < kTileCols && n0 + (int)threadIdx.x < a.width) a.scale[n0 + threadIdx.x] = scale_of(top[threadIdx.x]);
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    if (row_of(i) >= a.rows) continue;
    float v[4][E];
#pragma unroll
    for (int u = 0; u < 4; ++u) unpack<T>(raw[i][u], v[u]);
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const double by = up_of(top[piece * E + j]);
      *reinterpret_cast<uint32_t*>(tile + (piece * E + j) * STRIDE + row_of(i)) =
          low_bytes(to_eight(v[0][j], by), to_eight(v[1][j], by), to_eight(v[2][j], by), to_eight(v[3][j], by));
    }
  }
  __syncthreads();
  const int along = (a.rows + 15) / 16;
  for (int i = (int)threadIdx.x; i < kTileCols * along; i += 1024) {
    const int line = i / along, at = i % along * 16;
    if (n0 + line >= a.width) continue;
    store_line(a.q + (int64_t)(n0 + line) * a.ld_q + at, tile + line * STRIDE + at, a.rows - at);
  }
}

template <class T>
inline int column_chunks(int64_t rows, int64_t width) {       // of 128 rows and more, a workgroup for every CU
  const int64_t cols = (width + 64 * kE<T> - 1) / (64 * kE<T>), want = (256 + cols - 1) / cols, most = (rows + 127) / 128;
  return (int)(want < most ? want : most);
}
template <class T>
size_t columns_bytes(const ColumnsArgs& a) { return a.rows <= kOneRows ? 0 : (size_t)column_chunks<T>(a.rows, a.width) * a.width * sizeof(uint32_t); }

template <class T>
hipError_t columns(const ColumnsArgs& a, void* ws, hipStream_t s) {
  if (a.rows <= kOneRows) return launch(whole_columns_kernel<T>, (a.width + kTileCols - 1) / kTileCols, 1024, s, a);   // (no rows: the scales)
  const int chunks = column_chunks<T>(a.rows, a.width);
  const int rows_per = (a.rows + chunks - 1) / chunks;
  uint32_t* tops = static_cast<uint32_t*>(ws);
  hipError_t e = launch(column_tops_kernel<T>, (int64_t)chunks * ((a.width + 64 * kE<T> - 1) / (64 * kE<T>)), 1024, s, a, tops, rows_per);
  if (e != hipSuccess) return e;
  const int64_t down = (a.rows + kTileRows - 1) / kTileRows;
  return launch(columns_kernel<T>, down * ((a.width + kTileCols - 1) / kTileCols), 256, s, a, (const uint32_t*)tops, chunks);
}

}  // namespace norm
}  // namespace stgn
