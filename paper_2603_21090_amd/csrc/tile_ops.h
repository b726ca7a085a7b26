// Tiles of 16 x 16 products for operators on the caller's tensors, in three element types: fp32 (products in fp32), bf16 and
// fp16 (products in 16 bits); every sum is fp32.
//
// One FRAGMENT is 16 bytes per lane, four floats or eight 16-bit numbers: a 16-row operand with KF elements of the summed
// index (16 or 32).  Lane l serves row l % 16; lane group l / 16 owns E = 4 or 8 of the KF elements, and which ones does not
// matter as long as both operands agree.  Two orders are used:
//   straight  group g holds elements E g + j.  A row-major row in LDS gives it by one 16-byte read.
//   split     16-bit only: group g holds 4 g + j (j < 4) and 16 + 4 g + (j - 4).  That is how two accumulator blocks lie in
//             registers (row 4 g + r, column l % 16), so probabilities go from one product into the next without LDS.
//             With floats one accumulator block is a fragment in the straight order.
// An operand whose summed index runs down the rows of its LDS tile (V in P V) is read by the transposing LDS load of four
// 16-bit numbers, or by four 4-byte reads of floats.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace stgn {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
// rows of odd widths start anywhere, those of 8-bit numbers at any byte: global memory takes wide accesses at any address
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32_any __attribute__((aligned(1), may_alias));

template <class T> struct Elem;

template <> struct Elem<float> {
  using Frag = floatx4;
  using Four = floatx4;
  static constexpr int E = 4, KF = 16, PB = 1;               // elements a lane, elements of the summed index, accumulator blocks a fragment
  static __device__ inline floatx4 mma(const Frag& a, const Frag& b, floatx4 c) {
#pragma unroll
    for (int u = 0; u < 4; ++u) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[u], b[u], c, 0, 0, 0);
    return c;
  }
};

template <> struct Elem<__bf16> {
  using Frag = bf16x8;
  using Four = bf16x4;
  static constexpr int E = 8, KF = 32, PB = 2;
  static __device__ inline floatx4 mma(const Frag& a, const Frag& b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};

template <> struct Elem<_Float16> {
  using Frag = f16x8;
  using Four = f16x4;
  static constexpr int E = 8, KF = 32, PB = 2;
  static __device__ inline floatx4 mma(const Frag& a, const Frag& b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};

template <> struct Elem<int8_t> {                             // sums of 32-bit integers
  using Frag = i32x4;
  static constexpr int E = 16, KF = 64;
  static __device__ inline i32x4 mma(const Frag& a, const Frag& b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
  }
};

// PB accumulator blocks as one fragment, rounded to T: the factors of the next product, half a step each, as any 16-bit operand.  In the norm,
// against 64 bits, beside the results' own rounding: causal attention of lists of 2,049 to 4,096 in bf16 is 0.0020 off (0.0016 with 32-bit factors),
// its gradient 0.0024 (0.0017), in fp16 with a window 0.00030 (0.00021).  Factors kept as two 16-bit halves would take these products twice.
template <class T>
__device__ inline typename Elem<T>::Frag pack(const floatx4 (&blocks)[Elem<T>::PB]) {
  if constexpr (Elem<T>::PB == 1) {
    return blocks[0];
  } else {
    typename Elem<T>::Frag f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (T)blocks[j / 4][j % 4];
    return f;
  }
}

// LDS rows of `width` elements are 16 bytes longer: 16 rows of a fragment then start in 16 different groups of four banks
template <class T>
__host__ __device__ constexpr int lds_stride(int width) { return width + Elem<T>::E; }

// fragment of rows row .. row + 15, elements k .. k + KF - 1 of a row-major tile (straight order)
template <class T>
__device__ inline typename Elem<T>::Frag frag_rows(const T* tile, int stride, int row, int k) {
  const int lane = threadIdx.x & 63;
  return *reinterpret_cast<const typename Elem<T>::Frag*>(tile + (row + (lane & 15)) * stride + k + Elem<T>::E * (lane >> 4));
}

// The transposing LDS load: the sixteen lanes of a group read four rows of 16 numbers, 8 bytes each (lane i: row i / 4, numbers
// 4 (i % 4) and on), and lane i gets the four numbers of column i.
template <class T>
__device__ inline i16x4 read_transposed(const T* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p));
}
template <class T>
__device__ inline typename Elem<T>::Frag join_transposed(const i16x4& lo, const i16x4& hi) {
  typedef short i16x8 __attribute__((ext_vector_type(8)));
  const i16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(typename Elem<T>::Frag, both);
}

// fragment of columns col .. col + 15 whose summed index runs down rows row .. row + KF - 1 of the tile
template <class T, bool SPLIT>
__device__ inline typename Elem<T>::Frag frag_cols(const T* tile, int stride, int row, int col) {
  const int lane = threadIdx.x & 63, g = lane >> 4;
  if constexpr (sizeof(T) == 4) {
    floatx4 f;
#pragma unroll
    for (int u = 0; u < 4; ++u) f[u] = tile[(row + 4 * g + u) * stride + col + (lane & 15)];
    return f;
  } else {
    const int i = lane & 15;
    const T* p = tile + (row + (SPLIT ? 4 * g : 8 * g) + (i >> 2)) * stride + col + 4 * (i & 3);
    return join_transposed<T>(read_transposed(p), read_transposed(p + (SPLIT ? 16 : 4) * stride));
  }
}

// Where a row of a 16-bit tile lies that is read both ways (fragments along its rows, and down them in the split order).  LDS gives 256
// bytes a cycle: sixteen rows of 16 bytes, or eight rows of 32 bytes of a transposed read.  With rows 16 bytes longer than a multiple of 128,
// any order of sixteen rows serves the first; for the second, rows 0 .. 7 and 8 .. 15 lie two places apart.  (Rows in their own order: 40 % of
// the attention kernels' LDS cycles were conflicts.  Pieces permuted within a row instead of padding: no conflicts, but an address
// register per fragment.)  fp32 tiles are read down their rows four rows of 64 bytes a cycle: in their own order.
template <class T>
__device__ inline int placed(int row) {
  if constexpr (sizeof(T) == 4) return row;
  else return (row & ~15) | ((row & 7) << 1) | ((row >> 3) & 1);
}
template <class T, int COLS>
__device__ inline typename Elem<T>::Frag placed_rows(const T* tile, int row, int k) {        // row: a multiple of 16
  constexpr int S = lds_stride<T>(COLS);
  const int lane = threadIdx.x & 63;
  return *reinterpret_cast<const typename Elem<T>::Frag*>(tile + (row + placed<T>(lane & 15)) * S + k + Elem<T>::E * (lane >> 4));
}
template <class T, int COLS>
__device__ inline typename Elem<T>::Frag placed_cols(const T* tile, int row, int col) {      // the split order
  constexpr int S = lds_stride<T>(COLS);
  const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
  if constexpr (sizeof(T) == 4) {
    return frag_cols<T, true>(tile, S, row, col);
  } else {
    const T* p = tile + (row + placed<T>(4 * g + (i >> 2))) * S + col + 4 * (i & 3);
    return join_transposed<T>(read_transposed(p), read_transposed(p + 16 * S));
  }
}

// How the rows that a kernel reads in pieces of 16 bytes end: with a whole piece; with a part of one (WIDE: the row's last 16 bytes are
// read instead and moved down, one load without a branch); or the row is shorter than a piece and its elements are read one by one.
// Tiles on their way into LDS are moved down when they are stored: done behind the load, it waits for it (causal attention of 4 x 2,048, 8
// heads of 100, bf16: 146 us, 85 so; its gradient 311, 224).
enum RowEnd { kWhole, kWide, kShort };
template <class T>
__device__ inline RowEnd row_end(int width) { return width % Elem<T>::E == 0 ? kWhole : width > Elem<T>::E ? kWide : kShort; }

// v's last bytes, `bytes` of them dropped at the front, zeros behind
template <class T>
__device__ inline u32x4 moved_down(u32x4 v, int bytes) {
  v = bytes & 8 ? u32x4{v[2], v[3], 0u, 0u} : v;
  v = bytes & 4 ? u32x4{v[1], v[2], v[3], 0u} : v;
  if constexpr (sizeof(T) <= 2)
    v = bytes & 2 ? u32x4{__builtin_amdgcn_alignbyte(v[1], v[0], 2), __builtin_amdgcn_alignbyte(v[2], v[1], 2),
                          __builtin_amdgcn_alignbyte(v[3], v[2], 2), v[3] >> 16} : v;
  if constexpr (sizeof(T) == 1)
    v = bytes & 1 ? u32x4{__builtin_amdgcn_alignbyte(v[1], v[0], 1), __builtin_amdgcn_alignbyte(v[2], v[1], 1),
                          __builtin_amdgcn_alignbyte(v[3], v[2], 1), v[3] >> 8} : v;
  return v;
}

// 16 bytes at p of which `count` elements (one at least) are the row's last ones, or all; the rest zeros
template <class T, RowEnd END>
__device__ inline u32x4 load16(const T* p, int count) {
  constexpr int E = Elem<T>::E;
  if constexpr (END == kWhole) return *reinterpret_cast<const u32x4_any*>(p);
  if constexpr (END == kWide) {
    const int missing = count < E ? E - count : 0;
    return moved_down<T>(*reinterpret_cast<const u32x4_any*>(p - missing), missing * (int)sizeof(T));
  }
  union { T e[E]; u32x4 v; } u;
  u.v = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < E; ++j)
    if (j < count) u.e[j] = p[j];
  return u.v;
}
// ... the same for a row of any width
template <class T>
__device__ inline u32x4 load16(const T* p, int count, RowEnd end) {
  return end == kWhole ? load16<T, kWhole>(p, count) : end == kWide ? load16<T, kWide>(p, count) : load16<T, kShort>(p, count);
}
// f(std::integral_constant<RowEnd, end>): a copy of f's loads per kind, none with another kind's branches between them
template <class F>
__device__ inline void by_end(RowEnd end, F f) {
  if (end == kWhole) f(std::integral_constant<RowEnd, kWhole>());
  else if (end == kWide) f(std::integral_constant<RowEnd, kWide>());
  else f(std::integral_constant<RowEnd, kShort>());
}

// four sums as elements col .. col + 3 of a row of `cols` elements
template <class T>
__device__ inline void store4(T* row, int col, int cols, const floatx4& v) {
  typename Elem<T>::Four f;
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] = (T)v[j];
  if (col + 4 <= cols) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<u32x4_any*>(row + col) = __builtin_bit_cast(u32x4_any, f);
    else *reinterpret_cast<u32x2_any*>(row + col) = __builtin_bit_cast(u32x2_any, f);
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (col + j < cols) row[col + j] = f[j];
  }
}

template <class T>
__device__ inline floatx4 load4(const T* row, int col, int cols) {
  floatx4 v = {0.f, 0.f, 0.f, 0.f};
  if (col + 4 <= cols) {
    typename Elem<T>::Four f;
    if constexpr (sizeof(T) == 4) f = __builtin_bit_cast(typename Elem<T>::Four, *reinterpret_cast<const u32x4_any*>(row + col));
    else f = __builtin_bit_cast(typename Elem<T>::Four, *reinterpret_cast<const u32x2_any*>(row + col));
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = (float)f[j];
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (col + j < cols) v[j] = (float)row[col + j];
  }
  return v;
}

// eight neighbouring elements of 16-bit types: 16 bytes a lane
template <class T>
__device__ inline void add8(const T* row, int col, int cols, floatx4& u, floatx4& v) {
  if (col + 8 <= cols) {
    const typename Elem<T>::Frag f = __builtin_bit_cast(typename Elem<T>::Frag, *reinterpret_cast<const u32x4_any*>(row + col));
#pragma unroll
    for (int j = 0; j < 4; ++j) { u[j] += (float)f[j]; v[j] += (float)f[j + 4]; }
  } else {
    u += load4(row, col, cols);
    if (col + 4 < cols) v += load4(row, col + 4, cols);
  }
}
template <class T>
__device__ inline void store8(T* row, int col, int cols, const floatx4& u, const floatx4& v) {
  if (col + 8 <= cols) {
    typename Elem<T>::Frag f;
#pragma unroll
    for (int j = 0; j < 4; ++j) { f[j] = (T)u[j]; f[j + 4] = (T)v[j]; }
    *reinterpret_cast<u32x4_any*>(row + col) = __builtin_bit_cast(u32x4_any, f);
  } else {
    store4(row, col, cols, u);
    if (col + 4 < cols) store4(row, col + 4, cols, v);
  }
}

// An operand of a product on its way from global memory through registers into LDS, tile after tile along the summed index k: LINES of
// the output's rows or columns, BK elements of k.  ALONG: k runs along the matrix's rows, a tile is [LINES][BK]; else it has a row per k, a tile is
// [BK][LINES].  Every thread carries NP pieces of 16 bytes.  Lines and elements that the matrix does not have are zeros: what lies there
// is never read.
template <class T, int LINES, int BK, int THREADS, bool ALONG>
struct ProductMove {
  static constexpr int E = Elem<T>::E, ROWS = ALONG ? LINES : BK, PER_ROW = (ALONG ? BK : LINES) / E, PIECES = ROWS * PER_ROW;
  static constexpr int NP = (PIECES + THREADS - 1) / THREADS;
  static constexpr bool STEADY = THREADS % PER_ROW == 0;      // a thread's pieces lie below each other
  static constexpr int STRIDE = lds_stride<T>(ALONG ? BK : LINES);
  const T* base;                                              // the tile's first element
  int64_t ld;
  int lines, end;                                             // lines from the tile's first on; k that the sum ends in front of
  RowEnd row;
  static __device__ inline int row_of(int i) { return STEADY ? (int)threadIdx.x / PER_ROW + i * (THREADS / PER_ROW) : ((int)threadIdx.x + i * THREADS) / PER_ROW; }
  static __device__ inline int col_of(int i) { return (STEADY ? (int)threadIdx.x : (int)threadIdx.x + i * THREADS) % PER_ROW * E; }

  __device__ inline void start(const void* matrix, int64_t ld_, int first, int total_lines, int k, int end_, int total_k) {
    base = static_cast<const T*>(matrix) + (ALONG ? (int64_t)first * ld_ + k : (int64_t)k * ld_ + first);
    ld = ld_;
    lines = total_lines - first;
    end = end_;
    row = row_end<T>(ALONG ? total_k : total_lines);
  }
  // whether a row per k ends here with a part of a piece, and the elements in front of that part that the piece at column c holds then
  __device__ inline bool cut() const { return !ALONG && row == kWide && lines < LINES; }
  __device__ inline int early(int c) const { return min(max(E - (lines - c), 0), E); }

  // the tile at k, which is the next one
  __device__ inline void fetch(u32x4 (&r)[NP], int k) {
    const int rows = ALONG ? lines : end - k, cols = ALONG ? end - k : lines;
    auto each = [&](auto load) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int x = row_of(i), c = col_of(i);
        r[i] = u32x4{0, 0, 0, 0};
        if ((PIECES % THREADS == 0 || x < ROWS) && x < rows && c < cols) r[i] = load(base + (int64_t)x * ld + c, cols - c);
      }
    };
    if (cols >= (ALONG ? BK : LINES)) each([](const T* p, int) { return *reinterpret_cast<const u32x4_any*>(p); });
    else if (cut()) each([](const T* p, int count) { return *reinterpret_cast<const u32x4_any*>(p - max(E - count, 0)); });
    else by_end(row, [&](auto e) { each([](const T* p, int count) { return load16<T, decltype(e)::value>(p, count); }); });
    base += ALONG ? BK : BK * ld;
  }
  __device__ inline void store(T* tile, const u32x4 (&r)[NP]) const {
    auto each = [&](auto piece) {
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (PIECES % THREADS == 0 || row_of(i) < ROWS) *reinterpret_cast<u32x4*>(tile + row_of(i) * STRIDE + col_of(i)) = piece(r[i], col_of(i));
    };
    if (cut()) each([&](u32x4 v, int c) { return moved_down<T>(v, early(c) * (int)sizeof(T)); });
    else each([](u32x4 v, int) { return v; });
  }
};

// ROWS x COLS elements of a matrix on their way into LDS, tile after tile down its rows: addresses are computed once and advance by a tile.
template <class T, int ROWS, int COLS, int THREADS>
struct StreamMove {
  static constexpr int E = Elem<T>::E, PER_ROW = COLS / E, NP = ROWS * PER_ROW / THREADS, APART = THREADS / PER_ROW;
  static_assert(ROWS * PER_ROW % THREADS == 0 && THREADS % PER_ROW == 0, "every thread carries whole pieces of one column");
  const T* at;                                                // this thread's first piece of the next tile
  int64_t apart, step;                                        // elements from one of its pieces to the next, from tile to tile
  int row, count;                                             // its row in the tile; elements the matrix has from its column on
  u32x4 r[NP];

  static __device__ inline int early(int count) { return max(E - count, 0); }      // elements in front of a row's last part that its piece holds
  // first: the address of this thread's row threadIdx.x / PER_ROW of the first tile
  __device__ inline void start(const T* first, int64_t apart_, int64_t step_, int cols) {
    const int c = (int)threadIdx.x % PER_ROW * E;
    row = (int)threadIdx.x / PER_ROW;
    count = cols - c;
    at = first + c - (row_end<T>(cols) == kWide && count > 0 ? early(count) : 0);
    apart = apart_;
    step = step_;
  }
  __device__ inline void start_rows(const T* base, int64_t stride, int cols) {
    start(base + (int64_t)((int)threadIdx.x / PER_ROW) * stride, APART * stride, ROWS * stride, cols);
  }
  // rows: how many the matrix has from the tile's first row on (the same for all threads)
  __device__ inline void fetch(int rows, RowEnd end) {
    auto each = [&](auto load) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        r[i] = u32x4{0, 0, 0, 0};
        if (count > 0 && (rows >= ROWS || row + i * APART < rows)) r[i] = load(at + i * apart);
      }
    };
    if (end != kShort) each([](const T* p) { return *reinterpret_cast<const u32x4_any*>(p); });
    else each([&](const T* p) { return load16<T, kShort>(p, count); });
    at += step;
  }
  // count_: the elements that the matrix has from this thread's column on
  __device__ inline void store(T* tile, RowEnd end, int count_) const {
    auto each = [&](auto piece) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int x = (int)threadIdx.x / PER_ROW + i * APART;
        *reinterpret_cast<u32x4*>(tile + placed<T>(x) * lds_stride<T>(COLS) + (int)threadIdx.x % PER_ROW * E) = piece(r[i]);
      }
    };
    if (end == kWide) each([&](u32x4 v) { return moved_down<T>(v, min(early(count_), E) * (int)sizeof(T)); });
    else each([](u32x4 v) { return v; });
  }
  __device__ inline void store(T* tile, RowEnd end) const { store(tile, end, count); }
};

}  // namespace stgn
