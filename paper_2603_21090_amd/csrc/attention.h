// Softmax attention of lists of queries over lists of keys, and its gradients, on gfx950's matrix cores.
//
//   s_ij = scale q_i . k_j over the keys that i sees,  lse_i = log sum_j exp s_ij,  o_i = sum_j exp(s_ij - lse_i) v_j
//   p_ij = exp(s_ij - lse_i),  dv_j = sum_i p_ij do_i,  ds_ij = p_ij (do_i . v_j - do_i . o_i),
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i
//
// What a query sees: keys j < k_lens of its list; with `causal` the lists are aligned at their ends (query i stands at
// k_len - q_len + i and sees keys up to there), with `window` only the last `window` of those.
//
// Rows.  The `group` query heads that share a key head are one matrix: row r = i * group + (head in the group).  A key tile is
// loaded once for all of them, and the sums over shared heads in dk and dv need no step of their own.
//
// Every kernel has the same shape: a wave keeps NB blocks of 16 columns (queries, or keys in the dk/dv kernel) in registers as
// the right operand, the other side streams through LDS as the left one, and all results are transposed (accumulator
// column = the wave's own row).  A softmax maximum, a sum, an lse then belong to a lane, rescaling needs no exchange, and the
// probabilities are the next product's right operand as they lie in registers.
#pragma once
#include <math.h>

#include <type_traits>

#include "operators.h"
#include "tile_ops.h"

namespace stgn {
namespace attn {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Softmax weights as fp16 factors are taken 2^14 times: a weight of a long list is a small number, and below 2^-14 fp16 has
// fewer bits (5,000 keys: dv 0.5 % off).  None exceeds 1, so none overflows.
template <class T> constexpr float kShift = std::is_same<T, _Float16>::value ? 14.f : 0.f;
template <class T> constexpr float kUnshift = kShift<T> != 0.f ? 1.f / 16384.f : 1.f;

// In the forward call the reference score may lag the largest one by kLazy powers of two (see there): 2^7 times there.
template <class T> constexpr float kShiftLazy = kShift<T> / 2.f;
constexpr float kLazy = 8.f;

__device__ inline float over_groups_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float over_groups_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// ds has no such bound: beside dout of a mean over many rows it falls below fp16's numbers (4,000 keys, dout of 2^-14: its terms lose all bits), and
// beside large dout and values it passes 65,504.  As an fp16 factor it is taken a power of two times that belongs to the column of the
// accumulators (a row of dq, a key of dk): 2^64 times at first, and where a factor would pass 2^15 only so often that the largest lies above 2^8,
// the sums so far being taken along.  What is 2^-22 of the column's largest keeps all bits, and no term is off by more than 2^-33 of that one.
// (3 lists of up to 1,777, window 512, 6 heads of 80 on 2: dq, dk and dv 82.1 -> 85.3 us.)
template <class T> constexpr bool kFitted = std::is_same<T, _Float16>::value;
__device__ inline float exponent_of(float power_of_two) { return (float)((int)(__builtin_bit_cast(uint32_t, power_of_two) >> 23) - 127); }
template <int NB>
struct Fit {
  float times[NB];
  __device__ inline Fit() {
#pragma unroll
    for (int c = 0; c < NB; ++c) times[c] = 0x1p64f;
  }
  // 1 / times: both are powers of two
  __device__ inline float undo(int c) const { return __builtin_bit_cast(float, 0x7F000000u - __builtin_bit_cast(uint32_t, times[c])); }
  // top: the largest |ds| that this lane adds to column c next, as often as they are taken; sums(c, by): the column's factors and sums are to be
  // taken `by` times
  template <class F>
  __device__ inline void take(const float (&top)[NB], F sums) {
    bool grows = false;
#pragma unroll
    for (int c = 0; c < NB; ++c) grows |= top[c] > 0x1p15f;
    if (!__any(grows)) return;
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const float most = over_groups_max(top[c]);             // of the four lane groups that share the column
      if (!(most > 0x1p15f)) continue;
      const uint32_t power = __builtin_bit_cast(uint32_t, most) >> 23;               // most lies in 2^(power - 127) and twice that
      const float by = __builtin_bit_cast(float, (262u - power) << 23);
      times[c] *= by;
      sums(c, by);
    }
  }
};

// rows of a streamed tile: two buffers of two tiles of 64 x 128 16-bit numbers are 68 KB, two workgroups a CU
template <class T, int DP>
constexpr int stream_rows() {
  constexpr int n = 64 * 256 / (DP * (int)sizeof(T));
  return n > 64 ? 64 : n;
}

struct List {                                                 // one list: lengths and where its queries stand
  int qn, kn, shift;                                          // query i stands at key i + shift
};

__device__ inline List list_of(const AttnArgs& a, int b) {
  List l;
  l.qn = a.q_lens ? min(max(a.q_lens[b], 0), a.q_len) : a.q_len;
  l.kn = a.k_lens ? min(max(a.k_lens[b], 0), a.k_len) : a.k_len;
  l.shift = l.kn - l.qn;
  return l;
}

// keys [lo, hi) that query i sees
__device__ inline void seen(const AttnArgs& a, const List& l, int i, int& lo, int& hi) {
  lo = 0;
  hi = l.kn;
  if (a.causal) {
    hi = min(hi, i + l.shift + 1);
    if (a.window) lo = max(0, i + l.shift - a.window + 1);
  }
  if (i >= l.qn) hi = 0;
}

__device__ inline int query_of(const AttnArgs& a, int r) { return a.group == 1 ? r : (int)((unsigned)r / (unsigned)a.group); }

template <class T>
__device__ inline const T* row_of(const void* base, const Strides& s, int b, int row, int head) {
  return static_cast<const T*>(base) + (int64_t)b * s.list + (int64_t)row * s.row + (int64_t)head * s.head;
}

template <class T>
__device__ inline T* dense_row(const AttnArgs& a, void* base, int len, int heads, int b, int row, int head) {
  return static_cast<T*>(base) + (((int64_t)b * len + row) * heads + head) * a.d;
}

// NB blocks of 16 rows of the right operand: row(c) is the address of this lane's row in block c, or null
template <class T, int DP, int NB, class Row>
__device__ inline void load_cols(typename Elem<T>::Frag (&f)[NB][DP / Elem<T>::KF], Row row, int d, uint32_t flip = 0) {
  constexpr int KF = Elem<T>::KF, E = Elem<T>::E;
  const int g = (threadIdx.x & 63) >> 4;
  by_end(row_end<T>(d), [&](auto e) {
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const T* p = row(c);
#pragma unroll
      for (int k = 0; k < DP / KF; ++k) {
        const int at = k * KF + E * g;
        u32x4 v = {0, 0, 0, 0};
        if (p != nullptr && at < d) v = load16<T, decltype(e)::value>(p + at, d - at);
        if (flip) v ^= flip;
        f[c][k] = __builtin_bit_cast(typename Elem<T>::Frag, v);
      }
    }
  });
}

// what fits a CU at once: two workgroups, or one of eight waves whose rows are 128 numbers
template <int WAVES, int DP> constexpr bool kTwo = WAVES * DP <= 512;

// Workgroup -> (tile of a list and key head, run of the tile's stream, list, key head).  The longest tiles come first (with `causal` the
// last queries, or the first keys); where all workgroups are on the chip at once, two a CU, the second half comes in the
// other order instead, so that a long and a short one share a CU.  The same tile of all lists and heads lies side by side: workgroups that
// read the same keys are a multiple of their number apart, on one die where that is a multiple of eight.
struct Place { int tile, run, b, hk; };
__device__ inline Place place_of(const AttnArgs& a, int tiles, int runs, bool two, bool last_first) {
  const unsigned pairs = (unsigned)a.lists * (unsigned)a.kv_heads, bh = blockIdx.x % pairs, x = blockIdx.x / pairs;
  Place p;
  p.b = (int)(bh / (unsigned)a.kv_heads);
  p.hk = (int)(bh % (unsigned)a.kv_heads);
  p.run = (int)(x % (unsigned)runs);
  const int q = (int)(x / (unsigned)runs), half = (tiles + 1) / 2;
  const int nth = two && gridDim.x <= 512u && q >= half ? tiles - 1 - (q - half) : q;      // nth longest
  p.tile = last_first ? tiles - 1 - nth : nth;
  return p;
}

// A workgroup's run of the `n` streamed rows from `first` on, whole tiles of `tile` rows
__device__ inline void run_of(int run, int runs, int tile, int& first, int& end) {
  if (runs == 1) return;
  const int n = max(end - first, 0), per = (n + runs * tile - 1) / (runs * tile) * tile;
  const int from = min(first + run * per, end);
  end = min(from + per, end);
  first = from;
}

// Where the tiles are fewer than two workgroups a CU, each tile's stream is cut into runs of 512 rows or more (eight tiles, about what
// the launch costs that adds the runs' sums, in their order).
inline int runs_for(int64_t workgroups, int64_t streamed) {
  int64_t runs = workgroups ? 512 / workgroups : 1;
  if (runs > streamed / 512) runs = streamed / 512;
  return runs < 1 ? 1 : (int)runs;
}

// ---- forward
// The softmax needs some reference score per row, not the largest one: it moves only when a score exceeds it by more than 2^kLazy, which is
// rare after the first tiles, and the accumulators are rescaled only then.
template <class T, int DP, int NB, int WAVES, bool SKIP>
__global__ __launch_bounds__(WAVES * 64, DP > 128 ? 1 : 2) void forward_kernel(AttnArgs a, int runs, float* part) {
  using El = Elem<T>;
  constexpr int BK = stream_rows<T, DP>(), S = lds_stride<T>(DP), ROWS = WAVES * NB * 16, KB = BK / 16, DB = DP / 16;
  __shared__ __attribute__((aligned(16))) T ks[2][BK * S], vs[2][BK * S];
  const int lane = threadIdx.x & 63, g = lane >> 4, wave = threadIdx.x >> 6;
  const int rows = a.q_len * a.group, tiles = (rows + ROWS - 1) / ROWS;
  const Place at = place_of(a, tiles, runs, kTwo<WAVES, DP>, true);
  const int t = at.tile, b = at.b, hk = at.hk;
  const List l = list_of(a, b);

  int r[NB], lo[NB], hi[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    r[c] = t * ROWS + wave * NB * 16 + c * 16 + (lane & 15);
    seen(a, l, query_of(a, r[c]), lo[c], hi[c]);
  }
  // the tile's keys, and those that all of its queries see
  const int i0 = query_of(a, t * ROWS), i1 = min(query_of(a, t * ROWS + ROWS - 1), l.qn - 1);
  int k0, k1, all0, all1;
  seen(a, l, i0, k0, all1);
  seen(a, l, i1, all0, k1);
  if (i0 >= l.qn) k1 = 0;
  // the keys of this wave's queries
  int w0, w1, unused;
  seen(a, l, min(query_of(a, t * ROWS + wave * NB * 16), l.qn - 1), w0, unused);
  seen(a, l, min(query_of(a, t * ROWS + (wave + 1) * NB * 16 - 1), l.qn - 1), unused, w1);

  // scores keep their order under a scale above zero: a negative one flips the queries' signs, zero takes queries of zero
  const float scale2 = a.scale != 0.f ? fabsf(a.scale) * kLog2e : 1.f;
  typename El::Frag qf[NB][DP / El::KF];
  load_cols<T, DP, NB>(qf, [&](int c) -> const T* {
    const int i = query_of(a, r[c]);
    return i < l.qn && a.scale != 0.f ? row_of<T>(a.q, a.sq, b, i, hk * a.group + r[c] - i * a.group) : nullptr;
  }, a.d, a.scale < 0.f ? (sizeof(T) == 4 ? 0x80000000u : 0x80008000u) : 0u);

  floatx4 o[DB][NB];
  float m[NB], sum[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    m[c] = -INFINITY;
    sum[c] = 0.f;
#pragma unroll
    for (int x = 0; x < DB; ++x) o[x][c] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  StreamMove<T, BK, DP, WAVES * 64> mk, mv;
  int kt = k0 / 16 * 16, buf = 0;
  run_of(at.run, runs, BK, kt, k1);
  const RowEnd end = row_end<T>(a.d);
  mk.start_rows(row_of<T>(a.k, a.sk, b, kt, hk), a.sk.row, a.d);
  mv.start_rows(row_of<T>(a.v, a.sv, b, kt, hk), a.sv.row, a.d);
  if (kt < k1) {
    mk.fetch(l.kn - kt, end);
    mv.fetch(l.kn - kt, end);
    mk.store(ks[0], end);
    mv.store(vs[0], end);
  }
  for (; kt < k1; kt += BK, buf ^= 1) {
    __syncthreads();                                          // this tile is there, and nobody reads the other buffer any more
    const bool more = kt + BK < k1;
    if (more) {
      mk.fetch(l.kn - kt - BK, end);
      mv.fetch(l.kn - kt - BK, end);
    }
    if (kt < w1 && kt + BK > w0) {
      floatx4 s[KB][NB];
#pragma unroll
      for (int y = 0; y < KB; ++y) {
#pragma unroll
        for (int c = 0; c < NB; ++c) s[y][c] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < DP / El::KF; ++k) {
          if (SKIP && k > 0 && k * El::KF >= a.d) break;
          const typename El::Frag f = placed_rows<T, DP>(ks[buf], y * 16, k * El::KF);
#pragma unroll
          for (int c = 0; c < NB; ++c) s[y][c] = El::mma(f, qf[c][k], s[y][c]);
        }
      }
      if (kt < all0 || kt + BK > all1) {
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
          for (int y = 0; y < KB; ++y)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const int j = kt + y * 16 + 4 * g + u;
              s[y][c][u] = j >= lo[c] && j < hi[c] ? s[y][c][u] : -INFINITY;
            }
      }
      float top[NB];
      bool grows = false;
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        top[c] = -INFINITY;
#pragma unroll
        for (int y = 0; y < KB; ++y)
#pragma unroll
          for (int u = 0; u < 4; ++u) top[c] = fmaxf(top[c], s[y][c][u]);
        grows |= top[c] * scale2 > m[c] + kLazy;              // (a lane's own scores: the row's largest is among them in some lane)
      }
      if (__any(grows)) {
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          const float next = fmaxf(m[c], over_groups_max(top[c]) * scale2);
          const float shrink = __builtin_amdgcn_exp2f(m[c] - (next == -INFINITY ? 0.f : next));
          m[c] = next;
          sum[c] *= shrink;
#pragma unroll
          for (int x = 0; x < DB; ++x) o[x][c] *= shrink;
        }
      }
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const float less = kShiftLazy<T> - (m[c] == -INFINITY ? 0.f : m[c]);     // (a row that has seen no key yet: any)
#pragma unroll
        for (int y = 0; y < KB; ++y)
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[y][c][u], scale2, less));
            s[y][c][u] = p;
            sum[c] += p;
          }
      }
#pragma unroll
      for (int y = 0; y < KB; y += El::PB) {
        typename El::Frag pf[NB];
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          floatx4 blocks[El::PB];
#pragma unroll
          for (int u = 0; u < El::PB; ++u) blocks[u] = s[y + u][c];
          pf[c] = pack<T>(blocks);
        }
#pragma unroll
        for (int x = 0; x < DB; ++x) {
          if (SKIP && x > 0 && x * 16 >= a.d) break;
          const typename El::Frag f = placed_cols<T, DP>(vs[buf], y * 16, x * 16);
#pragma unroll
          for (int c = 0; c < NB; ++c) o[x][c] = El::mma(f, pf[c], o[x][c]);
        }
      }
    }
    if (more) {
      mk.store(ks[buf ^ 1], end);
      mv.store(vs[buf ^ 1], end);
    }
  }

#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const float total = over_groups_sum(sum[c]);
    if (r[c] >= rows) continue;
    const int i = query_of(a, r[c]), head = hk * a.group + r[c] - i * a.group;
    if (runs > 1) {                                           // (as the runs of few queries are kept)
      float* p = part + (((int64_t)(b * a.kv_heads + hk) * runs + at.run) * rows + r[c]) * (a.d + 2);
#pragma unroll
      for (int x = 0; x < DB; ++x) store4(p + 2, x * 16 + 4 * g, a.d, o[x][c]);
      if (g == 0) { p[0] = m[c] - kShiftLazy<T>; p[1] = total; }
      continue;
    }
    const bool any = hi[c] > lo[c];
    const float inv = any ? 1.f / total : 0.f;
    T* row = const_cast<T*>(row_of<T>(a.o, a.so, b, i, head));
#pragma unroll
    for (int x = 0; x < DB; ++x) {
      floatx4 v = any ? o[x][c] * inv : floatx4{0.f, 0.f, 0.f, 0.f};
      store4(row, x * 16 + 4 * g, a.d, v);
    }
    if (g == 0)
      a.lse[((int64_t)b * a.heads + head) * a.q_len + i] = any ? (m[c] - kShiftLazy<T> + __builtin_amdgcn_logf(total)) * kLn2 : -INFINITY;
  }
}

// ---- gradients
// dq, and delta_i = do_i . o_i (what the softmax's normalisation takes off every dp of the row) for the dk/dv kernel behind it: queries in
// registers, keys and values stream.  With 16-bit types, o is rounded; where a tile holds all keys of the list, delta is the sum of p dp
// instead, from the unrounded weights: a short list's delta is not small beside its dp (lists of 10 to 30 keys in bf16: dq 0.27 % off, 0.24 %
// with it; half of that is the rounding of dq itself).
template <class T, int DP, int NB, int WAVES, bool SKIP>
__global__ __launch_bounds__(WAVES * 64, DP > 128 ? 1 : 2) void query_grad_kernel(AttnArgs a, int runs, float* part) {
  using El = Elem<T>;
  constexpr int BK = stream_rows<T, DP>(), S = lds_stride<T>(DP), ROWS = WAVES * NB * 16, DB = DP / 16, PB = El::PB;
  __shared__ __attribute__((aligned(16))) T ks[2][BK * S], vs[2][BK * S];
  const int lane = threadIdx.x & 63, g = lane >> 4, wave = threadIdx.x >> 6;
  const int rows = a.q_len * a.group, tiles = (rows + ROWS - 1) / ROWS;
  const Place pos = place_of(a, tiles, runs, kTwo<WAVES, DP>, true);
  const int t = pos.tile, b = pos.b, hk = pos.hk;
  const List l = list_of(a, b);

  int r[NB], lo[NB], hi[NB], head[NB], qi[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    r[c] = t * ROWS + wave * NB * 16 + c * 16 + (lane & 15);
    qi[c] = query_of(a, r[c]);
    head[c] = hk * a.group + r[c] - qi[c] * a.group;
    seen(a, l, qi[c], lo[c], hi[c]);
  }
  const int i0 = query_of(a, t * ROWS), i1 = min(query_of(a, t * ROWS + ROWS - 1), l.qn - 1);
  int k0, k1, all0, all1;
  seen(a, l, i0, k0, all1);
  seen(a, l, i1, all0, k1);
  if (i0 >= l.qn) k1 = 0;
  int w0, w1, unused;
  seen(a, l, min(query_of(a, t * ROWS + wave * NB * 16), l.qn - 1), w0, unused);
  seen(a, l, min(query_of(a, t * ROWS + (wave + 1) * NB * 16 - 1), l.qn - 1), unused, w1);

  typename El::Frag qf[NB][DP / El::KF], df[NB][DP / El::KF];
  load_cols<T, DP, NB>(qf, [&](int c) -> const T* { return qi[c] < l.qn ? row_of<T>(a.q, a.sq, b, qi[c], head[c]) : nullptr; }, a.d);
  load_cols<T, DP, NB>(df, [&](int c) -> const T* { return qi[c] < l.qn ? row_of<T>(a.dout, a.sdo, b, qi[c], head[c]) : nullptr; }, a.d);

  StreamMove<T, BK, DP, WAVES * 64> mk, mv;
  int kt = k0 / 16 * 16, buf = 0;
  const bool one_tile = sizeof(T) == 2 && kt < k1 && k1 - kt <= BK;
  run_of(pos.run, runs, BK, kt, k1);
  const RowEnd end = row_end<T>(a.d);
  mk.start_rows(row_of<T>(a.k, a.sk, b, kt, hk), a.sk.row, a.d);
  mv.start_rows(row_of<T>(a.v, a.sv, b, kt, hk), a.sv.row, a.d);
  if (kt < k1) {
    mk.fetch(l.kn - kt, end);
    mv.fetch(l.kn - kt, end);
    mk.store(ks[0], end);
    mv.store(vs[0], end);
  }

  const float scale2 = a.scale * kLog2e;
  float lse2[NB], delta[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const bool any = hi[c] > lo[c];
    const int64_t at = ((int64_t)b * a.heads + head[c]) * a.q_len + qi[c];
    lse2[c] = any ? a.lse[at] * kLog2e : INFINITY;            // a row that sees nothing has no probability
    const T* o = row_of<T>(a.out, a.so, b, qi[c], head[c]);
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < DP / El::KF; ++k) {
      const int from = k * El::KF + El::E * g;
      const typename El::Frag f = __builtin_bit_cast(typename El::Frag, any && from < a.d ? load16(o + from, a.d - from, end) : u32x4{0, 0, 0, 0});
#pragma unroll
      for (int e = 0; e < El::E; ++e) sum = fmaf((float)df[c][k][e], (float)f[e], sum);
    }
    delta[c] = any ? over_groups_sum(sum) : 0.f;
  }
  // p and dp of the rows y .. y + PB of a tile
  auto weights = [&](int y, floatx4 (&p)[PB][NB], floatx4 (&dp)[PB][NB], bool partial) {
#pragma unroll
    for (int u = 0; u < PB; ++u) {
#pragma unroll
      for (int c = 0; c < NB; ++c) p[u][c] = dp[u][c] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < DP / El::KF; ++k) {
        if (SKIP && k > 0 && k * El::KF >= a.d) break;
        const typename El::Frag kf = placed_rows<T, DP>(ks[buf], (y + u) * 16, k * El::KF), vf = placed_rows<T, DP>(vs[buf], (y + u) * 16, k * El::KF);
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          p[u][c] = El::mma(kf, qf[c][k], p[u][c]);
          dp[u][c] = El::mma(vf, df[c][k], dp[u][c]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < PB; ++u)
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) p[u][c][e] = __builtin_amdgcn_exp2f(fmaf(p[u][c][e], scale2, -lse2[c]));
    if (partial) {
#pragma unroll
      for (int u = 0; u < PB; ++u)
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = kt + (y + u) * 16 + 4 * g + e;
            const bool sees = j >= lo[c] && j < hi[c];
            p[u][c][e] = sees ? p[u][c][e] : 0.f;
            dp[u][c][e] = sees ? dp[u][c][e] : 0.f;           // (a masked value may be the type's largest: zero times an infinite product)
          }
    }
  };
  if (one_tile && kt < k1) {
    __syncthreads();
    float sum[NB] = {};
    for (int y = 0; y < BK / 16; y += PB) {
      floatx4 p[PB][NB], dp[PB][NB];
      weights(y, p, dp, true);
#pragma unroll
      for (int u = 0; u < PB; ++u)
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[c] = fmaf(p[u][c][e], dp[u][c][e], sum[c]);
    }
#pragma unroll
    for (int c = 0; c < NB; ++c) delta[c] = over_groups_sum(sum[c]);
  }
#pragma unroll
  for (int c = 0; c < NB; ++c)
    if (g == 0 && r[c] < rows && pos.run == 0) a.delta[((int64_t)b * a.heads + head[c]) * a.q_len + qi[c]] = delta[c];

  floatx4 dq[DB][NB];
#pragma unroll
  for (int x = 0; x < DB; ++x)
#pragma unroll
    for (int c = 0; c < NB; ++c) dq[x][c] = floatx4{0.f, 0.f, 0.f, 0.f};
  Fit<NB> fit;                                                // (the weights' exponents carry its powers: they are for ds alone here)
#pragma unroll
  for (int c = 0; c < NB; ++c)
    if constexpr (kFitted<T>) lse2[c] -= exponent_of(fit.times[c]);
  for (; kt < k1; kt += BK, buf ^= 1) {
    __syncthreads();
    const bool more = kt + BK < k1;
    if (more) {
      mk.fetch(l.kn - kt - BK, end);
      mv.fetch(l.kn - kt - BK, end);
    }
    if (kt < w1 && kt + BK > w0) {
      const bool partial = kt < all0 || kt + BK > all1;
#pragma unroll
      for (int y = 0; y < BK / 16; y += PB) {
        floatx4 p[PB][NB], dp[PB][NB];
        weights(y, p, dp, partial);
        typename El::Frag f[NB];
        floatx4 ds[NB][PB];
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
          for (int u = 0; u < PB; ++u) ds[c][u] = p[u][c] * (dp[u][c] - delta[c]);
        if constexpr (kFitted<T>) {
          float top[NB] = {};
#pragma unroll
          for (int c = 0; c < NB; ++c)
#pragma unroll
            for (int u = 0; u < PB; ++u)
#pragma unroll
              for (int e = 0; e < 4; ++e) top[c] = fmaxf(top[c], fabsf(ds[c][u][e]));
          fit.take(top, [&](int c, float by) {
            lse2[c] -= exponent_of(by);
#pragma unroll
            for (int u = 0; u < PB; ++u) ds[c][u] *= by;
#pragma unroll
            for (int x = 0; x < DB; ++x) dq[x][c] *= by;
          });
        }
#pragma unroll
        for (int c = 0; c < NB; ++c) f[c] = pack<T>(ds[c]);
#pragma unroll
        for (int x = 0; x < DB; ++x) {
          if (SKIP && x > 0 && x * 16 >= a.d) break;
          const typename El::Frag kf = placed_cols<T, DP>(ks[buf], y * 16, x * 16);
#pragma unroll
          for (int c = 0; c < NB; ++c) dq[x][c] = El::mma(kf, f[c], dq[x][c]);
        }
      }
    }
    if (more) {
      mk.store(ks[buf ^ 1], end);
      mv.store(vs[buf ^ 1], end);
    }
  }
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    if (r[c] >= rows) continue;
    const bool any = hi[c] > lo[c];
    const float by = kFitted<T> ? a.scale * fit.undo(c) : a.scale;
    if (runs > 1) {
      float* p = part + (((int64_t)(b * a.kv_heads + hk) * runs + pos.run) * rows + r[c]) * a.d;
#pragma unroll
      for (int x = 0; x < DB; ++x) store4(p, x * 16 + 4 * g, a.d, any ? dq[x][c] * by : floatx4{0.f, 0.f, 0.f, 0.f});
      continue;
    }
    T* row = dense_row<T>(a, a.dq, a.q_len, a.heads, b, qi[c], head[c]);
#pragma unroll
    for (int x = 0; x < DB; ++x) store4(row, x * 16 + 4 * g, a.d, any ? dq[x][c] * by : floatx4{0.f, 0.f, 0.f, 0.f});
  }
}

// Rows (query, head) of one list and key head on their way into LDS.  Where the heads that share a key head divide the rows between a
// thread's pieces, its pieces keep their heads and advance by a tile's queries.  Other numbers of heads take a division a piece.
template <class T, int BQ, int DP, int THREADS>
struct RowMove : StreamMove<T, BQ, DP, THREADS> {
  using Base = StreamMove<T, BQ, DP, THREADS>;
  static __device__ inline bool steady(const AttnArgs& a) { return a.group_shift >= 0 && a.group <= Base::APART; }
  __device__ inline void start_queries(const AttnArgs& a, const void* base, const Strides& st, int b, int hk, int rt) {
    if (!steady(a)) return;                                   // (rt: the first row of a query)
    const int row = rt + (int)threadIdx.x / Base::PER_ROW, q = row >> a.group_shift;
    this->start(row_of<T>(base, st, b, q, hk * a.group + row - (q << a.group_shift)), (int64_t)(Base::APART >> a.group_shift) * st.row,
                (int64_t)(BQ >> a.group_shift) * st.row, a.d);
  }
  __device__ inline void fetch_queries(const AttnArgs& a, const void* base, const Strides& st, int b, int hk, int rt, int r1, RowEnd end) {
    if (steady(a)) {
      this->fetch(r1 - rt, end);
      return;
    }
    const int c = (int)threadIdx.x % Base::PER_ROW * Base::E, count = a.d - c;
#pragma unroll
    for (int i = 0; i < Base::NP; ++i) {
      const int row = rt + (int)threadIdx.x / Base::PER_ROW + i * Base::APART;
      this->r[i] = u32x4{0, 0, 0, 0};
      if (count > 0 && row < r1) {
        const int q = query_of(a, row);
        const T* p = row_of<T>(base, st, b, q, hk * a.group + row - q * a.group) + c;
        if (end == kShort) this->r[i] = load16<T, kShort>(p, count);
        else this->r[i] = *reinterpret_cast<const u32x4_any*>(p - (end == kWide ? Base::early(count) : 0));
      }
    }
  }
};

// dk, dv: keys and values in registers, queries and dout stream
template <class T, int DP, int NB, int WAVES, int BQ, int OCC, bool SKIP>
__global__ __launch_bounds__(WAVES * 64, OCC) void key_grad_kernel(AttnArgs a, int runs, float* part) {
  using El = Elem<T>;
  constexpr int S = lds_stride<T>(DP), KEYS = WAVES * NB * 16, DB = DP / 16, PB = El::PB;
  __shared__ __attribute__((aligned(16))) T qs[2][BQ * S], gs[2][BQ * S];
  __shared__ __attribute__((aligned(16))) float lses[2][BQ], deltas[2][BQ];
  __shared__ int los[2][BQ], his[2][BQ];
  const int lane = threadIdx.x & 63, g = lane >> 4, wave = threadIdx.x >> 6;
  const int tiles = (a.k_len + KEYS - 1) / KEYS;
  const Place pos = place_of(a, tiles, runs, kTwo<WAVES, DP>, false);
  const int t = pos.tile, b = pos.b, hk = pos.hk;
  const List l = list_of(a, b);
  const int j0 = t * KEYS, jw = j0 + wave * NB * 16 + (lane & 15);

  // queries that see a key of the tile, and those that see all of them
  int q0 = 0, q1 = l.qn, all0 = 0, all1 = l.qn;
  const int jlast = min(j0 + KEYS, l.kn) - 1;
  if (a.causal) {
    q0 = max(0, j0 - l.shift);
    all0 = max(0, j0 + KEYS - 1 - l.shift);
    if (a.window) {
      q1 = min(q1, jlast + a.window - l.shift);
      all1 = min(all1, j0 + a.window - l.shift);
    }
  }
  if (j0 >= l.kn) q1 = 0;
  q0 = min(q0, l.qn);
  q1 = max(q1, 0);
  const bool whole_tile = j0 + KEYS <= l.kn;

  typename El::Frag kf[NB][DP / El::KF], vf[NB][DP / El::KF];
  load_cols<T, DP, NB>(kf, [&](int c) -> const T* { return jw + c * 16 < l.kn ? row_of<T>(a.k, a.sk, b, jw + c * 16, hk) : nullptr; }, a.d);
  load_cols<T, DP, NB>(vf, [&](int c) -> const T* { return jw + c * 16 < l.kn ? row_of<T>(a.v, a.sv, b, jw + c * 16, hk) : nullptr; }, a.d);

  const float scale2 = a.scale * kLog2e;
  floatx4 dk[DB][NB], dv[DB][NB];
#pragma unroll
  for (int x = 0; x < DB; ++x)
#pragma unroll
    for (int c = 0; c < NB; ++c) dk[x][c] = dv[x][c] = floatx4{0.f, 0.f, 0.f, 0.f};
  Fit<NB> fit;

  RowMove<T, BQ, DP, WAVES * 64> mq, md;
  float ml = 0.f, mt = 0.f;
  int mlo = 0, mhi = 0;
  int rt = q0 * a.group, r1 = q1 * a.group, buf = 0;
  run_of(pos.run, runs, BQ, rt, r1);
  const RowEnd end = row_end<T>(a.d);
  mq.start_queries(a, a.q, a.sq, b, hk, rt);
  md.start_queries(a, a.dout, a.sdo, b, hk, rt);
  auto fetch = [&](int rt) {
    mq.fetch_queries(a, a.q, a.sq, b, hk, rt, r1, end);
    md.fetch_queries(a, a.dout, a.sdo, b, hk, rt, r1, end);
    if ((int)threadIdx.x < BQ) {
      const int r = rt + (int)threadIdx.x, i = query_of(a, r), head = hk * a.group + r - i * a.group;
      ml = INFINITY;                                          // a row that sees nothing has no probability
      mt = 0.f;
      mlo = mhi = 0;
      if (r < r1) {
        seen(a, l, i, mlo, mhi);
        const int64_t at = ((int64_t)b * a.heads + head) * a.q_len + i;
        if (mhi > mlo) { ml = a.lse[at] * kLog2e - kShift<T>; mt = a.delta[at]; }
      }
    }
  };
  auto store = [&](int buf) {
    mq.store(qs[buf], end, a.d - (int)threadIdx.x % mq.PER_ROW * El::E);
    md.store(gs[buf], end, a.d - (int)threadIdx.x % md.PER_ROW * El::E);
    if ((int)threadIdx.x < BQ) { lses[buf][threadIdx.x] = ml; deltas[buf][threadIdx.x] = mt; los[buf][threadIdx.x] = mlo; his[buf][threadIdx.x] = mhi; }
  };
  if (rt < r1) {
    fetch(rt);
    store(0);
  }
  for (; rt < r1; rt += BQ, buf ^= 1) {
    __syncthreads();
    const bool more = rt + BQ < r1;
    if (more) fetch(rt + BQ);
    const bool partial = !whole_tile || query_of(a, rt) < all0 || query_of(a, rt + BQ - 1) >= all1;
    const T *qt = qs[buf], *gt = gs[buf];
#pragma unroll
    for (int y = 0; y < BQ / 16; y += PB) {
      if (rt + y * 16 >= r1) break;                           // (the last tile's rows behind the end)
      floatx4 s[PB][NB], dp[PB][NB];
#pragma unroll
      for (int u = 0; u < PB; ++u) {
#pragma unroll
        for (int c = 0; c < NB; ++c) s[u][c] = dp[u][c] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < DP / El::KF; ++k) {
          if (SKIP && k > 0 && k * El::KF >= a.d) break;
          const typename El::Frag qf = placed_rows<T, DP>(qt, (y + u) * 16, k * El::KF), df = placed_rows<T, DP>(gt, (y + u) * 16, k * El::KF);
#pragma unroll
          for (int c = 0; c < NB; ++c) {
            s[u][c] = El::mma(qf, kf[c][k], s[u][c]);
            dp[u][c] = El::mma(df, vf[c][k], dp[u][c]);
          }
        }
      }
      typename El::Frag pf[NB], ef[NB];
#pragma unroll
      for (int u = 0; u < PB; ++u) {
        const int at = (y + u) * 16 + 4 * g;
        const floatx4 ls = *reinterpret_cast<const floatx4*>(lses[buf] + at), dl = *reinterpret_cast<const floatx4*>(deltas[buf] + at);
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float p = __builtin_amdgcn_exp2f(fmaf(s[u][c][e], scale2, -ls[e]));      // (2^kShift times)
            if (partial) {
              const int j = jw + c * 16;
              const bool sees = j >= los[buf][at + e] && j < his[buf][at + e];
              p = sees ? p : 0.f;
              dp[u][c][e] = sees ? dp[u][c][e] : 0.f;         // (as in the dq kernel)
            }
            s[u][c][e] = p;
            dp[u][c][e] = p * (dp[u][c][e] - dl[e]);
          }
      }
      if constexpr (kFitted<T>) {
        float top[NB] = {};
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
          for (int u = 0; u < PB; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              dp[u][c][e] *= fit.times[c];
              top[c] = fmaxf(top[c], fabsf(dp[u][c][e]));
            }
        fit.take(top, [&](int c, float by) {
#pragma unroll
          for (int u = 0; u < PB; ++u) dp[u][c] *= by;
#pragma unroll
          for (int x = 0; x < DB; ++x) dk[x][c] *= by;
        });
      }
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        floatx4 pb[PB], eb[PB];
#pragma unroll
        for (int u = 0; u < PB; ++u) { pb[u] = s[u][c]; eb[u] = dp[u][c]; }
        pf[c] = pack<T>(pb);
        ef[c] = pack<T>(eb);
      }
#pragma unroll
      for (int x = 0; x < DB; ++x) {
        if (SKIP && x > 0 && x * 16 >= a.d) break;
        const typename El::Frag df = placed_cols<T, DP>(gt, y * 16, x * 16), qf = placed_cols<T, DP>(qt, y * 16, x * 16);
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          dv[x][c] = El::mma(df, pf[c], dv[x][c]);
          dk[x][c] = El::mma(qf, ef[c], dk[x][c]);
        }
      }
    }
    if (more) store(buf ^ 1);
  }
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const int j = jw + c * 16;
    if (j >= a.k_len) continue;
    const float by = kFitted<T> ? a.scale * kUnshift<T> * fit.undo(c) : a.scale;
    if (runs > 1) {                                           // dk's runs, then dv's
      const int64_t unit = (int64_t)b * a.kv_heads + hk, kept = (int64_t)a.lists * a.kv_heads * runs * a.k_len * a.d;
      float* p = part + ((unit * runs + pos.run) * a.k_len + j) * a.d;
#pragma unroll
      for (int x = 0; x < DB; ++x) {
        store4(p, x * 16 + 4 * g, a.d, dk[x][c] * by);
        store4(p + kept, x * 16 + 4 * g, a.d, kShift<T> != 0.f ? dv[x][c] * kUnshift<T> : dv[x][c]);
      }
      continue;
    }
    T* krow = dense_row<T>(a, a.dk, a.k_len, a.kv_heads, b, j, hk);
    T* vrow = dense_row<T>(a, a.dv, a.k_len, a.kv_heads, b, j, hk);
#pragma unroll
    for (int x = 0; x < DB; ++x) {
      store4(krow, x * 16 + 4 * g, a.d, dk[x][c] * by);
      store4(vrow, x * 16 + 4 * g, a.d, kShift<T> != 0.f ? dv[x][c] * kUnshift<T> : dv[x][c]);
    }
  }
}

// The runs of a row are joined by a wave, or where they are many by the four waves of a workgroup (one row 256 runs one after the other
// took longer than the runs), four numbers a lane; always in the same order.
constexpr int kManyRuns = 16;
inline int64_t join_grid(int64_t rows, int runs) { return runs >= kManyRuns ? rows : (rows + 3) / 4; }

// sums of f(run) over the runs that this wave takes, then over the workgroup's waves where they share the row; true where the sum is
template <class F>
__device__ inline bool over_runs(int runs, F f, floatx4& v, float& extra) {
  __shared__ floatx4 part[4][64];
  __shared__ float parts[4][64];
  const bool many = runs >= kManyRuns;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = floatx4{0.f, 0.f, 0.f, 0.f};
  extra = 0.f;
#pragma unroll 4
  for (int s = many ? wave : 0; s < runs; s += many ? 4 : 1) f(s, v, extra);
  if (!many) return true;
  part[wave][lane] = v;
  parts[wave][lane] = extra;
  __syncthreads();
  if (wave) return false;
  v = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
  extra = (parts[0][lane] + parts[1][lane]) + (parts[2][lane] + parts[3][lane]);
  return true;
}

// out, lse: the runs' softmaxes
template <class T>
__global__ __launch_bounds__(256) void join_kernel(AttnArgs a, int runs, const float* part) {
  const int rows = a.q_len * a.group, lane = threadIdx.x & 63;
  const int64_t n = (int64_t)a.lists * a.kv_heads * rows, x = runs >= kManyRuns ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (x >= n) return;
  const int64_t unit = x / rows;
  const int r = (int)(x % rows), b = (int)(unit / a.kv_heads), hk = (int)(unit % a.kv_heads);
  const int i = query_of(a, r), head = hk * a.group + r - i * a.group;
  const List l = list_of(a, b);
  int lo, hi;
  seen(a, l, i, lo, hi);
  const bool any = hi > lo;
  const int64_t ld = a.d + 2;
  const float* p = part + (unit * runs * rows + r) * ld;
  float top = -INFINITY;
  for (int s = lane; s < runs; s += 64) top = fmaxf(top, p[(int64_t)s * rows * ld]);
  for (int w = 32; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
  const float ref = top == -INFINITY ? 0.f : top;
  float sum;
  floatx4 o;
  const int at = 4 * lane;
  const bool mine = over_runs(runs, [&](int s, floatx4& v, float& t) {
    const float* y = p + (int64_t)s * rows * ld;              // (a run behind the list's end holds zeros)
    const float w = __builtin_amdgcn_exp2f(y[0] - ref);
    t += y[1] * w;
    if (at < a.d) v += load4(y + 2, at, a.d) * w;
  }, o, sum);
  if (!mine) return;
  const float inv = any ? 1.f / sum : 0.f;
  if (at < a.d) store4(const_cast<T*>(row_of<T>(a.o, a.so, b, i, head)), at, a.d, any ? o * inv : floatx4{0.f, 0.f, 0.f, 0.f});
  if (lane == 0) a.lse[((int64_t)b * a.heads + head) * a.q_len + i] = any ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
}

// A gradient's rows [lists, len, kv_heads * group], or two gradients' one after the other: the runs' sums
template <class T>
__global__ __launch_bounds__(256) void sum_runs_kernel(AttnArgs a, void* out, void* second, int len, int group, int runs, const float* part) {
  const int rows = len * group, at = 4 * (threadIdx.x & 63);
  const int64_t n = (int64_t)a.lists * a.kv_heads * rows;
  int64_t x = runs >= kManyRuns ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (x >= n && second) {
    x -= n;
    out = second;
    part += n * runs * a.d;
  }
  if (x >= n) return;
  const int64_t unit = x / rows;
  const int r = (int)(x % rows), b = (int)(unit / a.kv_heads), hk = (int)(unit % a.kv_heads), i = r / group;
  const float* p = part + (unit * runs * rows + r) * a.d;
  floatx4 v;
  float none;
  const bool mine = over_runs(runs, [&](int s, floatx4& v, float&) {
    if (at < a.d) v += load4(p + (int64_t)s * rows * a.d, at, a.d);
  }, v, none);
  if (mine && at < a.d) store4(dense_row<T>(a, out, len, a.kv_heads * group, b, i, hk * group + r - i * group), at, a.d, v);
}
template <class T>
hipError_t sum_runs(const AttnArgs& a, void* out, void* second, int len, int group, int runs, const float* part, hipStream_t s) {
  const int64_t rows = (int64_t)a.lists * a.kv_heads * len * group * (second ? 2 : 1);
  return launch(sum_runs_kernel<T>, join_grid(rows, runs), 256, s, a, out, second, len, group, runs, part);
}

// How many rows or keys a workgroup takes.  16-bit types: 128 queries, four waves of 32; the dk/dv kernel keeps twice the operands and
// sums a wave, so eight waves of 16 keys (four of 32 in 479 registers, one wave a SIMD: half as long again; four of 32 with the values
// in LDS: as long as these).  fp32: 64, four waves
// of 16.
template <class T, int DP>
struct Shape {
  static constexpr int NB = sizeof(T) == 4 || DP > 128 ? 1 : 2, BQ = stream_rows<T, DP>();
  // rows between two barriers: twice as many where one workgroup has the CU to itself and its waves wait for each other (4 x 4,096 causal,
  // 16 heads on 4: the gradient 1,435 -> 1,342 us)
  static constexpr int KBQ = sizeof(T) == 2 && DP == 128 ? 128 : BQ;
  static constexpr int KW = sizeof(T) == 2 && DP <= 128 ? 8 : 4, OCC = DP > 128 ? 1 : sizeof(T) == 2 && DP == 64 ? 4 : 2;
  // Heads of up to three quarters of DP numbers have kernels that ask before every product whether it is all padding (80 of 128: fp32 a quarter
  // less time, bf16 a tenth); wider ones would only pay for the question (4 to 15 %).
  static bool skips(const AttnArgs& a) { return a.d * 4 <= DP * 3; }
  static int64_t query_tiles(const AttnArgs& a) { return ((int64_t)a.q_len * a.group + 64 * NB - 1) / (64 * NB); }
  static int64_t key_tiles(const AttnArgs& a) { return ((int64_t)a.k_len + 16 * KW - 1) / (16 * KW); }
  static int64_t pairs(const AttnArgs& a) { return (int64_t)a.lists * a.kv_heads; }
  static int64_t reach(const AttnArgs& a, int64_t len, int64_t tile) { return a.window && a.window + tile < len ? a.window + tile : len; }
  static int query_runs(const AttnArgs& a) { return runs_for(query_tiles(a) * pairs(a), reach(a, a.k_len, 64 * NB / a.group + 1)); }
  static int key_runs(const AttnArgs& a) { return runs_for(key_tiles(a) * pairs(a), reach(a, a.q_len, 16 * KW) * a.group); }
  static size_t forward_bytes(const AttnArgs& a) {
    const int r = query_runs(a);
    return r > 1 ? (size_t)pairs(a) * r * a.q_len * a.group * (a.d + 2) * sizeof(float) : 0;
  }
  // delta | the runs' sums of dq, and after it of dk and dv
  static size_t delta_bytes(const AttnArgs& a) { return ((size_t)a.lists * a.q_len * a.heads * sizeof(float) + 255) / 256 * 256; }
  static size_t backward_bytes(const AttnArgs& a) {
    const int rq = query_runs(a), rk = key_runs(a);
    const size_t q = rq > 1 ? (size_t)pairs(a) * rq * a.q_len * a.group * a.d : 0, k = rk > 1 ? (size_t)pairs(a) * rk * a.k_len * a.d * 2 : 0;
    return delta_bytes(a) + (q > k ? q : k) * sizeof(float);
  }
};

template <class T, int DP>
hipError_t forward(const AttnArgs& a, float* part, hipStream_t s) {
  using Sh = Shape<T, DP>;
  const int runs = Sh::query_runs(a);
  const auto kernel = Sh::skips(a) ? forward_kernel<T, DP, Sh::NB, 4, true> : forward_kernel<T, DP, Sh::NB, 4, false>;
  const hipError_t e = launch(kernel, Sh::query_tiles(a) * Sh::pairs(a) * runs, 256, s, a, runs, part);
  if (e != hipSuccess || runs == 1) return e;
  return launch(join_kernel<T>, join_grid(Sh::pairs(a) * a.q_len * a.group, runs), 256, s, a, runs, (const float*)part);
}

template <class T, int DP>
hipError_t backward(AttnArgs a, void* ws, hipStream_t s) {
  using Sh = Shape<T, DP>;
  a.delta = static_cast<float*>(ws);
  float* part = reinterpret_cast<float*>(static_cast<char*>(ws) + Sh::delta_bytes(a));
  const int rq = Sh::query_runs(a), rk = Sh::key_runs(a);
  hipError_t e = hipSuccess;
  if (a.q_len) {
    const auto kernel = Sh::skips(a) ? query_grad_kernel<T, DP, Sh::NB, 4, true> : query_grad_kernel<T, DP, Sh::NB, 4, false>;
    e = launch(kernel, Sh::query_tiles(a) * Sh::pairs(a) * rq, 256, s, a, rq, part);
    if (e == hipSuccess && rq > 1) e = sum_runs<T>(a, a.dq, nullptr, a.q_len, a.group, rq, part, s);
  }
  if (e == hipSuccess && a.k_len) {
    const auto kernel = Sh::skips(a) ? key_grad_kernel<T, DP, 1, Sh::KW, Sh::KBQ, Sh::OCC, true> : key_grad_kernel<T, DP, 1, Sh::KW, Sh::KBQ, Sh::OCC, false>;
    e = launch(kernel, Sh::key_tiles(a) * Sh::pairs(a) * rk, Sh::KW * 64, s, a, rk, part);
    if (e == hipSuccess && rk > 1) e = sum_runs<T>(a, a.dk, a.dv, a.k_len, 1, rk, part, s);
  }
  return e;
}

template <class T, class F>
auto by_width(const AttnArgs& a, F f) {
  return a.d <= 64 ? f(Shape<T, 64>(), std::integral_constant<int, 64>()) : a.d <= 128 ? f(Shape<T, 128>(), std::integral_constant<int, 128>())
                                                                                       : f(Shape<T, 256>(), std::integral_constant<int, 256>());
}
template <class T>
hipError_t forward_of(const AttnArgs& a, void* ws, hipStream_t s) {
  return by_width<T>(a, [&](auto, auto d) { return forward<T, d()>(a, static_cast<float*>(ws), s); });
}
template <class T>
hipError_t backward_of(const AttnArgs& a, void* ws, hipStream_t s) {
  return by_width<T>(a, [&](auto, auto d) { return backward<T, d()>(a, ws, s); });
}
template <class T>
size_t forward_bytes_of(const AttnArgs& a) { return by_width<T>(a, [&](auto sh, auto) { return sh.forward_bytes(a); }); }
template <class T>
size_t backward_bytes_of(const AttnArgs& a) { return by_width<T>(a, [&](auto sh, auto) { return sh.backward_bytes(a); }); }

}  // namespace attn
}  // namespace stgn
