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
// fewer bits (5,000 keys: dv 0.5 % off).  None exceeds 1, so none overflows.  (ds has no such bound and is taken as it is.)
template <class T> constexpr float kShift = std::is_same<T, _Float16>::value ? 14.f : 0.f;
template <class T> constexpr float kUnshift = kShift<T> != 0.f ? 1.f / 16384.f : 1.f;

// In the forward call the reference score may lag the largest one by kLazy powers of two (see there): 2^7 times there.
template <class T> constexpr float kShiftLazy = kShift<T> / 2.f;
constexpr float kLazy = 8.f;

// rows of a streamed tile: two tiles of 64 x 128 16-bit numbers and their padding are 34 KB, four workgroups a CU
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
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const T* p = row(c);
#pragma unroll
    for (int k = 0; k < DP / KF; ++k) {
      const int at = k * KF + E * g;
      u32x4 v = p != nullptr ? load16(p + at, d - at) : u32x4{0, 0, 0, 0};
      if (flip) v ^= flip;
      f[c][k] = __builtin_bit_cast(typename Elem<T>::Frag, v);
    }
  }
}

__device__ inline float over_groups_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float over_groups_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Workgroup -> (tile of a list and key head, list, key head).  The last tiles come first: with `causal` they are the longest.  One tile
// number of all lists and heads after the other, so that workgroups that read the same keys are a multiple of the number of lists
// and heads apart, on one die where that is a multiple of eight.
__device__ inline int place_of(const AttnArgs& a, int tiles, int& b, int& hk) {
  const unsigned pairs = (unsigned)a.lists * (unsigned)a.kv_heads, bh = blockIdx.x % pairs;
  b = (int)(bh / (unsigned)a.kv_heads);
  hk = (int)(bh % (unsigned)a.kv_heads);
  return tiles - 1 - (int)(blockIdx.x / pairs);
}

// ---- forward
// The softmax needs some reference score per row, not the largest one: it moves only when a score exceeds it by more than 2^kLazy, which is
// rare after the first tiles, and the accumulators are rescaled only then.
template <class T, int DP, int NB, int WAVES>
__global__ __launch_bounds__(WAVES * 64, DP > 128 ? 1 : 2) void forward_kernel(AttnArgs a) {
  using El = Elem<T>;
  constexpr int BK = stream_rows<T, DP>(), S = lds_stride<T>(DP), ROWS = WAVES * NB * 16, KB = BK / 16, DB = DP / 16;
  __shared__ __attribute__((aligned(16))) T ks[2][BK * S], vs[2][BK * S];
  const int lane = threadIdx.x & 63, g = lane >> 4, wave = threadIdx.x >> 6;
  const int rows = a.q_len * a.group, tiles = (rows + ROWS - 1) / ROWS;
  int b, hk;
  const int t = place_of(a, tiles, b, hk);
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
  mk.start(row_of<T>(a.k, a.sk, b, kt, hk), a.sk.row, a.d);
  mv.start(row_of<T>(a.v, a.sv, b, kt, hk), a.sv.row, a.d);
  if (kt < k1) {
    mk.fetch(l.kn - kt);
    mv.fetch(l.kn - kt);
    mk.store(ks[0], S);
    mv.store(vs[0], S);
  }
  for (; kt < k1; kt += BK, buf ^= 1) {
    __syncthreads();                                          // this tile is there, and nobody reads the other buffer any more
    const bool more = kt + BK < k1;
    if (more) {
      mk.fetch(l.kn - kt - BK);
      mv.fetch(l.kn - kt - BK);
    }
    if (kt < w1 && kt + BK > w0) {
      floatx4 s[KB][NB];
#pragma unroll
      for (int y = 0; y < KB; ++y) {
#pragma unroll
        for (int c = 0; c < NB; ++c) s[y][c] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < DP / El::KF; ++k) {
          const typename El::Frag f = frag_rows(ks[buf], S, y * 16, k * El::KF);
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
        top[c] = over_groups_max(top[c]) * scale2;
        grows |= top[c] > m[c] + kLazy;
      }
      if (__any(grows)) {
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          const float next = fmaxf(m[c], top[c]);
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
          const typename El::Frag f = frag_cols<T, true>(vs[buf], S, y * 16, x * 16);
#pragma unroll
          for (int c = 0; c < NB; ++c) o[x][c] = El::mma(f, pf[c], o[x][c]);
        }
      }
    }
    if (more) {
      mk.store(ks[buf ^ 1], S);
      mv.store(vs[buf ^ 1], S);
    }
  }

#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const float total = over_groups_sum(sum[c]);
    if (r[c] >= rows) continue;
    const int i = query_of(a, r[c]), head = hk * a.group + r[c] - i * a.group;
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
template <class T, int DP, int NB, int WAVES>
__global__ __launch_bounds__(WAVES * 64, DP > 128 ? 1 : 2) void query_grad_kernel(AttnArgs a) {
  using El = Elem<T>;
  constexpr int BK = stream_rows<T, DP>(), S = lds_stride<T>(DP), ROWS = WAVES * NB * 16, DB = DP / 16, PB = El::PB;
  __shared__ __attribute__((aligned(16))) T ks[2][BK * S], vs[2][BK * S];
  const int lane = threadIdx.x & 63, g = lane >> 4, wave = threadIdx.x >> 6;
  const int rows = a.q_len * a.group, tiles = (rows + ROWS - 1) / ROWS;
  int b, hk;
  const int t = place_of(a, tiles, b, hk);
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
  mk.start(row_of<T>(a.k, a.sk, b, kt, hk), a.sk.row, a.d);
  mv.start(row_of<T>(a.v, a.sv, b, kt, hk), a.sv.row, a.d);
  if (kt < k1) {
    mk.fetch(l.kn - kt);
    mv.fetch(l.kn - kt);
    mk.store(ks[0], S);
    mv.store(vs[0], S);
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
      const typename El::Frag f = __builtin_bit_cast(typename El::Frag, any ? load16(o + from, a.d - from) : u32x4{0, 0, 0, 0});
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
        const typename El::Frag kf = frag_rows(ks[buf], S, (y + u) * 16, k * El::KF), vf = frag_rows(vs[buf], S, (y + u) * 16, k * El::KF);
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
            p[u][c][e] = j >= lo[c] && j < hi[c] ? p[u][c][e] : 0.f;
          }
    }
  };
  if (sizeof(T) == 2 && kt < k1 && k1 - kt <= BK) {
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
    if (g == 0 && r[c] < rows) a.delta[((int64_t)b * a.heads + head[c]) * a.q_len + qi[c]] = delta[c];

  floatx4 dq[DB][NB];
#pragma unroll
  for (int x = 0; x < DB; ++x)
#pragma unroll
    for (int c = 0; c < NB; ++c) dq[x][c] = floatx4{0.f, 0.f, 0.f, 0.f};
  for (; kt < k1; kt += BK, buf ^= 1) {
    __syncthreads();
    const bool more = kt + BK < k1;
    if (more) {
      mk.fetch(l.kn - kt - BK);
      mv.fetch(l.kn - kt - BK);
    }
    if (kt < w1 && kt + BK > w0) {
      const bool partial = kt < all0 || kt + BK > all1;
#pragma unroll
      for (int y = 0; y < BK / 16; y += PB) {
        floatx4 p[PB][NB], dp[PB][NB];
        weights(y, p, dp, partial);
        typename El::Frag f[NB];
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          floatx4 ds[PB];
#pragma unroll
          for (int u = 0; u < PB; ++u) ds[u] = p[u][c] * (dp[u][c] - delta[c]);
          f[c] = pack<T>(ds);
        }
#pragma unroll
        for (int x = 0; x < DB; ++x) {
          const typename El::Frag kf = frag_cols<T, true>(ks[buf], S, y * 16, x * 16);
#pragma unroll
          for (int c = 0; c < NB; ++c) dq[x][c] = El::mma(kf, f[c], dq[x][c]);
        }
      }
    }
    if (more) {
      mk.store(ks[buf ^ 1], S);
      mv.store(vs[buf ^ 1], S);
    }
  }
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    if (r[c] >= rows) continue;
    T* row = dense_row<T>(a, a.dq, a.q_len, a.heads, b, qi[c], head[c]);
    const bool any = hi[c] > lo[c];
#pragma unroll
    for (int x = 0; x < DB; ++x) store4(row, x * 16 + 4 * g, a.d, any ? dq[x][c] * a.scale : floatx4{0.f, 0.f, 0.f, 0.f});
  }
}

// Rows (query, head) of one list and key head on their way into LDS.  A tile holds whole queries where the heads that share a key
// head divide it: then a thread's pieces keep their heads and advance by a tile's queries.  Other numbers of heads take a division a piece.
template <class T, int BQ, int DP, int THREADS>
struct RowMove {
  static constexpr int E = Elem<T>::E, PER_ROW = DP / E, NP = BQ * PER_ROW / THREADS, APART = THREADS / PER_ROW;
  u32x4 r[NP];
  __device__ inline void fetch(const AttnArgs& a, const void* base, const Strides& st, int b, int hk, int rt, int r1) {
    const int t = (int)threadIdx.x, c = t % PER_ROW * E, count = a.d - c;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int row = rt + t / PER_ROW + i * APART;
      r[i] = u32x4{0, 0, 0, 0};
      if (count > 0 && row < r1) {
        const int q = a.group_shift >= 0 ? row >> a.group_shift : query_of(a, row);
        r[i] = load16(row_of<T>(base, st, b, q, hk * a.group + row - q * a.group) + c, count);
      }
    }
  }
  __device__ inline void store(T* tile, int lds_row) const {
    T* to = tile + (int)threadIdx.x / PER_ROW * lds_row + (int)threadIdx.x % PER_ROW * E;
#pragma unroll
    for (int i = 0; i < NP; ++i) *reinterpret_cast<u32x4*>(to + i * APART * lds_row) = r[i];
  }
};

// dk, dv: keys and values in registers, queries and dout stream
template <class T, int DP, int NB, int WAVES, int BQ, int OCC>
__global__ __launch_bounds__(WAVES * 64, OCC) void key_grad_kernel(AttnArgs a) {
  using El = Elem<T>;
  constexpr int S = lds_stride<T>(DP), KEYS = WAVES * NB * 16, DB = DP / 16, PB = El::PB;
  __shared__ __attribute__((aligned(16))) T qs[2][BQ * S], gs[2][BQ * S];
  __shared__ __attribute__((aligned(16))) float lses[2][BQ], deltas[2][BQ];
  __shared__ int los[2][BQ], his[2][BQ];
  const int lane = threadIdx.x & 63, g = lane >> 4, wave = threadIdx.x >> 6;
  const int tiles = (a.k_len + KEYS - 1) / KEYS;
  int b, hk;
  const int t = tiles - 1 - place_of(a, tiles, b, hk);        // with `causal` the first keys are seen by the most queries
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

  RowMove<T, BQ, DP, WAVES * 64> mq, md;
  float ml = 0.f, mt = 0.f;
  int mlo = 0, mhi = 0;
  const int r1 = q1 * a.group;
  auto fetch = [&](int rt) {
    mq.fetch(a, a.q, a.sq, b, hk, rt, r1);
    md.fetch(a, a.dout, a.sdo, b, hk, rt, r1);
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
    mq.store(qs[buf], S);
    md.store(gs[buf], S);
    if ((int)threadIdx.x < BQ) { lses[buf][threadIdx.x] = ml; deltas[buf][threadIdx.x] = mt; los[buf][threadIdx.x] = mlo; his[buf][threadIdx.x] = mhi; }
  };
  int rt = q0 * a.group, buf = 0;
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
      floatx4 s[PB][NB], dp[PB][NB];
#pragma unroll
      for (int u = 0; u < PB; ++u) {
#pragma unroll
        for (int c = 0; c < NB; ++c) s[u][c] = dp[u][c] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < DP / El::KF; ++k) {
          const typename El::Frag qf = frag_rows(qt, S, (y + u) * 16, k * El::KF), df = frag_rows(gt, S, (y + u) * 16, k * El::KF);
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
              p = j >= los[buf][at + e] && j < his[buf][at + e] ? p : 0.f;
            }
            s[u][c][e] = p;
            float ds = p * (dp[u][c][e] - dl[e]);
            if constexpr (kShift<T> != 0.f) ds *= kUnshift<T>;
            dp[u][c][e] = ds;
          }
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
        const typename El::Frag df = frag_cols<T, true>(gt, S, y * 16, x * 16), qf = frag_cols<T, true>(qt, S, y * 16, x * 16);
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
    T* krow = dense_row<T>(a, a.dk, a.k_len, a.kv_heads, b, j, hk);
    T* vrow = dense_row<T>(a, a.dv, a.k_len, a.kv_heads, b, j, hk);
#pragma unroll
    for (int x = 0; x < DB; ++x) {
      store4(krow, x * 16 + 4 * g, a.d, dk[x][c] * a.scale);
      store4(vrow, x * 16 + 4 * g, a.d, kShift<T> != 0.f ? dv[x][c] * kUnshift<T> : dv[x][c]);
    }
  }
}

template <class T, int DP>
hipError_t forward(const AttnArgs& a, hipStream_t s) {
  constexpr int NB = sizeof(T) == 4 || DP > 128 ? 1 : 2;
  const int64_t tiles = ((int64_t)a.q_len * a.group + 64 * NB - 1) / (64 * NB);
  return launch(forward_kernel<T, DP, NB, 4>, tiles * a.lists * a.kv_heads, 256, s, a);
}

template <class T, int DP>
hipError_t backward(const AttnArgs& a, hipStream_t s) {
  constexpr int NB = sizeof(T) == 4 || DP > 128 ? 1 : 2, BQ = stream_rows<T, DP>();
  const int64_t qt = ((int64_t)a.q_len * a.group + 64 * NB - 1) / (64 * NB), kt = ((int64_t)a.k_len + 64 * NB - 1) / (64 * NB);
  hipError_t e = hipSuccess;
  if (qt) e = launch(query_grad_kernel<T, DP, NB, 4>, qt * a.lists * a.kv_heads, 256, s, a);
  if (e == hipSuccess && kt) e = launch(key_grad_kernel<T, DP, NB, 4, BQ, 1>, kt * a.lists * a.kv_heads, 256, s, a);
  return e;
}

template <class T>
hipError_t forward_of(const AttnArgs& a, hipStream_t s) {
  return a.d <= 64 ? forward<T, 64>(a, s) : a.d <= 128 ? forward<T, 128>(a, s) : forward<T, 256>(a, s);
}
template <class T>
hipError_t backward_of(const AttnArgs& a, hipStream_t s) {
  return a.d <= 64 ? backward<T, 64>(a, s) : a.d <= 128 ? backward<T, 128>(a, s) : backward<T, 256>(a, s);
}

}  // namespace attn
}  // namespace stgn
