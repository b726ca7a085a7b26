// Attention of lists with few queries, and its gradients: up to eight rows (queries times the heads that share a key head).
//
// Nothing here is worth a matrix instruction: every key and value is read once, meets a handful of rows, and in the gradient dk
// and dv are written once.  Bytes bound it.  L lanes hold one key (16 bytes each), so a wave has 64 / L keys at a time, U times
// over to keep loads in flight; the rows' parts lie in registers.  Every lane group keeps a softmax of its own (maximum, sum,
// weighted values) and they are joined once, at the end of the list.
//
// Short lists: a wave a list and key head.  Long ones (WIDE): four waves take turns at one list's keys and the list is cut
// into `splits` runs of `per` keys where the lists alone do not fill the chip; the runs' softmaxes are joined by a second launch
// in the order of the runs.
#pragma once
#include "attention.h"

namespace stgn {
namespace attn {

template <int CTRL>
__device__ inline float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}

// sum over groups of L neighbouring lanes, in all of them
template <int L>
__device__ inline float lanes_sum(float x) {
  if constexpr (L >= 2) x += dpp<0xB1>(x);                    // quad_perm 1 0 3 2
  if constexpr (L >= 4) x += dpp<0x4E>(x);                    // quad_perm 2 3 0 1
  if constexpr (L >= 8) x += dpp<0x141>(x);                   // row_half_mirror
  if constexpr (L >= 16) x += dpp<0x140>(x);                  // row_mirror
  if constexpr (L >= 32) x += __shfl_xor(x, 16);
  if constexpr (L >= 64) x += __shfl_xor(x, 32);
  return x;
}

template <class T>
__device__ inline void spread(const u32x4& v, float (&f)[Elem<T>::E]) {
  if constexpr (sizeof(T) == 4) {
    const floatx4 x = __builtin_bit_cast(floatx4, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = x[j];
  } else {
    const typename Elem<T>::Frag x = __builtin_bit_cast(typename Elem<T>::Frag, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (float)x[j];
  }
}

template <int E>
__device__ inline float dot(const float (&x)[E], const float (&y)[E]) {
  float s = x[0] * y[0];
#pragma unroll
  for (int j = 1; j < E; ++j) s = fmaf(x[j], y[j], s);
  return s;
}

template <class T>
__device__ inline void store_piece(T* p, const float (&f)[Elem<T>::E], int count) {
  constexpr int E = Elem<T>::E;
  union { T e[E]; u32x4 v; } u;
#pragma unroll
  for (int j = 0; j < E; ++j) u.e[j] = (T)f[j];
  if (count >= E) {
    *reinterpret_cast<u32x4_any*>(p) = u.v;
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < E - 1; ++j)
      if (j < count) p[j] = u.e[j];
  } else {                                                    // halves and quarters (bf16 500 lists of 2,000, 4 heads of 101: 1,174 -> 1,097 us; fp32 loses by it)
    union { u32x4 v; T e[E]; } w = {u.v};
    if (count & 4) {
      *reinterpret_cast<u32x2_any*>(p) = u32x2_any{w.v[0], w.v[1]};
      p += 4;
      w.v[0] = w.v[2];
      w.v[1] = w.v[3];
    }
    if (count & 2) {
      *reinterpret_cast<u32_any*>(p) = w.v[0];
      p += 2;
      w.v[0] = w.v[1];
    }
    if (count & 1) *p = w.e[0];
  }
}

struct RowPlan { int splits, per; };                          // runs a list, keys a run

// A row's softmax over some of its keys: reference score (in powers of two), sum of weights, weighted values (one piece of 16
// bytes' numbers a lane)
template <int E>
struct Softmax {
  float m, sum, o[E];
  __device__ inline void clear() {
    m = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < E; ++j) o[j] = 0.f;
  }
  __device__ inline void join(float m2, float sum2, const float (&o2)[E]) {
    const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
    const float x = __builtin_amdgcn_exp2f(m - ref), y = __builtin_amdgcn_exp2f(m2 - ref);
    m = top;
    sum = sum * x + sum2 * y;
#pragma unroll
    for (int j = 0; j < E; ++j) o[j] = o[j] * x + o2[j] * y;
  }
  // ... with the lane groups `step` lanes away
  __device__ inline void join_lanes(int step) {
    float o2[E];
#pragma unroll
    for (int j = 0; j < E; ++j) o2[j] = __shfl_xor(o[j], step);
    const float m2 = __shfl_xor(m, step), s2 = __shfl_xor(sum, step);
    join(m2, s2, o2);
  }
};

template <class T, int E>
__device__ inline void write_row(const AttnArgs& a, int b, int i, int head, const Softmax<E>& x, int at, bool any) {
  float f[E];
  const float inv = any ? 1.f / x.sum : 0.f;
#pragma unroll
  for (int j = 0; j < E; ++j) f[j] = any ? x.o[j] * inv : 0.f;
  if (at < a.d) store_piece(const_cast<T*>(row_of<T>(a.o, a.so, b, i, head)) + at, f, a.d - at);
  if (at == 0) a.lse[((int64_t)b * a.heads + head) * a.q_len + i] = any ? (x.m + __builtin_amdgcn_logf(x.sum)) * kLn2 : -INFINITY;
}

template <class T, int L, int R, int U, bool WIDE>
__global__ __launch_bounds__(256) void rows_forward_kernel(AttnArgs a, RowPlan plan, float* part) {
  constexpr int E = Elem<T>::E, G = 64 / L, STEP = G * U;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), slot = lane / L, at = lane % L * E;
  const int64_t unit = WIDE ? (int64_t)(blockIdx.x / (unsigned)plan.splits) : (int64_t)blockIdx.x * 4 + wave;
  const int split = WIDE ? (int)(blockIdx.x % (unsigned)plan.splits) : 0;
  if (unit >= (int64_t)a.lists * a.kv_heads) return;
  const int b = (int)(unit / a.kv_heads), hk = (int)(unit % a.kv_heads), rows = a.q_len * a.group;
  const List l = list_of(a, b);

  int lo[R], hi[R], k0 = a.k_len, k1 = 0, all0 = 0, all1 = a.k_len;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    lo[r] = hi[r] = 0;
    if (r < rows) seen(a, l, query_of(a, r), lo[r], hi[r]);
    if (hi[r] > lo[r]) {
      k0 = min(k0, lo[r]);
      k1 = max(k1, hi[r]);
    }
    all0 = max(all0, lo[r]);
    all1 = min(all1, hi[r]);
  }
  if (WIDE) {
    k0 = max(k0, split * plan.per);
    k1 = min(k1, (split + 1) * plan.per);
  }
  const float scale2 = a.scale * kLog2e;
  const RowEnd end = row_end<T>(a.d);
  const int early = end == kWide && at < a.d ? max(E - (a.d - at), 0) : 0;                 // elements in front of the head's last part that its piece holds
  const T* kp = row_of<T>(a.k, a.sk, b, 0, hk) + at - early;
  const T* vp = row_of<T>(a.v, a.sv, b, 0, hk) + at - early;
  u32x4 kr[U], vr[U];
  auto fetch = [&](int base) {
    auto each = [&](auto load) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int j = base + u * G + slot;
        kr[u] = vr[u] = u32x4{0, 0, 0, 0};
        if (j < k1 && at < a.d) {
          kr[u] = load(kp + (int64_t)j * a.sk.row);
          vr[u] = load(vp + (int64_t)j * a.sv.row);
        }
      }
    };
    if (end != kShort) each([](const T* p) { return *reinterpret_cast<const u32x4_any*>(p); });
    else each([&](const T* p) { return load16<T, kShort>(p, a.d - at); });
  };
  int base = k0 + (WIDE ? wave * STEP : 0);
  if (base < k1) fetch(base);                                 // (with the rows on their way too: one wait for a short list)

  float q[R][E];
  Softmax<E> x[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int i = query_of(a, r);
    u32x4 raw = {0, 0, 0, 0};
    if (r < rows && i < l.qn && at < a.d) raw = load16(row_of<T>(a.q, a.sq, b, i, hk * a.group + r - i * a.group) + at, a.d - at, end);
    spread<T>(raw, q[r]);
    x[r].clear();
  }

  while (base < k1) {
    if (end == kWide)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        kr[u] = moved_down<T>(kr[u], early * (int)sizeof(T));
        vr[u] = moved_down<T>(vr[u], early * (int)sizeof(T));
      }
    const bool partial = base < all0 || base + STEP > min(all1, k1);
    float s[R][U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!WIDE && base + u * G >= k1) {                      // (the same for all lanes)
#pragma unroll
        for (int r = 0; r < R; ++r) s[r][u] = -INFINITY;
        continue;
      }
      float f[E];
      spread<T>(kr[u], f);
      const int j = base + u * G + slot;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        s[r][u] = lanes_sum<L>(dot(q[r], f)) * scale2;
        if (partial) s[r][u] = j >= lo[r] && j < min(hi[r], k1) ? s[r][u] : -INFINITY;
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float top = x[r].m;
#pragma unroll
      for (int u = 0; u < U; ++u) top = fmaxf(top, s[r][u]);
      const float ref = top == -INFINITY ? 0.f : top, shrink = __builtin_amdgcn_exp2f(x[r].m - ref);
      x[r].m = top;
      x[r].sum *= shrink;
#pragma unroll
      for (int j = 0; j < E; ++j) x[r].o[j] *= shrink;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        s[r][u] = __builtin_amdgcn_exp2f(s[r][u] - ref);
        x[r].sum += s[r][u];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!WIDE && base + u * G >= k1) continue;
      float f[E];
      spread<T>(vr[u], f);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < E; ++j) x[r].o[j] = fmaf(s[r][u], f[j], x[r].o[j]);
    }
    base += WIDE ? 4 * STEP : STEP;
    if (base < k1) fetch(base);
  }

#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int step = L; step < 64; step *= 2) x[r].join_lanes(step);

  if constexpr (!WIDE) {
    if (slot == 0)
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (r < rows) write_row<T, E>(a, b, query_of(a, r), hk * a.group + r - query_of(a, r) * a.group, x[r], at, hi[r] > lo[r]);
  } else {
    __shared__ float ms[4][R], sums[4][R], os[4][R][L * E];
    if (slot == 0)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (lane == 0) { ms[wave][r] = x[r].m; sums[wave][r] = x[r].sum; }
#pragma unroll
        for (int j = 0; j < E; ++j) os[wave][r][at + j] = x[r].o[j];
      }
    __syncthreads();
    if (slot != 0) return;
    for (int r = wave; r < rows; r += 4) {
      Softmax<E> y;
      y.clear();
      for (int w = 0; w < 4; ++w) {
        float o2[E];
#pragma unroll
        for (int j = 0; j < E; ++j) o2[j] = os[w][r][at + j];
        y.join(ms[w][r], sums[w][r], o2);
      }
      const int i = query_of(a, r), head = hk * a.group + r - i * a.group;
      if (plan.splits == 1) {
        int l0, h0;
        seen(a, l, i, l0, h0);
        write_row<T, E>(a, b, i, head, y, at, h0 > l0);
      } else {
        float* p = part + ((unit * plan.splits + split) * rows + r) * (int64_t)(a.d + 2);
#pragma unroll
        for (int j = 0; j < E; ++j)
          if (at + j < a.d) p[2 + at + j] = y.o[j];
        if (at == 0) { p[0] = y.m; p[1] = y.sum; }
      }
    }
  }
}

// Gradients: one pass over the keys; each is written back as dk and dv, and dq adds up in the lane groups.
template <class T, int L, int R, int U, bool WIDE>
__global__ __launch_bounds__(256) void rows_grad_kernel(AttnArgs a, RowPlan plan, float* part) {
  constexpr int E = Elem<T>::E, G = 64 / L, STEP = G * U;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), slot = lane / L, at = lane % L * E;
  const int64_t unit = WIDE ? (int64_t)(blockIdx.x / (unsigned)plan.splits) : (int64_t)blockIdx.x * 4 + wave;
  const int split = WIDE ? (int)(blockIdx.x % (unsigned)plan.splits) : 0;
  if (unit >= (int64_t)a.lists * a.kv_heads) return;
  const int b = (int)(unit / a.kv_heads), hk = (int)(unit % a.kv_heads), rows = a.q_len * a.group;
  const List l = list_of(a, b);

  int lo[R], hi[R], k0 = a.k_len, k1 = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    lo[r] = hi[r] = 0;
    if (r < rows) seen(a, l, query_of(a, r), lo[r], hi[r]);
    if (hi[r] > lo[r]) {
      k0 = min(k0, lo[r]);
      k1 = max(k1, hi[r]);
    }
  }
  const int first = WIDE ? split * plan.per : 0, last = WIDE ? min(a.k_len, (split + 1) * plan.per) : a.k_len;
  k1 = min(k1, last);                                         // (the next run's keys: zeros here, which add nothing to dq)
  const RowEnd end = row_end<T>(a.d);
  const int early = end == kWide && at < a.d ? max(E - (a.d - at), 0) : 0;                 // elements in front of the head's last part that its piece holds
  const T* kp = row_of<T>(a.k, a.sk, b, 0, hk) + at - early;
  const T* vp = row_of<T>(a.v, a.sv, b, 0, hk) + at - early;
  u32x4 kr[U], vr[U];
  auto fetch = [&](int base) {
    auto each = [&](auto load) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int j = base + u * G + slot;
        kr[u] = vr[u] = u32x4{0, 0, 0, 0};
        if (j >= k0 && j < k1 && at < a.d) {
          kr[u] = load(kp + (int64_t)j * a.sk.row);
          vr[u] = load(vp + (int64_t)j * a.sv.row);
        }
      }
    };
    if (end != kShort) each([](const T* p) { return *reinterpret_cast<const u32x4_any*>(p); });
    else each([&](const T* p) { return load16<T, kShort>(p, a.d - at); });
  };
  int base = first + (WIDE ? wave * STEP : 0);
  if (base < last) fetch(base);                               // (with the rows on their way too: one wait for a short list)

  float q[R][E], go[R][E], dq[R][E], lse2[R], delta[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int i = query_of(a, r), head = hk * a.group + r - i * a.group;
    u32x4 rq = {0, 0, 0, 0}, rd = rq, ro = rq;
    lse2[r] = INFINITY;                                       // a row that sees nothing has no probability
    if (hi[r] > lo[r]) {
      lse2[r] = a.lse[((int64_t)b * a.heads + head) * a.q_len + i] * kLog2e;
      if (at < a.d) {
        rq = load16(row_of<T>(a.q, a.sq, b, i, head) + at, a.d - at, end);
        rd = load16(row_of<T>(a.dout, a.sdo, b, i, head) + at, a.d - at, end);
        ro = load16(row_of<T>(a.out, a.so, b, i, head) + at, a.d - at, end);
      }
    }
    float o[E];
    spread<T>(rq, q[r]);
    spread<T>(rd, go[r]);
    spread<T>(ro, o);
    delta[r] = lanes_sum<L>(dot(go[r], o));
#pragma unroll
    for (int j = 0; j < E; ++j) dq[r][j] = 0.f;
  }
  const float scale2 = a.scale * kLog2e;
  const int64_t out_row = (int64_t)a.kv_heads * a.d, out0 = ((int64_t)b * a.k_len * a.kv_heads + hk) * a.d + at;
  T *dk = static_cast<T*>(a.dk) + out0, *dv = static_cast<T*>(a.dv) + out0;

  while (base < last) {
    if (end == kWide)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        kr[u] = moved_down<T>(kr[u], early * (int)sizeof(T));
        vr[u] = moved_down<T>(vr[u], early * (int)sizeof(T));
      }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = base + u * G + slot;
      if (base + u * G >= last) continue;                     // (the same for all lanes)
      float k[E], v[E], gk[E], gv[E];
      spread<T>(kr[u], k);
      spread<T>(vr[u], v);
#pragma unroll
      for (int e = 0; e < E; ++e) gk[e] = gv[e] = 0.f;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const bool sees = j >= lo[r] && j < hi[r];
        const float s = lanes_sum<L>(dot(q[r], k)), dp = lanes_sum<L>(dot(go[r], v));
        const float p = sees ? __builtin_amdgcn_exp2f(fmaf(s, scale2, -lse2[r])) : 0.f;
        const float ds = sees ? p * (dp - delta[r]) * a.scale : 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          gk[e] = fmaf(ds, q[r][e], gk[e]);
          gv[e] = fmaf(p, go[r][e], gv[e]);
          dq[r][e] = fmaf(ds, k[e], dq[r][e]);
        }
      }
      if (j < last && at < a.d) {
        store_piece(dk + (int64_t)j * out_row, gk, a.d - at);
        store_piece(dv + (int64_t)j * out_row, gv, a.d - at);
      }
    }
    base += WIDE ? 4 * STEP : STEP;
    if (base < last) fetch(base);
  }

#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < E; ++j)
#pragma unroll
      for (int step = L; step < 64; step *= 2) dq[r][j] += __shfl_xor(dq[r][j], step);

  if constexpr (!WIDE) {
    if (slot == 0 && at < a.d)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int i = query_of(a, r), head = hk * a.group + r - i * a.group;
        if (r < rows) store_piece(dense_row<T>(a, a.dq, a.q_len, a.heads, b, i, head) + at, dq[r], a.d - at);
      }
  } else {
    __shared__ float dqs[4][R][L * E];
    if (slot == 0)
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < E; ++j) dqs[wave][r][at + j] = dq[r][j];
    __syncthreads();
    if (slot != 0 || at >= a.d) return;
    for (int r = wave; r < rows; r += 4) {
      float f[E];
#pragma unroll
      for (int j = 0; j < E; ++j) f[j] = (dqs[0][r][at + j] + dqs[1][r][at + j]) + (dqs[2][r][at + j] + dqs[3][r][at + j]);
      const int i = query_of(a, r), head = hk * a.group + r - i * a.group;
      if (plan.splits == 1) {
        store_piece(dense_row<T>(a, a.dq, a.q_len, a.heads, b, i, head) + at, f, a.d - at);
      } else {
        float* p = part + ((unit * plan.splits + split) * rows + r) * (int64_t)a.d + at;
#pragma unroll
        for (int j = 0; j < E; ++j)
          if (at + j < a.d) p[j] = f[j];
      }
    }
  }
}

// Rows a list and key head that go this way: eight; four in the gradient of 16-bit types, whose lanes hold twice the numbers
// (q, dout and dq of eight rows would be 192 registers).
inline int most_rows(bool grad, bool narrow) { return grad && narrow ? 4 : 8; }

// A wave a list up to 128 keys.  Longer lists get a workgroup each, and are cut into runs of at least 256 keys, 64 a list at most (joining
// 256 took as long as the runs), until there are 2,048 workgroups, eight a CU.
inline bool wide_rows(const AttnArgs& a) { return a.k_len > 128; }
inline RowPlan row_plan(const AttnArgs& a) {
  const int64_t units = (int64_t)a.lists * a.kv_heads;
  int64_t splits = wide_rows(a) && units ? (2048 + units - 1) / units : 1;
  const int64_t most = (a.k_len + 255) / 256;
  if (splits > most) splits = most;
  if (splits > 64) splits = 64;
  if (splits < 1) splits = 1;
  RowPlan p;
  p.per = (int)((a.k_len + splits - 1) / splits);
  if (p.per < 1) p.per = 1;
  p.splits = a.k_len ? (a.k_len + p.per - 1) / p.per : 1;
  return p;
}
inline size_t row_part_bytes(const AttnArgs& a, bool grad) {
  const RowPlan p = row_plan(a);
  return p.splits > 1 ? (size_t)a.lists * a.kv_heads * p.splits * a.q_len * a.group * (a.d + (grad ? 0 : 2)) * sizeof(float) : 0;
}

template <class T, int L, int R, bool GRAD>
hipError_t rows_launch(const AttnArgs& a, float* part, hipStream_t s) {
  constexpr int U = R >= 8 ? 2 : 4;                           // (more rows, fewer registers for keys in flight)
  // short fp32 lists' gradients: eight, all keys of most lists at once (40,000 lists of twenty, heads of 50: 318 -> 300 us; the forward call
  // loses a sixth by it)
  constexpr int US = GRAD && R == 1 && sizeof(T) == 4 ? 8 : U;
  const RowPlan p = row_plan(a);
  const int64_t units = (int64_t)a.lists * a.kv_heads, rows = (int64_t)a.q_len * a.group;
  hipError_t e;
  if constexpr (GRAD)
    e = wide_rows(a) ? launch(rows_grad_kernel<T, L, R, U, true>, units * p.splits, 256, s, a, p, part)
                     : launch(rows_grad_kernel<T, L, R, US, false>, (units + 3) / 4, 256, s, a, p, part);
  else
    e = wide_rows(a) ? launch(rows_forward_kernel<T, L, R, U, true>, units * p.splits, 256, s, a, p, part)
                     : launch(rows_forward_kernel<T, L, R, US, false>, (units + 3) / 4, 256, s, a, p, part);
  if (e != hipSuccess || p.splits == 1 || rows == 0) return e;      // (no queries: dk and dv are zeros, and there is no dq to add up)
  if constexpr (GRAD) return sum_runs<T>(a, a.dq, nullptr, a.q_len, a.group, p.splits, part, s);
  else return launch(join_kernel<T>, join_grid(units * rows, p.splits), 256, s, a, p.splits, (const float*)part);
}

template <class T, int L, bool GRAD>
hipError_t rows_by_count(const AttnArgs& a, float* part, hipStream_t s) {
  const int rows = a.q_len * a.group;
  return rows <= 1   ? rows_launch<T, L, 1, GRAD>(a, part, s)
         : rows <= 2 ? rows_launch<T, L, 2, GRAD>(a, part, s)
         : rows <= 4 ? rows_launch<T, L, 4, GRAD>(a, part, s)
                     : rows_launch<T, L, GRAD && sizeof(T) == 2 ? 4 : 8, GRAD>(a, part, s);
}

// lanes a key: the power of two that covers the head by 16 bytes a lane, four at least
template <class T, bool GRAD>
hipError_t rows_of(const AttnArgs& a, float* part, hipStream_t s) {
  const int pieces = (a.d + Elem<T>::E - 1) / Elem<T>::E;
  if constexpr (sizeof(T) == 4)
    if (pieces > 32) return rows_by_count<T, 64, GRAD>(a, part, s);
  return pieces <= 4    ? rows_by_count<T, 4, GRAD>(a, part, s)
         : pieces <= 8  ? rows_by_count<T, 8, GRAD>(a, part, s)
         : pieces <= 16 ? rows_by_count<T, 16, GRAD>(a, part, s)
                        : rows_by_count<T, 32, GRAD>(a, part, s);
}

}  // namespace attn
}  // namespace stgn
