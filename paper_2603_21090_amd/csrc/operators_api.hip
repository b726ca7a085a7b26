// extern "C" boundary of the operators on the caller's tensors: argument checks and dispatch by element type.
#include <math.h>
#include <utility>

#include "attention_rows.h"
#include "linear_i8.h"
#include "operators.h"
#include "streamtgn.h"

namespace stgn {

#define STGN_PER_TYPE(T)                                                                  \
  size_t attention_bytes_##T(const AttnArgs& a);                                          \
  size_t attention_grad_bytes_##T(const AttnArgs& a);                                     \
  hipError_t attention_##T(const AttnArgs& a, void* ws, hipStream_t s);                   \
  hipError_t attention_grad_##T(const AttnArgs& a, void* ws, hipStream_t s);              \
  hipError_t attention_rows_##T(const AttnArgs& a, void* ws, hipStream_t s);              \
  hipError_t attention_rows_grad_##T(const AttnArgs& a, void* ws, hipStream_t s);         \
  size_t linear_bytes_##T(const LinearArgs& a);                                           \
  size_t linear_grad_bytes_##T(const LinearGradArgs& a);                                  \
  hipError_t linear_##T(const LinearArgs& a, void* ws, hipStream_t s);                    \
  hipError_t linear_grad_##T(const LinearGradArgs& a, void* ws, hipStream_t s);           \
  hipError_t rms_norm_##T(const NormArgs& a, hipStream_t s);                              \
  size_t rms_norm_grad_bytes_##T(const NormGradArgs& a);                                  \
  hipError_t rms_norm_grad_##T(const NormGradArgs& a, void* ws, hipStream_t s);           \
  hipError_t rows_in_8_##T(const NormArgs& a, hipStream_t s);                             \
  size_t columns_bytes_##T(const ColumnsArgs& a);                                         \
  hipError_t columns_in_8_##T(const ColumnsArgs& a, void* ws, hipStream_t s);             \
  hipError_t linear_i8_##T(const Linear8Args& a, void* ws, hipStream_t s);                \
  hipError_t dropout_##T(const DropoutArgs& a, hipStream_t s);
STGN_PER_TYPE(f32)
STGN_PER_TYPE(bf16)
STGN_PER_TYPE(f16)
#undef STGN_PER_TYPE

#define STGN_BY_TYPE(dtype, call, ...)                                                    \
  ((dtype) == STGN_F32 ? call##_f32(__VA_ARGS__) : (dtype) == STGN_BF16 ? call##_bf16(__VA_ARGS__) : call##_f16(__VA_ARGS__))

size_t linear_bytes(const LinearArgs& a, int dtype) { return STGN_BY_TYPE(dtype, linear_bytes, a); }
size_t linear_grad_bytes(const LinearGradArgs& a, int dtype) { return STGN_BY_TYPE(dtype, linear_grad_bytes, a); }
hipError_t launch_linear(const LinearArgs& a, int dtype, void* ws, hipStream_t s) { return STGN_BY_TYPE(dtype, linear, a, ws, s); }

bool few_rows(const AttnArgs& a, int dtype, bool grad) {
  return (int64_t)a.q_len * a.group <= attn::most_rows(grad, dtype != STGN_F32);
}

size_t attention_bytes(const AttnArgs& a, int dtype) {
  return few_rows(a, dtype, false) ? attn::row_part_bytes(a, false) : STGN_BY_TYPE(dtype, attention_bytes, a);
}
size_t attention_grad_bytes(const AttnArgs& a, int dtype) {
  return few_rows(a, dtype, true) ? attn::row_part_bytes(a, true) : STGN_BY_TYPE(dtype, attention_grad_bytes, a);
}

}  // namespace stgn

using namespace stgn;

namespace {

int no(const char* why) { return fail_operator(STGN_E_INVALID_ARG, why); }

size_t size_of(uint32_t dtype) { return dtype == STGN_F32 ? 4 : 2; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

struct Span { const char* a; size_t n; };
// `rows` rows of `width` elements, `ld` apart
Span span_of(const void* p, uint64_t rows, uint64_t width, uint64_t ld, size_t es) {
  return {static_cast<const char*>(p), p && rows && width ? ((rows - 1) * ld + width) * es : 0};
}
// Whether elements at these steps reach over more than the 2^48 bytes that a device address can tell apart: below that the spans' ends stay
// 64-bit numbers, and no overlap is missed.
bool too_far(uint64_t n0, uint64_t s0, uint64_t n1, uint64_t s1, uint64_t n2, uint64_t s2, uint64_t width, size_t es) {
  if (!n0 || !n1 || !n2) return false;
  const unsigned __int128 last = (unsigned __int128)(n0 - 1) * s0 + (unsigned __int128)(n1 - 1) * s1 + (unsigned __int128)(n2 - 1) * s2 + width;
  return last * es > (unsigned __int128)1 << 48;
}
bool meet(const Span& x, const Span& y) { return x.n && y.n && x.a < y.a + y.n && y.a < x.a + x.n; }
// rows of x and y, both `ld` bytes apart, whose columns lie side by side in one wider matrix
bool beside(const Span& x, size_t x_width, const Span& y, size_t y_width, size_t ld) {
  const size_t to_y = y.a >= x.a ? (size_t)(y.a - x.a) % ld : (ld - (size_t)(x.a - y.a) % ld) % ld;
  return to_y >= x_width && to_y + y_width <= ld;
}

int finish(hipError_t e) { return e == hipSuccess ? STGN_OK : fail_operator(STGN_E_DEVICE, hipGetErrorString(e)); }

int check_workspace(size_t need, const void* ws, size_t bytes) {
  if (need == 0) return STGN_OK;
  if (!ws || bytes < need || !aligned(ws, 256))
    return fail_operator(STGN_E_WORKSPACE, "workspace missing, too small or not aligned to 256 bytes");
  return STGN_OK;
}

constexpr uint64_t kMaxLen = 1u << 29;                        // sums of a position, a length and a window stay 32-bit numbers
constexpr uint64_t kMaxRows = 1u << 30, kMaxWidth = 1u << 24, kMaxLd = 1ull << 40;
constexpr uint64_t kMaxGroups = (1ull << 24) - 1;             // workgroups of 256 threads a launch may hold

int check_linear(const stgn_linear_args* a, bool grad, bool sizes_only) {
  if (!a) return no("NULL arguments");
  if (a->dtype > STGN_F16) return no("dtype must be STGN_F32, STGN_BF16 or STGN_F16");
  if (a->activation > STGN_ACT_SILU) return no("unknown activation");
  if (a->reserved) return no("reserved must be 0");
  if (a->rows > kMaxRows) return no("rows out of range");
  if (a->d_in == 0 || a->d_out == 0 || a->d_in > kMaxWidth || a->d_out > kMaxWidth) return no("d_in and d_out must lie in 1 .. 2^24");
  // every product's tiles of 64 x 64 (or its splits, at most 512 more) are one launch
  auto tiles = [](uint64_t m, uint64_t n) { return ((m + 63) / 64) * ((n + 63) / 64); };
  if (tiles(a->rows, a->d_out) > kMaxGroups - 512 || tiles(a->rows, a->d_in) > kMaxGroups - 512 || tiles(a->d_in, a->d_out) > kMaxGroups - 512)
    return no("the product has more tiles than a launch");
  if (sizes_only) return STGN_OK;
  const size_t es = size_of(a->dtype);
  const void* all[] = {a->x, a->w, a->bias, a->residual, a->y, a->pre, a->dy, a->dx, a->dw, a->db};
  for (const void* p : all)
    if (!aligned(p, es)) return no("a pointer is not aligned to its element");
  if (a->ld_x < a->d_in || a->ld_w < a->d_out || a->ld_x > kMaxLd || a->ld_w > kMaxLd) return no("ld_x or ld_w below the row's width");
  if (!a->w || (a->rows && !a->x)) return no("NULL x or w");
  const char* const far = "a matrix reaches over more than 2^48 bytes";
  const auto wide = [&](uint64_t rows, uint64_t ld, uint64_t width) { return too_far(rows, ld, 1, 0, 1, 0, width, es); };
  if (wide(a->rows, a->ld_x, a->d_in) || wide(a->d_in, a->ld_w, a->d_out)) return no(far);
  const Span x = span_of(a->x, a->rows, a->d_in, a->ld_x, es), w = span_of(a->w, a->d_in, a->d_out, a->ld_w, es);
  if (!grad) {
    if (a->rows && !a->y) return no("NULL y");
    if (a->ld_y < a->d_out || a->ld_y > kMaxLd) return no("ld_y below the row's width");
    if (a->residual && (a->ld_residual < a->d_out || a->ld_residual > kMaxLd)) return no("ld_residual below the row's width");
    if (a->pre && (a->ld_pre < a->d_out || a->ld_pre > kMaxLd)) return no("ld_pre below the row's width");
    if (wide(a->rows, a->ld_y, a->d_out) || (a->residual && wide(a->rows, a->ld_residual, a->d_out)) || (a->pre && wide(a->rows, a->ld_pre, a->d_out)))
      return no(far);
    const Span y = span_of(a->y, a->rows, a->d_out, a->ld_y, es), p = span_of(a->pre, a->rows, a->d_out, a->ld_pre, es),
               b = span_of(a->bias, 1, a->d_out, 0, es), r = span_of(a->residual, a->rows, a->d_out, a->ld_residual, es);
    const bool in_place = a->residual == a->y && a->ld_residual == a->ld_y;
    // (matrices of rows the same distance apart may be columns of one)
    const auto hit = [&](const Span& s, uint64_t sw, uint64_t sl, const Span& t, uint64_t tw, uint64_t tl) {
      return meet(s, t) && !(sl == tl && beside(s, sw * es, t, tw * es, sl * es));
    };
    const uint64_t in = a->d_in, n = a->d_out;
    if (hit(y, n, a->ld_y, x, in, a->ld_x) || hit(y, n, a->ld_y, p, n, a->ld_pre) || hit(p, n, a->ld_pre, x, in, a->ld_x) ||
        hit(p, n, a->ld_pre, r, n, a->ld_residual) || (!in_place && hit(y, n, a->ld_y, r, n, a->ld_residual)) || meet(y, w) || meet(y, b) || meet(p, w) || meet(p, b))
      return no("an output overlaps an input or the other output (y may be exactly the residual)");
    return STGN_OK;
  }
  if (a->rows && !a->dy) return no("NULL dy");
  if (a->ld_dy < a->d_out || a->ld_dy > kMaxLd) return no("ld_dy below the row's width");
  if (a->activation != STGN_ACT_NONE) {
    if (a->rows && !a->pre) return no("the gradient of an activation needs pre");
    if (a->ld_pre < a->d_out || a->ld_pre > kMaxLd) return no("ld_pre below the row's width");
  }
  if (wide(a->rows, a->ld_dy, a->d_out) || (a->activation != STGN_ACT_NONE && wide(a->rows, a->ld_pre, a->d_out))) return no(far);
  const Span in[] = {x, w, span_of(a->dy, a->rows, a->d_out, a->ld_dy, es),
                     span_of(a->activation != STGN_ACT_NONE ? a->pre : nullptr, a->rows, a->d_out, a->ld_pre, es)};
  const Span out[] = {span_of(a->dx, a->rows, a->d_in, a->d_in, es), span_of(a->dw, a->d_in, a->d_out, a->d_out, es),
                      span_of(a->db, 1, a->d_out, 0, es)};
  for (int i = 0; i < 3; ++i) {
    for (const Span& s : in)
      if (meet(out[i], s)) return no("a gradient overlaps an input");
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return no("two gradients overlap");
  }
  return STGN_OK;
}

LinearArgs linear_args(const stgn_linear_args* a) {
  LinearArgs l{};
  l.x = a->x; l.w = a->w; l.bias = a->bias; l.residual = a->residual; l.y = a->y; l.pre = a->pre;
  l.ld_x = (int64_t)a->ld_x; l.ld_w = (int64_t)a->ld_w; l.ld_res = (int64_t)a->ld_residual; l.ld_y = (int64_t)a->ld_y; l.ld_pre = (int64_t)a->ld_pre;
  l.rows = (int)a->rows; l.d_in = (int)a->d_in; l.d_out = (int)a->d_out; l.act = (int)a->activation;
  return l;
}

LinearGradArgs linear_grad_args(const stgn_linear_args* a) {
  LinearGradArgs l{};
  l.dy = a->dy; l.x = a->x; l.w = a->w; l.pre = a->pre; l.dx = a->dx; l.dw = a->dw; l.db = a->db;
  l.ld_dy = (int64_t)a->ld_dy; l.ld_x = (int64_t)a->ld_x; l.ld_w = (int64_t)a->ld_w; l.ld_pre = (int64_t)a->ld_pre;
  l.rows = (int)a->rows; l.d_in = (int)a->d_in; l.d_out = (int)a->d_out; l.act = (int)a->activation;
  return l;
}

// whether the rows of d numbers at these strides lie clear of each other: each stride reaches over all that smaller ones span
bool apart(uint64_t n0, uint64_t s0, uint64_t n1, uint64_t s1, uint64_t n2, uint64_t s2, uint64_t d) {
  uint64_t n[3] = {n0, n1, n2}, s[3] = {s0, s1, s2}, span = d;
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < 2; ++j)
      if (s[j] > s[j + 1]) { std::swap(s[j], s[j + 1]); std::swap(n[j], n[j + 1]); }
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    if (s[i] < span) return false;
    span += (n[i] - 1) * s[i];
  }
  return true;
}

int check_attention(const stgn_attention_args* a, bool grad, bool sizes_only) {
  if (!a) return no("NULL arguments");
  if (a->dtype > STGN_F16) return no("dtype must be STGN_F32, STGN_BF16 or STGN_F16");
  if (a->d_head == 0 || a->d_head > 256) return no("d_head must lie in 1 .. 256");
  if (a->heads == 0 || a->kv_heads == 0 || a->heads % a->kv_heads) return no("kv_heads must divide heads");
  if (a->heads > 65535) return no("heads out of range");
  if (a->causal > 1) return no("causal must be 0 or 1");
  if (a->window && !a->causal) return no("a window needs causal = 1");
  if (a->lists > kMaxRows || a->q_len > kMaxLen || a->k_len > kMaxLen) return no("lists, q_len or k_len out of range");
  const uint64_t rows = (uint64_t)a->q_len * (a->heads / a->kv_heads);
  if (rows > kMaxRows) return no("q_len times the heads that share a key head out of range");
  const uint64_t pairs = (uint64_t)a->lists * a->kv_heads;
  if (pairs > kMaxGroups / 2 || ((rows + 63) / 64) * pairs > kMaxGroups / 2 || (((uint64_t)a->k_len + 63) / 64) * pairs > kMaxGroups / 2)   // (of up to 512 threads)
    return no("the lists have more tiles than a launch");
  if (sizes_only) return STGN_OK;
  if (!(a->scale == a->scale) || a->scale - a->scale != 0.0f) return no("scale must be finite");
  const size_t es = size_of(a->dtype);
  const void* all[] = {a->q, a->k, a->v, a->out, a->dout, a->dq, a->dk, a->dv};
  for (const void* p : all)
    if (!aligned(p, es)) return no("a pointer is not aligned to its element");
  if (!aligned(a->lse, 4) || !aligned(a->q_lens, 4) || !aligned(a->k_lens, 4)) return no("a pointer is not aligned to its element");
  const uint64_t strides[] = {a->q_list, a->q_row, a->q_head, a->k_list, a->k_row, a->k_head, a->v_list, a->v_row, a->v_head, a->out_list, a->out_row, a->out_head};
  for (uint64_t s : strides)
    if (s > kMaxLd) return no("a stride is out of range");
  const bool have_q = a->lists && a->q_len, have_k = a->lists && a->k_len;
  if (have_q && (!a->q || !a->out || !a->lse)) return no("NULL q, out or lse");
  if (have_k && (!a->k || !a->v)) return no("NULL k or v");
  const auto beyond = [&](uint64_t len, uint64_t heads, uint64_t sl, uint64_t sr, uint64_t sh) {
    return too_far(a->lists, sl, len, sr, heads, sh, a->d_head, es);
  };
  const char* const far = "a tensor reaches over more than 2^48 bytes";
  if (beyond(a->q_len, a->heads, a->q_list, a->q_row, a->q_head) || beyond(a->k_len, a->kv_heads, a->k_list, a->k_row, a->k_head) ||
      beyond(a->k_len, a->kv_heads, a->v_list, a->v_row, a->v_head) || beyond(a->q_len, a->heads, a->out_list, a->out_row, a->out_head))
    return no(far);
  auto reach = [&](const void* p, uint64_t len, uint64_t heads, uint64_t sl, uint64_t sr, uint64_t sh) {
    Span s{static_cast<const char*>(p), 0};
    if (p && a->lists && len) s.n = ((a->lists - 1) * sl + (len - 1) * sr + (heads - 1) * sh + a->d_head) * es;
    return s;
  };
  const uint64_t nq = (uint64_t)a->lists * a->q_len * a->heads, nk = (uint64_t)a->lists * a->k_len * a->kv_heads;
  const Span q = reach(a->q, a->q_len, a->heads, a->q_list, a->q_row, a->q_head), k = reach(a->k, a->k_len, a->kv_heads, a->k_list, a->k_row, a->k_head),
             v = reach(a->v, a->k_len, a->kv_heads, a->v_list, a->v_row, a->v_head);
  const Span o = reach(a->out, a->q_len, a->heads, a->out_list, a->out_row, a->out_head), lse = span_of(a->lse, 1, nq, 0, 4);
  const Span ql = span_of(a->q_lens, 1, a->lists, 0, 4), kl = span_of(a->k_lens, 1, a->lists, 0, 4);
  if (!grad) {
    for (const Span& s : {q, k, v, ql, kl})
      if (meet(o, s) || meet(lse, s)) return no("an output overlaps an input");
    if (meet(o, lse)) return no("out and lse overlap");
    if (have_q && !apart(a->lists, a->out_list, a->q_len, a->out_row, a->heads, a->out_head, a->d_head)) return no("two numbers of out share a place");
    return STGN_OK;
  }
  if (a->dout_list > kMaxLd || a->dout_row > kMaxLd || a->dout_head > kMaxLd) return no("a stride is out of range");
  if (beyond(a->q_len, a->heads, a->dout_list, a->dout_row, a->dout_head)) return no(far);
  if (have_q && (!a->dout || !a->dq)) return no("NULL dout or dq");
  if (have_k && (!a->dk || !a->dv)) return no("NULL dk or dv");
  const Span d = reach(a->dout, a->q_len, a->heads, a->dout_list, a->dout_row, a->dout_head);
  const Span out[] = {span_of(a->dq, 1, nq * a->d_head, 0, es), span_of(a->dk, 1, nk * a->d_head, 0, es), span_of(a->dv, 1, nk * a->d_head, 0, es)};
  for (int i = 0; i < 3; ++i) {
    for (const Span& s : {q, k, v, o, lse, d, ql, kl})
      if (meet(out[i], s)) return no("a gradient overlaps an input");
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return no("two gradients overlap");
  }
  return STGN_OK;
}

AttnArgs attention_args(const stgn_attention_args* a) {
  AttnArgs t{};
  t.q = a->q; t.k = a->k; t.v = a->v; t.dout = a->dout; t.out = a->out; t.o = a->out;
  t.dq = a->dq; t.dk = a->dk; t.dv = a->dv; t.lse = a->lse;
  t.q_lens = a->q_lens; t.k_lens = a->k_lens;
  t.sq = {(int64_t)a->q_list, (int64_t)a->q_row, (int64_t)a->q_head};
  t.sk = {(int64_t)a->k_list, (int64_t)a->k_row, (int64_t)a->k_head};
  t.sv = {(int64_t)a->v_list, (int64_t)a->v_row, (int64_t)a->v_head};
  t.so = {(int64_t)a->out_list, (int64_t)a->out_row, (int64_t)a->out_head};
  t.sdo = {(int64_t)a->dout_list, (int64_t)a->dout_row, (int64_t)a->dout_head};
  t.lists = (int)a->lists; t.q_len = (int)a->q_len; t.k_len = (int)a->k_len;
  t.heads = (int)a->heads; t.kv_heads = (int)a->kv_heads; t.group = (int)(a->heads / a->kv_heads); t.d = (int)a->d_head;
  t.group_shift = (t.group & (t.group - 1)) == 0 ? __builtin_ctz((unsigned)t.group) : -1;
  t.causal = (int)a->causal; t.window = (int)(a->window < a->k_len ? a->window : a->k_len); t.scale = a->scale;
  return t;
}

// Matrices [rows x width] that a call reads or writes: one that it writes may be exactly one that it reads, or lie beside it in one wider matrix
struct Matrix { const void* p; uint64_t ld; };
bool apart_or_same(const Matrix& out, const Matrix& other, bool same_allowed, uint64_t rows, uint64_t width, size_t es) {
  if (!out.p || !other.p) return true;
  if (same_allowed && out.p == other.p && out.ld == other.ld) return true;
  const Span s = span_of(out.p, rows, width, out.ld, es), t = span_of(other.p, rows, width, other.ld, es);
  return !meet(s, t) || (out.ld == other.ld && beside(s, width * es, t, width * es, out.ld * es));
}
const char* const kFar = "a matrix reaches over more than 2^48 bytes";
// why a matrix's rows are refused, or NULL
const char* bad_matrix(const Matrix& m, uint64_t rows, uint64_t width, size_t es) {
  if (!m.p) return nullptr;
  if (!aligned(m.p, es)) return "a pointer is not aligned to its element";
  if (m.ld < width || m.ld > kMaxLd) return "rows lie closer together than their width, or too far apart";
  return too_far(rows, m.ld, 1, 0, 1, 0, width, es) ? kFar : nullptr;
}

int check_rms_norm(const stgn_rms_norm_args* a, bool grad, bool sizes_only) {
  if (!a) return no("NULL arguments");
  if (a->dtype > STGN_F16) return no("dtype must be STGN_F32, STGN_BF16 or STGN_F16");
  if (a->reserved) return no("reserved must be 0");
  if (a->rows > kMaxRows) return no("rows out of range");
  if (a->width == 0 || a->width > kMaxWidth) return no("width must lie in 1 .. 2^24");
  if (sizes_only) return STGN_OK;
  if (!(a->eps >= 0.0) || a->eps - a->eps != 0.0) return no("eps must be finite and not negative");
  const size_t es = size_of(a->dtype);
  const uint64_t rows = a->rows, width = a->width;
  if (!a->gain) return no("NULL gain");
  if (!aligned(a->gain, es) || !aligned(a->dgain, es) || !aligned(a->dx, es)) return no("a pointer is not aligned to its element");
  const Span gain = span_of(a->gain, 1, width, 0, es);
  if (!grad) {
    if (rows && !a->x) return no("NULL x");
    if (rows && !a->y && !a->q) return no("NULL y and q");
    if (rows && a->q && !a->scale) return no("q needs scale");
    const Matrix x{a->x, a->ld_x}, res{a->residual, a->ld_residual}, h{a->h, a->ld_h}, y{a->y, a->ld_y}, q{a->q, a->ld_q};
    for (const Matrix& m : {x, res, h, y})
      if (const char* why = bad_matrix(m, rows, width, es)) return no(why);
    if (const char* why = bad_matrix(q, rows, width, 1)) return no(why);
    if (a->q && !aligned(a->scale, 4)) return no("a pointer is not aligned to its element");
    for (const Matrix& out : {h, y})
      for (const Matrix& in : {x, res})
        if (!apart_or_same(out, in, true, rows, width, es)) return no("h and y may each be exactly x or the residual, or overlap neither");
    if (!apart_or_same(h, y, false, rows, width, es)) return no("two outputs overlap");
    const Span sq = span_of(a->q, rows, width, a->ld_q, 1), sc = span_of(a->q ? a->scale : nullptr, 1, rows, 0, 4);
    for (const Matrix& m : {x, res, h, y}) {
      const Span t = span_of(m.p, rows, width, m.ld, es);
      if (meet(sq, t) || meet(sc, t)) return no("q or scale overlaps another tensor");
    }
    for (const Matrix& m : {h, y})
      if (meet(gain, span_of(m.p, rows, width, m.ld, es))) return no("an output overlaps the gain");
    if (meet(sq, gain) || meet(sc, gain) || meet(sq, sc)) return no("q or scale overlaps another tensor");
    return STGN_OK;
  }
  if (rows && (!a->h || !a->dy)) return no("NULL h or dy");
  const Matrix in[] = {{a->h, a->ld_h}, {a->dy, a->ld_dy}, {a->dh, a->ld_dh}};
  for (const Matrix& m : in)
    if (const char* why = bad_matrix(m, rows, width, es)) return no(why);
  if (a->dx && too_far(rows, width, 1, 0, 1, 0, width, es)) return no(kFar);
  const Span dx = span_of(a->dx, rows, width, width, es), dg = span_of(a->dgain, 1, width, 0, es);
  for (const Matrix& m : in) {
    const Span t = span_of(m.p, rows, width, m.ld, es);
    if (meet(dx, t) || meet(dg, t)) return no("a gradient overlaps an input");
  }
  if (meet(dx, gain) || meet(dg, gain)) return no("a gradient overlaps an input");
  if (meet(dx, dg)) return no("two gradients overlap");
  return STGN_OK;
}

NormArgs norm_args(const stgn_rms_norm_args* a) {
  NormArgs n{};
  n.x = a->x; n.residual = a->residual; n.gain = a->gain; n.h = a->h; n.y = a->y; n.q = a->q; n.scale = a->scale;
  n.ld_x = (int64_t)a->ld_x; n.ld_res = (int64_t)a->ld_residual; n.ld_h = (int64_t)a->ld_h; n.ld_y = (int64_t)a->ld_y; n.ld_q = (int64_t)a->ld_q;
  n.rows = (int)a->rows; n.width = (int)a->width; n.eps = a->eps;
  return n;
}

NormGradArgs norm_grad_args(const stgn_rms_norm_args* a) {
  NormGradArgs n{};
  n.dy = a->dy; n.h = a->h; n.gain = a->gain; n.dh = a->dh; n.dx = a->dx; n.dgain = a->dgain;
  n.ld_dy = (int64_t)a->ld_dy; n.ld_h = (int64_t)a->ld_h; n.ld_dh = (int64_t)a->ld_dh; n.ld_dx = (int64_t)a->width;
  n.rows = (int)a->rows; n.width = (int)a->width; n.eps = a->eps;
  return n;
}

int check_quantize(const stgn_quantize_args* a, bool sizes_only) {
  if (!a) return no("NULL arguments");
  if (a->dtype > STGN_F16) return no("dtype must be STGN_F32, STGN_BF16 or STGN_F16");
  if (a->columns > 1) return no("columns must be 0 or 1");
  if (a->rows > kMaxRows) return no("rows out of range");
  if (a->width == 0 || a->width > kMaxWidth) return no("width must lie in 1 .. 2^24");
  if (a->columns && (((uint64_t)a->rows + 127) / 128) * (((uint64_t)a->width + 63) / 64) > kMaxGroups) return no("the matrix has more tiles than a launch");
  if (sizes_only) return STGN_OK;
  const size_t es = size_of(a->dtype);
  const uint64_t q_rows = a->columns ? a->width : a->rows, q_width = a->columns ? a->rows : a->width;
  if ((a->rows && (!a->x || !a->q)) || (q_rows && !a->scale)) return no("NULL x, q or scale");
  if (const char* why = bad_matrix({a->x, a->ld_x}, a->rows, a->width, es)) return no(why);
  if (const char* why = bad_matrix({a->q, a->ld_q}, q_rows, q_width, 1)) return no(why);
  if (!aligned(a->scale, 4)) return no("a pointer is not aligned to its element");
  const Span x = span_of(a->x, a->rows, a->width, a->ld_x, es), q = span_of(a->q, q_rows, q_width, a->ld_q, 1), sc = span_of(a->scale, 1, q_rows, 0, 4);
  if (meet(x, q) || meet(x, sc) || meet(q, sc)) return no("an output overlaps the input or the other output");
  return STGN_OK;
}

ColumnsArgs columns_args(const stgn_quantize_args* a) {
  ColumnsArgs c{};
  c.x = a->x; c.q = a->q; c.scale = a->scale; c.ld_x = (int64_t)a->ld_x; c.ld_q = (int64_t)a->ld_q;
  c.rows = (int)a->rows; c.width = (int)a->width;
  return c;
}

int check_linear_i8(const stgn_linear_quantized_args* a, bool sizes_only) {
  if (!a) return no("NULL arguments");
  if (a->dtype > STGN_F16) return no("dtype must be STGN_F32, STGN_BF16 or STGN_F16");
  if (a->activation > STGN_ACT_SILU) return no("unknown activation");
  if (a->reserved) return no("reserved must be 0");
  if (a->rows > kMaxRows) return no("rows out of range");
  if (a->d_in == 0 || a->d_in > 131071) return no("d_in must lie in 1 .. 131071");
  if (a->d_out == 0 || a->d_out > kMaxWidth) return no("d_out must lie in 1 .. 2^24");
  if ((((uint64_t)a->rows + 63) / 64) * (((uint64_t)a->d_out + 63) / 64) > kMaxGroups - 1024) return no("the product has more tiles than a launch");
  if (sizes_only) return STGN_OK;
  const size_t es = size_of(a->dtype);
  const uint64_t rows = a->rows, n = a->d_out;
  if (!a->w || !a->w_scale || (rows && (!a->x || !a->x_scale || !a->y))) return no("NULL x, w, a scale or y");
  if (!aligned(a->x_scale, 4) || !aligned(a->w_scale, 4) || !aligned(a->bias, es)) return no("a pointer is not aligned to its element");
  const Matrix x{a->x, a->ld_x}, w{a->w, a->ld_w}, y{a->y, a->ld_y}, res{a->residual, a->ld_residual};
  if (const char* why = bad_matrix(x, rows, a->d_in, 1)) return no(why);
  if (const char* why = bad_matrix(w, n, a->d_in, 1)) return no(why);
  for (const Matrix& m : {y, res})
    if (const char* why = bad_matrix(m, rows, n, es)) return no(why);
  if (!apart_or_same(y, res, true, rows, n, es)) return no("y overlaps the residual (it may be exactly the residual)");
  const Span out = span_of(a->y, rows, n, a->ld_y, es);
  for (const Span& t : {span_of(a->x, rows, a->d_in, a->ld_x, 1), span_of(a->w, n, a->d_in, a->ld_w, 1), span_of(a->x_scale, 1, rows, 0, 4),
                        span_of(a->w_scale, 1, n, 0, 4), span_of(a->bias, 1, n, 0, es)})
    if (meet(out, t)) return no("y overlaps an input");
  return STGN_OK;
}

Linear8Args linear_i8_args(const stgn_linear_quantized_args* a) {
  Linear8Args l{};
  l.x = a->x; l.w = a->w; l.x_scale = a->x_scale; l.w_scale = a->w_scale; l.bias = a->bias; l.residual = a->residual; l.y = a->y;
  l.ld_x = (int64_t)a->ld_x; l.ld_w = (int64_t)a->ld_w; l.ld_res = (int64_t)a->ld_residual; l.ld_y = (int64_t)a->ld_y;
  l.rows = (int)a->rows; l.d_in = (int)a->d_in; l.d_out = (int)a->d_out; l.act = (int)a->activation;
  return l;
}

int check_dropout(const stgn_dropout_args* a) {
  if (!a) return no("NULL arguments");
  if (a->dtype > STGN_F16) return no("dtype must be STGN_F32, STGN_BF16 or STGN_F16");
  if (a->rows > kMaxRows) return no("rows out of range");
  if (a->width == 0 || a->width > kMaxWidth) return no("width must lie in 1 .. 2^24");
  if (a->site > 65535) return no("site must lie in 0 .. 65535");
  if (!(a->p >= 0.0 && a->p <= 1.0)) return no("p must lie in 0 .. 1");
  const size_t es = size_of(a->dtype);
  const uint64_t rows = a->rows, width = a->width;
  if ((rows && (!a->x || !a->y)) || !a->rng) return no("NULL x, y or rng");
  if (!aligned(a->rng, 8)) return no("a pointer is not aligned to its element");
  const Matrix x{a->x, a->ld_x}, res{a->residual, a->ld_residual}, y{a->y, a->ld_y};
  for (const Matrix& m : {x, res, y})
    if (const char* why = bad_matrix(m, rows, width, es)) return no(why);
  for (const Matrix& in : {x, res})
    if (!apart_or_same(y, in, true, rows, width, es)) return no("y may be exactly x or the residual, or overlap neither");
  if (meet(span_of(a->y, rows, width, a->ld_y, es), span_of(a->rng, 1, 2, 0, 8))) return no("y overlaps rng");
  return STGN_OK;
}

}  // namespace

extern "C" {

int stgn_linear_workspace(const stgn_linear_args* args, size_t* forward_bytes, size_t* grad_bytes) {
  if (const int rc = check_linear(args, false, true)) return rc;
  if (forward_bytes) *forward_bytes = linear_bytes(linear_args(args), (int)args->dtype);
  if (grad_bytes) *grad_bytes = linear_grad_bytes(linear_grad_args(args), (int)args->dtype);
  return STGN_OK;
}

int stgn_linear(const stgn_linear_args* args, void* device_workspace, size_t device_bytes, void* hip_stream) {
  if (const int rc = check_linear(args, false, false)) return rc;
  const LinearArgs a = linear_args(args);
  if (const int rc = check_workspace(linear_bytes(a, (int)args->dtype), device_workspace, device_bytes)) return rc;
  if (a.rows == 0) return STGN_OK;
  return finish(launch_linear(a, (int)args->dtype, device_workspace, static_cast<hipStream_t>(hip_stream)));
}

int stgn_linear_grad(const stgn_linear_args* args, void* device_workspace, size_t device_bytes, void* hip_stream) {
  if (const int rc = check_linear(args, true, false)) return rc;
  const LinearGradArgs a = linear_grad_args(args);
  if (const int rc = check_workspace(linear_grad_bytes(a, (int)args->dtype), device_workspace, device_bytes)) return rc;
  return finish(STGN_BY_TYPE(args->dtype, linear_grad, a, device_workspace, static_cast<hipStream_t>(hip_stream)));
}

int stgn_attention_workspace(const stgn_attention_args* args, size_t* forward_bytes, size_t* grad_bytes) {
  if (const int rc = check_attention(args, false, true)) return rc;
  const AttnArgs a = attention_args(args);
  if (forward_bytes) *forward_bytes = attention_bytes(a, (int)args->dtype);
  if (grad_bytes) *grad_bytes = attention_grad_bytes(a, (int)args->dtype);
  return STGN_OK;
}

int stgn_attention(const stgn_attention_args* args, void* device_workspace, size_t device_bytes, void* hip_stream) {
  if (const int rc = check_attention(args, false, false)) return rc;
  const AttnArgs a = attention_args(args);
  if (const int rc = check_workspace(attention_bytes(a, (int)args->dtype), device_workspace, device_bytes)) return rc;
  if (a.lists == 0 || a.q_len == 0) return STGN_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (few_rows(a, (int)args->dtype, false)) return finish(STGN_BY_TYPE(args->dtype, attention_rows, a, device_workspace, s));
  return finish(STGN_BY_TYPE(args->dtype, attention, a, device_workspace, s));
}

int stgn_attention_grad(const stgn_attention_args* args, void* device_workspace, size_t device_bytes, void* hip_stream) {
  if (const int rc = check_attention(args, true, false)) return rc;
  const AttnArgs a = attention_args(args);
  if (const int rc = check_workspace(attention_grad_bytes(a, (int)args->dtype), device_workspace, device_bytes)) return rc;
  if (a.lists == 0 || (a.q_len == 0 && a.k_len == 0)) return STGN_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (few_rows(a, (int)args->dtype, true)) return finish(STGN_BY_TYPE(args->dtype, attention_rows_grad, a, device_workspace, s));
  return finish(STGN_BY_TYPE(args->dtype, attention_grad, a, device_workspace, s));
}

int stgn_rms_norm_workspace(const stgn_rms_norm_args* args, size_t* forward_bytes, size_t* grad_bytes) {
  if (const int rc = check_rms_norm(args, false, true)) return rc;
  if (forward_bytes) *forward_bytes = 0;
  if (grad_bytes) *grad_bytes = STGN_BY_TYPE(args->dtype, rms_norm_grad_bytes, norm_grad_args(args));
  return STGN_OK;
}

int stgn_rms_norm(const stgn_rms_norm_args* args, void*, size_t, void* hip_stream) {
  if (const int rc = check_rms_norm(args, false, false)) return rc;
  if (args->rows == 0) return STGN_OK;
  return finish(STGN_BY_TYPE(args->dtype, rms_norm, norm_args(args), static_cast<hipStream_t>(hip_stream)));
}

int stgn_rms_norm_grad(const stgn_rms_norm_args* args, void* device_workspace, size_t device_bytes, void* hip_stream) {
  if (const int rc = check_rms_norm(args, true, false)) return rc;
  const NormGradArgs a = norm_grad_args(args);
  if (const int rc = check_workspace(STGN_BY_TYPE(args->dtype, rms_norm_grad_bytes, a), device_workspace, device_bytes)) return rc;
  if (!a.dx && !a.dgain) return STGN_OK;
  return finish(STGN_BY_TYPE(args->dtype, rms_norm_grad, a, device_workspace, static_cast<hipStream_t>(hip_stream)));
}

int stgn_quantize_workspace(const stgn_quantize_args* args, size_t* bytes) {
  if (const int rc = check_quantize(args, true)) return rc;
  if (bytes) *bytes = args->columns ? STGN_BY_TYPE(args->dtype, columns_bytes, columns_args(args)) : 0;
  return STGN_OK;
}

int stgn_quantize(const stgn_quantize_args* args, void* device_workspace, size_t device_bytes, void* hip_stream) {
  if (const int rc = check_quantize(args, false)) return rc;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (args->columns) {
    const ColumnsArgs a = columns_args(args);
    if (const int rc = check_workspace(STGN_BY_TYPE(args->dtype, columns_bytes, a), device_workspace, device_bytes)) return rc;
    return finish(STGN_BY_TYPE(args->dtype, columns_in_8, a, device_workspace, s));
  }
  if (args->rows == 0) return STGN_OK;
  NormArgs a{};
  a.x = args->x; a.q = args->q; a.scale = args->scale; a.ld_x = (int64_t)args->ld_x; a.ld_q = (int64_t)args->ld_q;
  a.rows = (int)args->rows; a.width = (int)args->width;
  return finish(STGN_BY_TYPE(args->dtype, rows_in_8, a, s));
}

int stgn_linear_quantized_workspace(const stgn_linear_quantized_args* args, size_t* bytes) {
  if (const int rc = check_linear_i8(args, true)) return rc;
  if (bytes) *bytes = dense8::part_bytes(linear_i8_args(args));
  return STGN_OK;
}

int stgn_linear_quantized(const stgn_linear_quantized_args* args, void* device_workspace, size_t device_bytes, void* hip_stream) {
  if (const int rc = check_linear_i8(args, false)) return rc;
  const Linear8Args a = linear_i8_args(args);
  if (const int rc = check_workspace(dense8::part_bytes(a), device_workspace, device_bytes)) return rc;
  if (a.rows == 0) return STGN_OK;
  return finish(STGN_BY_TYPE(args->dtype, linear_i8, a, device_workspace, static_cast<hipStream_t>(hip_stream)));
}

int stgn_dropout(const stgn_dropout_args* args, void* hip_stream) {
  if (const int rc = check_dropout(args)) return rc;
  if (args->rows == 0) return STGN_OK;
  DropoutArgs a{};
  a.x = args->x; a.residual = args->residual; a.y = args->y; a.rng = args->rng;
  a.ld_x = (int64_t)args->ld_x; a.ld_res = (int64_t)args->ld_residual; a.ld_y = (int64_t)args->ld_y;
  a.rows = (int)args->rows; a.width = (int)args->width; a.site = args->site;
  a.border = (uint32_t)nearbyint(args->p * 65536.0);
  a.scale = a.border < 65536u ? (float)(65536.0 / (65536.0 - a.border)) : 0.f;
  return finish(STGN_BY_TYPE(args->dtype, dropout, a, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
