// C ABI of the rotary positions and query/key norms (include/losa.h): the position
// table, argument checks, dispatch.
#include "losa.h"

#include <algorithm>
#include <cmath>

#include "abi.hpp"
#include "rope.hpp"

losa_status losa::take_view(const char* name, const losa_view* from, losa_view* to, int el, int B,
                            int64_t N, int H, int d, bool out) {
  if (!from || !from->data) return fail(LOSA_ERR_NULL_POINTER, "%s must be non-NULL", name);
  *to = *from;
  int64_t* const s[3] = {&to->batch, &to->token, &to->head};
  const int64_t n[3] = {B, N, H};
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) {
      *s[i] = d;
      continue;
    }
    if (*s[i] < 0 || *s[i] >= ((int64_t)1 << 40))
      return fail(LOSA_ERR_INVALID_SHAPE, "%s: stride %lld out of range", name, (long long)*s[i]);
    if (*s[i] * el % 16 != 0)
      return fail(LOSA_ERR_ALIGNMENT, "%s: strides must be multiples of 16 bytes", name);
    if (out && *s[i] < d)
      return fail(LOSA_ERR_INVALID_SHAPE, "%s: rows of an output overlap (stride %lld < d=%d)",
                  name, (long long)*s[i], d);
  }
  if (!aligned16(to->data)) return fail(LOSA_ERR_ALIGNMENT, "%s must be 16-byte aligned", name);
  return LOSA_OK;
}

bool losa::same_rows(const losa_view& a, const losa_view& b) {
  return a.data == b.data && a.batch == b.batch && a.token == b.token && a.head == b.head;
}

namespace {

using losa::aligned16;
using losa::elem_bytes;
using losa::fail;
using losa::hip_status;
using losa::same_rows;
using losa::take_view;

losa_status check_rows(losa_dtype dtype, int B, int N, int N_pad, int H, int d) {
  if (B <= 0 || N <= 0 || H <= 0 || d <= 0)
    return fail(LOSA_ERR_INVALID_SHAPE, "B=%d N=%d H=%d d=%d must all be > 0", B, N, H, d);
  if (N_pad < N) return fail(LOSA_ERR_INVALID_SHAPE, "N_pad=%d < N=%d", N_pad, N);
  if (N_pad > (1 << 30) || H > (1 << 20))
    return fail(LOSA_ERR_INVALID_SHAPE, "N_pad=%d or H=%d is too large", N_pad, H);
  if (dtype != LOSA_DTYPE_F32 && dtype != LOSA_DTYPE_BF16)
    return fail(LOSA_ERR_UNSUPPORTED, "unknown dtype %d", (int)dtype);
  if (d != 64 && d != 128)
    return fail(LOSA_ERR_UNSUPPORTED, "head dim d=%d not supported (64 or 128)", d);
  return LOSA_OK;
}

// Rows of an output: an axis steps over all that those of smaller strides span, as in any
// slice or permutation of a contiguous tensor.
losa_status check_spread(const char* name, const losa_view& y, int B, int N, int H, int d) {
  const int64_t stride[3] = {y.batch, y.token, y.head}, n[3] = {B, N, H};
  int by[3] = {0, 1, 2};
  std::sort(by, by + 3, [&](int i, int j) { return stride[i] < stride[j]; });
  __int128 span = d;
  for (int i : by) {
    if (n[i] <= 1) continue;
    if (stride[i] < span)
      return fail(LOSA_ERR_INVALID_SHAPE, "%s: rows of an output overlap (stride %lld)", name,
                  (long long)stride[i]);
    span += (__int128)stride[i] * (n[i] - 1);
  }
  return LOSA_OK;
}

// Axes of a rotation: their dims and table offsets.  d <= 0: no bound on their sum.
losa_status check_axes(int n_axes, const int* dim, const int* len, int d, int* rot, int64_t* floats) {
  if (n_axes < 1 || n_axes > losa::kMaxAxes)
    return fail(LOSA_ERR_INVALID_SHAPE, "n_axes=%d not in [1, %d]", n_axes, losa::kMaxAxes);
  int64_t sum = 0;
  *floats = 0;
  for (int a = 0; a < n_axes; ++a) {
    if (dim[a] <= 0 || dim[a] % 2 != 0 || len[a] <= 0)
      return fail(LOSA_ERR_INVALID_SHAPE, "axis %d: dim=%d must be even and > 0, len=%d > 0", a,
                  dim[a], len[a]);
    sum += dim[a];
    *floats += (int64_t)dim[a] * len[a];
    if (*floats >= ((int64_t)1 << 31))
      return fail(LOSA_ERR_INVALID_SHAPE, "the position table exceeds the 32-bit index range");
  }
  if (d > 0 && (sum > d || sum % 8 != 0))
    return fail(LOSA_ERR_INVALID_SHAPE, "axis dims sum to %lld: not a multiple of 8 up to d=%d",
                (long long)sum, d);
  *rot = (int)sum;
  return LOSA_OK;
}

losa_status check_rotation(const losa_rotation* r, int N, int d, losa::RowsArgs* a) {
  int rot = 0;
  int64_t floats = 0;
  const losa_status st = check_axes(r->n_axes, r->axis_dim, r->axis_len, d, &rot, &floats);
  if (st != LOSA_OK) return st;
  if (!r->table || !r->pos)
    return fail(LOSA_ERR_NULL_POINTER, "the rotation's table and pos must be non-NULL");
  if (!aligned16(r->table) || (reinterpret_cast<uintptr_t>(r->pos) & 3u) != 0)
    return fail(LOSA_ERR_ALIGNMENT, "the rotation's table must be 16-byte, pos 4-byte aligned");
  if (r->pos_batch < 0 || r->pos_batch >= ((int64_t)1 << 40) ||
      (r->pos_batch != 0 && r->pos_batch < (int64_t)r->n_axes * N))
    return fail(LOSA_ERR_INVALID_SHAPE, "pos_batch=%lld must be 0 or hold n_axes*N positions",
                (long long)r->pos_batch);
  if (r->pairs != LOSA_PAIRS_NEIGHBOURS && r->pairs != LOSA_PAIRS_HALVES)
    return fail(LOSA_ERR_UNSUPPORTED, "unknown pairs %d", (int)r->pairs);
  a->table = r->table;
  a->pos = r->pos;
  a->pos_batch = r->pos_batch;
  a->axes = r->n_axes;
  a->rot8 = rot / 8;
  int pair = 0, off = 0;
  for (int x = 0; x < r->n_axes; ++x) {
    a->pair0[x] = pair;
    a->dim[x] = r->axis_dim[x];
    a->len[x] = r->axis_len[x];
    a->off[x] = off;
    pair += r->axis_dim[x] / 2;
    off += r->axis_dim[x] * r->axis_len[x];
  }
  return LOSA_OK;
}

losa_status rows_status(hipError_t e, const char* what) {
  if (e == hipErrorInvalidConfiguration)
    return fail(LOSA_ERR_INVALID_SHAPE, "%s: more workgroups than one launch takes", what);
  return hip_status(e, what);
}

// Outputs that start where another tensor of the call does: only an output over its own
// input, row for row.  (Views that overlap elsewhere are the caller's to avoid.)
losa_status check_apart(const losa_view* in, const losa_view* out, int n, bool padded) {
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < n; ++j) {
      if (out[i].data == in[j].data && (i != j || padded || !same_rows(out[i], in[j])))
        return fail(LOSA_ERR_INVALID_SHAPE,
                    "an output may lie over its own input only as the same view, with N_pad = N");
      if (i != j && out[i].data == out[j].data)
        return fail(LOSA_ERR_INVALID_SHAPE, "two outputs lie over each other");
    }
  return LOSA_OK;
}

void set_tensor(losa::RowsTensor* t, const losa_view& x, const losa_view& y, int H) {
  t->x = x.data;
  t->xb = x.batch;
  t->xt = x.token;
  t->xh = x.head;
  t->y = y.data;
  t->yb = y.batch;
  t->yt = y.token;
  t->yh = y.head;
  t->H = H;
}

}  // namespace

extern "C" {

losa_status losa_rope_table(int n_axes, const int* axis_dim, const int* axis_len, double base,
                            float* table, int64_t capacity) {
  if (!axis_dim || !axis_len || !table)
    return fail(LOSA_ERR_NULL_POINTER, "axis_dim, axis_len and table must be non-NULL");
  int rot = 0;
  int64_t floats = 0;
  const losa_status st = check_axes(n_axes, axis_dim, axis_len, 0, &rot, &floats);
  if (st != LOSA_OK) return st;
  if (!std::isfinite(base) || !(base > 0.0))
    return fail(LOSA_ERR_INVALID_SHAPE, "base must be finite and > 0");
  if (capacity < floats)
    return fail(LOSA_ERR_CAPACITY, "capacity=%lld < %lld floats", (long long)capacity,
                (long long)floats);
  for (int a = 0; a < n_axes; ++a)
    for (int p = 0; p < axis_len[a]; ++p)
      for (int j = 0; j < axis_dim[a] / 2; ++j) {
        const double angle = p * std::pow(base, -2.0 * j / axis_dim[a]);
        *table++ = (float)std::cos(angle);
        *table++ = (float)std::sin(angle);
      }
  return LOSA_OK;
}

losa_status losa_rope(const losa_view* x, losa_dtype dtype, int B, int N, int N_pad, int H, int d,
                      const losa_rotation* rot, const losa_view* y, void* stream) {
  if (!rot) return fail(LOSA_ERR_NULL_POINTER, "rot must be non-NULL");
  losa_status st = check_rows(dtype, B, N, N_pad, H, d);
  if (st != LOSA_OK) return st;
  const int el = (int)elem_bytes(dtype);
  losa_view xv, yv;
  if ((st = take_view("x", x, &xv, el, B, N, H, d, false)) != LOSA_OK) return st;
  if ((st = take_view("y", y, &yv, el, B, N_pad, H, d, true)) != LOSA_OK) return st;
  if ((st = check_spread("y", yv, B, N_pad, H, d)) != LOSA_OK) return st;
  losa::RowsArgs a = {};
  if ((st = check_rotation(rot, N, d, &a)) != LOSA_OK) return st;
  if ((st = check_apart(&xv, &yv, 1, N_pad != N)) != LOSA_OK) return st;
  a.B = B;
  a.N = N;
  a.n_pad = N_pad;
  set_tensor(&a.t[0], xv, yv, H);
  a.t[0].rotate = 1;
  return rows_status(losa::launch_rows(d, dtype == LOSA_DTYPE_BF16,
                                      rot->pairs == LOSA_PAIRS_HALVES, a, 1, false,
                                      static_cast<hipStream_t>(stream)),
                    "losa_rope");
}

losa_status losa_qk_norm_rope(const losa_view* q, const losa_view* k, const losa_view* v,
                              losa_dtype dtype, int B, int N, int N_pad, int H, int H_kv, int d,
                              const losa_qk_norm_args* norm, const losa_rotation* rot,
                              const losa_view* q_out, const losa_view* k_out,
                              const losa_view* v_out, void* stream) {
  losa_status st = check_rows(dtype, B, N, N_pad, H, d);
  if (st != LOSA_OK) return st;
  if ((st = check_rows(dtype, B, N, N_pad, H_kv, d)) != LOSA_OK) return st;
  const int el = (int)elem_bytes(dtype);
  losa_view in[3], to[3];
  if ((st = take_view("q", q, &in[0], el, B, N, H, d, false)) != LOSA_OK) return st;
  if ((st = take_view("k", k, &in[1], el, B, N, H_kv, d, false)) != LOSA_OK) return st;
  if ((st = take_view("q_out", q_out, &to[0], el, B, N_pad, H, d, true)) != LOSA_OK) return st;
  if ((st = take_view("k_out", k_out, &to[1], el, B, N_pad, H_kv, d, true)) != LOSA_OK) return st;
  if ((st = check_spread("q_out", to[0], B, N_pad, H, d)) != LOSA_OK) return st;
  if ((st = check_spread("k_out", to[1], B, N_pad, H_kv, d)) != LOSA_OK) return st;
  if ((v == nullptr) != (v_out == nullptr))
    return fail(LOSA_ERR_NULL_POINTER, "v and v_out must both be given or both be NULL");
  if (v) {
    if ((st = take_view("v", v, &in[2], el, B, N, H_kv, d, false)) != LOSA_OK) return st;
    if ((st = take_view("v_out", v_out, &to[2], el, B, N_pad, H_kv, d, true)) != LOSA_OK) return st;
    if ((st = check_spread("v_out", to[2], B, N_pad, H_kv, d)) != LOSA_OK) return st;
  }
  losa::RowsArgs a = {};
  if (rot && (st = check_rotation(rot, N, d, &a)) != LOSA_OK) return st;
  bool all = false;
  if (norm) {
    if (norm->kind != LOSA_NORM_RMS && norm->kind != LOSA_NORM_LAYER)
      return fail(LOSA_ERR_UNSUPPORTED, "unknown norm kind %d", (int)norm->kind);
    if (!std::isfinite(norm->eps) || norm->eps < 0.f)
      return fail(LOSA_ERR_INVALID_SHAPE, "eps must be finite and >= 0");
    if ((norm->q_weight && !aligned16(norm->q_weight)) || (norm->q_bias && !aligned16(norm->q_bias)) ||
        (norm->k_weight && !aligned16(norm->k_weight)) || (norm->k_bias && !aligned16(norm->k_bias)))
      return fail(LOSA_ERR_ALIGNMENT, "norm weights and biases must be 16-byte aligned");
    all = norm->all_heads != 0;
  }
  if ((st = check_apart(in, to, v ? 3 : 2, N_pad != N)) != LOSA_OK) return st;
  a.B = B;
  a.N = N;
  a.n_pad = N_pad;
  set_tensor(&a.t[0], in[0], to[0], H);
  set_tensor(&a.t[1], in[1], to[1], H_kv);
  if (v) set_tensor(&a.t[2], in[2], to[2], H_kv);
  a.t[0].rotate = a.t[1].rotate = rot != nullptr;
  if (norm) {
    a.eps = norm->eps;
    a.t[0].norm = a.t[1].norm = norm->kind == LOSA_NORM_RMS ? losa::kNormRms : losa::kNormLayer;
    a.t[0].w = norm->q_weight;
    a.t[0].b = norm->q_bias;
    a.t[1].w = norm->k_weight;
    a.t[1].b = norm->k_bias;
  }
  return rows_status(losa::launch_rows(d, dtype == LOSA_DTYPE_BF16,
                                      rot && rot->pairs == LOSA_PAIRS_HALVES, a, v ? 3 : 2, all,
                                      static_cast<hipStream_t>(stream)),
                    "losa_qk_norm_rope");
}

}  // extern "C"
