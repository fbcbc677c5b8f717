// C ABI of the packed attention (include/losa.h): argument checks, dispatch.
#include "losa.h"

#include <algorithm>
#include <cmath>
#include <new>

#include "abi.hpp"
#include "packed.hpp"

namespace {

using losa::aligned16;
using losa::elem_bytes;
using losa::fail;
using losa::hip_status;
using losa::take_view;

// Refuses sequences that own the same row of q; *run: the most neighbouring rows that
// sequences own.
losa_status check_disjoint(const int64_t* start, const int32_t* len, int n, int64_t* run) {
  *run = 0;
  if (!start) {  // one after another
    for (int i = 0; i < n; ++i) *run += len[i];
    return LOSA_OK;
  }
  if (n == 0) return LOSA_OK;
  int* const by = new (std::nothrow) int[n];
  if (!by) return fail(LOSA_ERR_CAPACITY, "no host memory to order %d sequences", n);
  for (int i = 0; i < n; ++i) by[i] = i;
  std::sort(by, by + n, [&](int a, int b) { return start[a] != start[b] ? start[a] < start[b] : a < b; });
  losa_status st = LOSA_OK;
  int64_t first = -1, end = -1;  // the present run
  int who = -1;
  for (int x = 0; x < n && st == LOSA_OK; ++x) {
    const int i = by[x];
    if (len[i] == 0) continue;
    if (start[i] < end)
      st = fail(LOSA_ERR_INVALID_SHAPE, "sequences %d and %d own the same rows of q", who, i);
    if (start[i] != end) first = start[i];
    end = start[i] + len[i];
    *run = std::max(*run, end - first);
    who = i;
  }
  delete[] by;
  return st;
}

// Whether two of `rows` neighbouring rows of H heads share elements: rows a apart and
// heads b apart lie |a token - b head| apart, so for each b the two nearest a are looked at.
bool rows_overlap(const losa_view& y, int64_t rows, int H, int d) {
  if (rows < 2 || H < 2 || (H - 1) * y.head + d <= y.token || (rows - 1) * y.token + d <= y.head)
    return false;
  for (int64_t b = 1; b < H; ++b) {
    const int64_t a = b * y.head / y.token, past = b * y.head - a * y.token;
    if ((a > 0 && a < rows && past < d) || (a + 1 < rows && y.token - past < d)) return true;
  }
  return false;
}

bool info_ok(const losa_packed_info* i) {
  return i->bytes >= 0 && i->q_rows >= 0 && i->k_rows >= 0 && i->part_rows >= 0 &&
         i->q_run >= 0 && i->q_run <= i->q_rows && i->n_tiles >= 0 &&
         i->n_few >= 0 && i->n_wide >= 0 && i->n_joins >= i->n_wide && i->H > 0 && i->H_kv > 0 && i->H % i->H_kv == 0 &&
         (i->dtype == LOSA_DTYPE_F32 || i->dtype == LOSA_DTYPE_BF16) &&
         (size_t)i->bytes == losa::packed_plan_bytes({i->n_tiles, i->n_few, i->n_joins, i->n_wide, i->tile_rows, i->part_rows}) &&
         (i->tile_rows == losa::kPackedTile[i->dtype == LOSA_DTYPE_BF16] ||
          (i->dtype == LOSA_DTYPE_F32 && i->tile_rows == losa::kPackedNarrow));
}

}  // namespace

extern "C" {

losa_status losa_packed_plan(const int64_t* q_start, const int32_t* q_len, const int64_t* k_start,
                             const int32_t* k_len, int n_seq, losa_dtype dtype, int H, int H_kv,
                             int causal, void* plan, size_t plan_bytes, losa_packed_info* info) {
  if (!info || (n_seq > 0 && (!q_len || !k_len)))
    return fail(LOSA_ERR_NULL_POINTER, "q_len, k_len and info must be non-NULL");
  if (n_seq < 0 || H <= 0 || H_kv <= 0 || H % H_kv != 0 || H > (1 << 20))
    return fail(LOSA_ERR_INVALID_SHAPE, "n_seq=%d H=%d H_kv=%d: H must be a multiple of H_kv",
                n_seq, H, H_kv);
  if (dtype != LOSA_DTYPE_F32 && dtype != LOSA_DTYPE_BF16)
    return fail(LOSA_ERR_UNSUPPORTED, "unknown dtype %d", (int)dtype);
  const int64_t far = (int64_t)1 << 40;
  int64_t q0 = 0, k0 = 0, q_rows = 0, k_rows = 0;
  for (int i = 0; i < n_seq; ++i) {
    const int64_t qs = q_start ? q_start[i] : q0, ks = k_start ? k_start[i] : k0;
    if (q_len[i] < 0 || k_len[i] < 0 || qs < 0 || ks < 0 || qs > far || ks > far)
      return fail(LOSA_ERR_INVALID_SHAPE, "sequence %d: lengths and starts must be >= 0", i);
    if (q_len[i] > (1 << 30) || k_len[i] > (1 << 30) ||
        (int64_t)q_len[i] * (H / H_kv) > (1 << 30))
      return fail(LOSA_ERR_INVALID_SHAPE, "sequence %d is too long", i);
    q0 += q_len[i];
    k0 += k_len[i];
    if (q_len[i] > 0 && qs + q_len[i] > q_rows) q_rows = qs + q_len[i];
    if (q_len[i] > 0 && k_len[i] > 0 && ks + k_len[i] > k_rows) k_rows = ks + k_len[i];
  }
  int64_t q_run = 0;
  const losa_status st = check_disjoint(q_start, q_len, n_seq, &q_run);
  if (st != LOSA_OK) return st;
  const losa::PackedSeqs s = {q_start, k_start, q_len, k_len, n_seq, H / H_kv, H_kv,
                              causal != 0, dtype == LOSA_DTYPE_BF16};
  losa::PackedCounts c;
  if (!losa::packed_counts(s, &c))
    return fail(LOSA_ERR_INVALID_SHAPE, "the batch has more units of work than one launch takes");
  const losa_packed_info got = {(int64_t)losa::packed_plan_bytes(c), q_rows, k_rows, c.part_rows,
                                q_run, c.tiles, c.few, c.joins, c.wide, c.tile_rows, H, H_kv,
                                causal != 0, dtype};
  if (plan) {
    if ((reinterpret_cast<uintptr_t>(plan) & 7u) != 0)
      return fail(LOSA_ERR_ALIGNMENT, "plan must be 8-byte aligned");
    if (plan_bytes < (size_t)got.bytes)
      return fail(LOSA_ERR_CAPACITY, "plan_bytes=%zu < %lld", plan_bytes, (long long)got.bytes);
    losa::packed_fill(s, c, plan);
  }
  *info = got;
  return LOSA_OK;
}

size_t losa_packed_workspace_bytes(const losa_packed_info* info, int d) {
  if (!info || !info_ok(info) || d <= 0) return 0;
  return (size_t)info->part_rows * info->H_kv * (d + 2) * sizeof(float);
}

losa_status losa_packed_attn_fwd(const losa_view* q, const losa_view* k, const losa_view* v,
                                 int64_t q_rows, int64_t k_rows, const losa_packed_info* info,
                                 const void* plan, int d, float scale, const losa_view* o,
                                 float* lse, int64_t lse_head, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  if (!q || !k || !v || !info || !o)
    return fail(LOSA_ERR_NULL_POINTER, "q, k, v, info and o must be non-NULL");
  if (!info_ok(info))
    return fail(LOSA_ERR_INVALID_SHAPE, "info is not what losa_packed_plan filled");
  if (d <= 0) return fail(LOSA_ERR_INVALID_SHAPE, "d=%d must be > 0", d);
  if (d != 64 && d != 128)
    return fail(LOSA_ERR_UNSUPPORTED, "head dim d=%d not supported (64 or 128)", d);
  if (!std::isfinite(scale) || !(scale > 0.f))
    return fail(LOSA_ERR_INVALID_SHAPE, "scale must be finite and > 0");
  if (q_rows < info->q_rows || k_rows < info->k_rows)
    return fail(LOSA_ERR_INVALID_SHAPE, "the plan needs %lld rows of q (got %lld), %lld of k (%lld)",
                (long long)info->q_rows, (long long)q_rows, (long long)info->k_rows,
                (long long)k_rows);
  if (info->n_tiles == 0 && info->n_few == 0) return LOSA_OK;  // no row is owned
  if (!plan) return fail(LOSA_ERR_NULL_POINTER, "plan must be non-NULL");
  if ((reinterpret_cast<uintptr_t>(plan) & 7u) != 0)
    return fail(LOSA_ERR_ALIGNMENT, "plan must be 8-byte aligned");
  const bool bf16 = info->dtype == LOSA_DTYPE_BF16;
  const int el = (int)elem_bytes(info->dtype);
  losa_status st;
  losa_view qv, kv[2] = {}, ov;
  if ((st = take_view("q", q, &qv, el, 1, q_rows, info->H, d, false)) != LOSA_OK) return st;
  if ((st = take_view("o", o, &ov, el, 1, q_rows, info->H, d, true)) != LOSA_OK) return st;
  if (((qv.token | qv.head | ov.token | ov.head) >> 31) != 0)
    return fail(LOSA_ERR_INVALID_SHAPE, "q and o: strides must be below 2^31 elements");
  if (rows_overlap(ov, info->q_run, info->H, d))
    return fail(LOSA_ERR_INVALID_SHAPE, "o: rows overlap (token stride %lld, head stride %lld)",
                (long long)ov.token, (long long)ov.head);
  if (info->k_rows > 0) {
    for (int i = 0; i < 2; ++i) {
      const char* const name = i == 0 ? "k" : "v";
      st = take_view(name, i == 0 ? k : v, &kv[i], el, 1, k_rows, info->H_kv, d, false);
      if (st != LOSA_OK) return st;
      if (kv[i].token < d || kv[i].token * el > ((int64_t)1 << 26))
        return fail(LOSA_ERR_INVALID_SHAPE, "%s: token stride %lld not in [d, 64 MiB]", name,
                    (long long)kv[i].token);
    }
  }
  if (lse) {
    if ((reinterpret_cast<uintptr_t>(lse) & 3u) != 0)
      return fail(LOSA_ERR_ALIGNMENT, "lse must be 4-byte aligned");
    if (lse_head < info->q_rows)
      return fail(LOSA_ERR_INVALID_SHAPE, "lse_head=%lld < %lld rows", (long long)lse_head,
                  (long long)info->q_rows);
  }
  const size_t need = losa_packed_workspace_bytes(info, d);
  if (need > 0) {
    if (!workspace) return fail(LOSA_ERR_NULL_POINTER, "the plan needs a workspace of %zu bytes", need);
    if (!aligned16(workspace)) return fail(LOSA_ERR_ALIGNMENT, "workspace must be 16-byte aligned");
    if (workspace_bytes < need)
      return fail(LOSA_ERR_CAPACITY, "workspace_bytes=%zu < %zu", workspace_bytes, need);
  }
  if ((ov.data == qv.data && !losa::same_rows(ov, qv)) || ov.data == kv[0].data || ov.data == kv[1].data)
    return fail(LOSA_ERR_INVALID_SHAPE, "o may lie over q only as the same view, and not over k or v");
  losa::PackedArgs a = {};
  a.items = static_cast<const losa::PackedItem*>(plan);
  a.joins = reinterpret_cast<const losa::PackedJoin*>(a.items + info->n_tiles + info->n_few);
  a.q = qv.data;
  a.k = kv[0].data;
  a.v = kv[1].data;
  a.o = ov.data;
  a.lse = lse;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = a.part_o + (size_t)info->part_rows * info->H_kv * d;
  a.qt = qv.token;
  a.qh = qv.head;
  a.kt = kv[0].token;
  a.kh = kv[0].head;
  a.vt = kv[1].token;
  a.vh = kv[1].head;
  a.ot = ov.token;
  a.oh = ov.head;
  a.lse_head = lse_head;
  a.q_rows = q_rows;
  a.k_rows = k_rows;
  a.part_rows = info->part_rows;
  a.H_kv = info->H_kv;
  a.G = info->H / info->H_kv;
  a.by_G = losa::fast_div((uint32_t)a.G);
  a.by_H_kv = losa::fast_div((uint32_t)a.H_kv);
  a.n_tiles = info->n_tiles;
  a.n_joins = info->n_joins;
  a.n_wide = info->n_wide;
  a.tile_rows = info->tile_rows;
  a.scale_log2 = scale * 1.4426950408889634f;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  st = hip_status((bf16 ? losa::launch_packed_bf16 : losa::launch_packed_f32)(d, a, info->n_few, hs),
                  "losa_packed_attn_fwd");
  if (st != LOSA_OK) return st;
  return hip_status(losa::launch_packed_join(d, bf16, a, hs),
                    "losa_packed_attn_fwd (join)");
}

}  // extern "C"
