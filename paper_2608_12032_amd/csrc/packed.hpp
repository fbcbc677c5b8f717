// Internal launchers and plan of the packed attention; arguments are checked in
// abi_packed.cpp.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace losa {

// Packed attention (packed_plan.cpp, packed_bf16.hip, packed_f32.hip).  A row of a
// sequence is one query token under one query head of a key head's group, numbered
// token * G + head in group, so that rows which share keys fill a tile together.
// One unit of work: a tile's or part's rows against a range of keys.  Row r (from 0) is
// token t under head h of the group, (t, h) = divmod(head0 + r, G), and sees the first
// seen + t of the keys, `keys` at most.
struct PackedItem {
  int64_t q_row, k_row;  // rows of q and of k of the unit's first token and key
  int32_t head0;
  int32_t rows;  // rows of the sequence from the unit's first on
  int32_t keys;  // keys that some row of the unit sees
  int32_t seen;  // (kAllSeen: every row sees them all)
  int32_t part;  // first partial row to write, or -1: the result itself
  int32_t split;  // fp32: 2^split waves of the workgroup share a row set
};
constexpr int32_t kAllSeen = 1 << 30;
// One row whose keys were split: n partial rows at part, part + step, ...
struct PackedJoin {
  int64_t q_row;  // row of q
  int32_t in_group, part, step, n;
};
// Division by a number of the call, n / d for any 32-bit n: a product and two shifts
// (Granlund and Montgomery, "Division by Invariant Integers using Multiplication").
struct FastDiv {
  uint32_t d, m, s1, s2;
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t l = 0;
  while (((uint64_t)1 << l) < d) ++l;
  return {d, (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << l) - d)) / d + 1), l < 1 ? l : 1,
          l < 1 ? 0 : l - 1};
}
__device__ __forceinline__ int divide(int n, const FastDiv& f) {
  const uint32_t t = __umulhi(f.m, (uint32_t)n);
  return (int)((t + (((uint32_t)n - t) >> f.s1)) >> f.s2);
}

struct PackedArgs {
  const PackedItem* items;
  const PackedJoin* joins;
  const void *q, *k, *v;
  void* o;
  float* lse;
  float *part_o, *part_ml;               // [partial row][H_kv][d], [...][2]: max (log2 units), sum
  int64_t qt, qh, kt, kh, vt, vh, ot, oh;  // token and head strides, elements
  int64_t lse_head;
  int64_t q_rows, k_rows, part_rows;
  int H_kv, G;
  FastDiv by_G, by_H_kv;
  int n_tiles;  // items below this are tiles, the others parts of few-row sequences
  int n_joins, n_wide;  // rows to join; the first n_wide are of more than kFewParts parts
  int tile_rows;
  float scale_log2;
};
// Whether the unit's rows (`tile` at most), keys and partial rows lie inside q, k and the
// workspace, and a join's inside q and the workspace.  (A plan's do; nothing is read or
// written for one that does not.)
__device__ __forceinline__ bool inside(const PackedArgs& a, const PackedItem& it, int tile) {
  const int rows = it.rows < tile ? it.rows : tile;
  // (rows of 62 bits: the sums below do not wrap)
  return ((uint64_t)(it.q_row | it.k_row) >> 62 == 0) & (it.head0 >= 0) & (it.head0 < a.G) &
         (it.rows > 0) & (it.keys >= 0) &
         (it.q_row + divide(it.head0 + rows - 1, a.by_G) < a.q_rows) &
         (it.k_row + it.keys <= a.k_rows) &
         ((it.part < 0) | ((int64_t)it.part + rows <= a.part_rows));
}
constexpr int kMostParts = 256, kFewParts = 16;
__device__ __forceinline__ bool inside(const PackedArgs& a, const PackedJoin& j) {
  return (j.q_row >= 0) & (j.q_row < a.q_rows) & (j.in_group >= 0) & (j.in_group < a.G) &
         (j.part >= 0) & (j.step >= 0) & (j.n > 0) & (j.n <= kMostParts) &
         (j.part + (int64_t)(j.n - 1) * j.step < a.part_rows);
}

// Rows of a tile (fp32: of a wide row set; a call of few units takes sets of 16), rows of
// a sequence that make it a few-row one.
constexpr int kPackedTile[2] = {32, 128};  // [bf16]
constexpr int kPackedFew[2] = {16, 32};
constexpr int kPackedNarrow = 16;
// Waves of a workgroup: of units, of joins (a row of up to kFewParts parts a wave).
constexpr int kPackedWaves[2] = {8, 4};  // [bf16]
constexpr int kJoinWaves = 8;
// Workgroups of one launch: it counts its threads in 32 bits.
constexpr int64_t most_workgroups(int waves) { return (((int64_t)1 << 32) - 1) / (64 * waves); }
// The sequences of a call as the plan takes them (starts null: one after another).
struct PackedSeqs {
  const int64_t *q_start, *k_start;
  const int32_t *q_len, *k_len;
  int n, G, H_kv, causal;
  bool bf16;
};
struct PackedCounts {
  int tiles, few, joins, wide;
  int tile_rows;
  int64_t part_rows;
};
// False: more units than a launch takes.  The plan is tiles, few-row units, joins.
bool packed_counts(const PackedSeqs& s, PackedCounts* out);
void packed_fill(const PackedSeqs& s, const PackedCounts& n, void* plan);
inline size_t packed_plan_bytes(const PackedCounts& n) {
  return ((size_t)n.tiles + n.few) * sizeof(PackedItem) + (size_t)n.joins * sizeof(PackedJoin);
}
hipError_t launch_packed_bf16(int d, const PackedArgs& a, int n_few, hipStream_t stream);
hipError_t launch_packed_f32(int d, const PackedArgs& a, int n_few, hipStream_t stream);
hipError_t launch_packed_join(int d, bool bf16, const PackedArgs& a, hipStream_t stream);

}  // namespace losa
