// Attention over packed sequences of different lengths, grouped heads, causal or
// not: bf16 in, fp32 accumulation on gfx950 MFMA.
//
// Mathematics.  Row (token i, head h) of a sequence with key head h / G:
//   O = sum_j softmax_j(scale q . k_j) v_j over the keys j it sees (causal:
//   j <= i + k_len - q_len), by the online softmax: running max, sum and O^T.
//
// Rounding.  Probabilities are rounded to bf16 for P V, the operand type of the matrix
// instruction (in two parts they would double that product, and the matrix cores and the
// instructions around them bound the tiles); their sum is taken before that, in fp32.
// Relative error of O against 64 bits 1.1e-3 to 2.3e-3; rounding O alone gives 0.9e-3 to
// 1.7e-3, plain arithmetic with such probabilities 1.1e-3 to 2.1e-3.
//
// Work unit.  A workgroup of four waves owns a tile of 128 rows, 32 a wave, of one sequence
// and key head and walks a range of its keys.  Rows are numbered token * G + head in group, so a tile's rows
// share their keys whatever G is: G heads of one token fill a tile where each alone
// would leave it nearly empty.  The plan lists the units, longest first.  Orientation,
// key order, LDS images, the two rings and the pipelined sub-iteration are those of
// the block-sparse forward (sparse_fwd.hip, attn_bf16.hpp); the stream is simply the
// unit's keys in order.
//
// Sequences of few rows (32 or fewer: single tokens with grouped heads) are bound by
// HBM, K and V read once, and have no rows to fill the chip with: their keys are split
// into parts (packed_plan.cpp) of a workgroup each, whose waves take the sub-tiles in turn.
// Where few tiles meet many keys, their keys are split too.  Parts leave O, max and sum in
// the workspace, and join_kernel joins them in a fixed order.  How a sequence is split
// follows from its own lengths alone, so it gives the same bits alone and packed among
// others.
//
// Bounds.  K and V are read through a buffer resource of one sub-tile each, cut at the
// unit's last key and rebuilt per sub-tile from 64-bit addresses: rows behind the end
// (of the sequence, or behind the last key that any row of the unit sees) read as 0
// whatever lies there, and no offset passes 32 bits in a long cache.
//
// Values that are not finite.  A probability of 0 times an infinite or NaN value would
// spread it to rows that do not see the key.  Rows behind the unit's last key read as 0;
// inside the diagonal sub-tiles of a causal unit the products are taken as they come,
// and only if the result is not finite the unit is done again, slowly, with such values
// kept out of the matrix products and added to the rows that see them.
#include <type_traits>

#include "attn_bf16.hpp"
#include "common.hpp"
#include "packed.hpp"

namespace losa {

namespace {

// Scores of the sub-tile's keys (this lane's 16) at or beyond `left` -> -inf.
__device__ __forceinline__ void mask_left(f32x16_t& s, int left, int g) {
  const int lim = left - 4 * g;  // (compared with constants: no register each)
#pragma unroll
  for (int t = 0; t < 16; ++t)
    if (lim <= ((t >> 2) << 3) + (t & 3)) s[t] = -INFINITY;
}

// Bound on a lane's sum of 16 probabilities before the running max is raised, as in
// the block-sparse forward.
constexpr float kSumBound = 1048576.0f;

__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < INFINITY; }

// The sub-tiles of 32 rows of D elements, `stride` bytes apart, of a range of rows, one
// after another.  Each has a buffer resource of its own, so that rows behind the end read
// as 0 and no offset passes 32 bits.
template <int D>
struct Stream {
  const char* at;  // the next sub-tile
  int left;        // rows from it on
  uint32_t stride;

  __device__ __forceinline__ Stream(const char* base, int n, uint32_t st, int first)
      : at(base + (int64_t)first * 32 * st), left(n - 32 * first), stride(st) {}
  __device__ __forceinline__ i32x4_t next() {
    const int rows = left > 32 ? 32 : left;
    const i32x4_t rs = rsrc_words(at, rows <= 0 ? 0u : (uint32_t)(rows - 1) * stride + 2 * D);
    at += (uint64_t)stride * 32;
    left -= 32;
    return rs;
  }
};

// The call's arguments, read again from where the launch put them.  After the loop a
// kernel takes what it needs from here, so that the loop carries none of it.
__device__ __forceinline__ PackedArgs late_args() {
  PackedArgs b;
  uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  __builtin_memcpy(&b, reinterpret_cast<__attribute__((address_space(4))) const char*>(at),
                   sizeof(b));
  return b;
}

// This lane's number, counted anew behind an opaque zero, for the same reason.
__device__ __forceinline__ int late_lane() {
  uint32_t zero = 0;
  launder(zero);
  return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
}

// The scalar registers of a buffer resource are written: five wait states until a load
// may read them, which the compiler does not count for loads in inline assembly.
__device__ __forceinline__ void settle(i32x4_t& a) { asm volatile("s_nop 4" : "+s"(a)); }
__device__ __forceinline__ void settle(i32x4_t& a, i32x4_t& b) {
  asm volatile("s_nop 4" : "+s"(a), "+s"(b));
}

// Row r of a unit; rows behind the last are the last row once more: they see what it
// sees and give what it gives.
struct RowAt {
  uint32_t t, h;  // token from the unit's first on, head in the group
};
__device__ __forceinline__ RowAt row_at(const PackedArgs& a, const PackedItem& it, int r) {
  const int x = it.head0 + (r < it.rows ? r : it.rows - 1);
  const int t = divide(x, a.by_G);
  return {(uint32_t)t, (uint32_t)(x - t * a.G)};
}
// Element offset of a row in a view (q and o: strides below 2^31, see abi_packed.cpp).
__device__ __forceinline__ int64_t row_offset(const PackedArgs& a, const PackedItem& it,
                                              const RowAt& at, int kvh, int64_t token, int64_t head) {
  const int64_t base = it.q_row * token + (int64_t)(kvh * a.G) * head;
  return base + (int64_t)((uint64_t)at.t * (uint32_t)token + (uint64_t)at.h * (uint32_t)head);
}
// Keys of the unit that its token t sees.
__device__ __forceinline__ int keys_seen(const PackedItem& it, int t) {
  const int seen = it.seen + t;
  return seen < it.keys ? seen : it.keys;
}
// Keys that every row from r on sees (rows see no fewer than those before them).
__device__ __forceinline__ int seen_from(const PackedArgs& a, const PackedItem& it, int r) {
  return keys_seen(it, divide(it.head0 + (r < it.rows ? r : it.rows - 1), a.by_G));
}

// A lane's row: its query operand, and how many of the unit's keys it sees.
template <int D>
struct Row {
  bf16x8_t q[D / 16];
  int left;
};
template <int D>
__device__ __forceinline__ Row<D> row_of(const PackedArgs& a, const PackedItem& it, const RowAt& at,
                                         int kvh, int g) {
  Row<D> r;
  r.left = keys_seen(it, (int)at.t);
  const __bf16* qp = static_cast<const __bf16*>(a.q) + row_offset(a, it, at, kvh, a.qt, a.qh) + 8 * g;
#pragma unroll
  for (int st = 0; st < D / 16; ++st)
    r.q[st] = *reinterpret_cast<const bf16x8_t*>(qp + 16 * st);
  return r;
}

// Per-lane global offsets, inside a sub-tile, of the direct load that fills bytes
// o .. o + 15 of its LDS image (the images of sparse_fwd.hip, the caller's row strides).
template <int D>
__device__ __forceinline__ uint32_t k_offset(int o, uint32_t stride) {
  using C = FwdCfg<D, 32, 32>;
  const int r = o / C::KROW;
  return r * stride + (kswz<D, 32, 32>(r, (o % C::KROW) >> 4) << 4);
}
template <int D>
__device__ __forceinline__ uint32_t v_offset(int o, uint32_t stride) {
  using C = FwdCfg<D, 32, 32>;
  const int rem = o % C::VPC;
  return (4 * (o / C::VPC) + ((rem >> 6) & 3)) * stride + (rem >> 8) * 64 + (rem & 63);
}

// LDS addresses of a lane's operand reads in the K image (k-step st) or V image at `at`.
template <int D>
__device__ __forceinline__ uint32_t k_operand(uint32_t at, int lane, int st) {
  using C = FwdCfg<D, 32, 32>;
  return at + (lane & 31) * C::KROW + (kswz<D, 32, 32>(lane & 31, 2 * st + (lane >> 5)) << 4);
}
template <int D>
__device__ __forceinline__ uint32_t v_operand(uint32_t at, int lane) {
  using C = FwdCfg<D, 32, 32>;
  return at + (lane >> 5) * C::VPC + ((lane >> 2) & 3) * 64 + ((lane >> 4) & 1) * 32 +
         (lane & 3) * 8;
}

// Waits of one wave: until at most N of its memory operations are outstanding; until its
// LDS reads have returned.  Neither lets a memory access move across.
template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void lds_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// One 32-key sub-tile of a unit that is done again because its result was not finite
// (K and V images at kbase and vbase in LDS): values that are not finite stay out of the
// matrix products of a sub-tile that some row does not see whole, and are added, key by
// key, to the rows that see them.  pw: 2 KiB of this wave's for its probabilities.
template <int D>
__device__ __forceinline__ void slow_sub(uint32_t kbase, const char* vptr, uint32_t vbase,
                                         __bf16* pw, const Row<D>& row, int first, int whole,
                                         float scale_log2, int lane, f32x16_t* oacc, float& m_run,
                                         float& l_run) {
  using C = FwdCfg<D, 32, 32>;
  const int r = lane & 31, g = lane >> 5;
  f32x16_t cur = {};
  bf16x8_t pb[2];
#pragma unroll
  for (int st = 0; st < C::KS; ++st) {
    cur = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read16(k_operand<D>(kbase, lane, st)),
                                                  row.q[st], cur, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
  mask_left(cur, row.left - first, g);
  const float m_new = fmaxf(m_run, sub_max(cur) * scale_log2);
  const float alpha = fast_exp2(m_run - m_new);
  m_run = m_new;
#pragma unroll
  for (int db = 0; db < C::DB; ++db) oacc[db] *= alpha;
  l_run = l_run * alpha + softmax_sub(cur, scale_log2, m_run, pb);
  const bool all = whole >= first + 32;  // every row sees every key of the sub-tile
  // (K's image is read: the probabilities may overwrite it)
  lds_reads_done();
#pragma unroll
  for (int st = 0; st < 2; ++st) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      pw[(16 * st + 4 * g + (e & 3) + 8 * (e >> 2)) * 32 + r] = pb[st][e];
#pragma unroll
    for (int db = 0; db < C::DB; ++db) {
      bf16x8_t v = read_v<D, 32, 32>(v_operand<D>(vbase, lane), st, db);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = all || finite((float)v[e]) ? v[e] : (__bf16)0.f;
      oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pb[st], oacc[db], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (all) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll 1
  for (int key = 0; key < 32; ++key) {
    const float p = (float)pw[key * 32 + r];
    const bool sees = first + key < row.left;
    const char* vrow = vptr + (key >> 2) * C::VPC + (key & 3) * 64 + g * 8;
#pragma unroll
    for (int db = 0; db < C::DB; ++db)
#pragma unroll
      for (int qd = 0; qd < 4; ++qd) {
        const bf16x4_t v = *reinterpret_cast<const bf16x4_t*>(vrow + db * 256 + qd * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (sees && !finite((float)v[e])) oacc[db][4 * qd + e] += p * (float)v[e];
        __builtin_amdgcn_sched_barrier(0);  // (few registers: nothing here is in a hurry)
      }
  }
}

// Whether a result holds a value that is not finite.
template <int DB>
__device__ __forceinline__ bool not_finite(const f32x16_t* oacc) {
  float bad = 0.f;  // becomes NaN
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int t = 0; t < 16; ++t) bad = __builtin_fmaf(oacc[db][t], 0.f, bad);
  return __ballot(bad != 0.f) != 0;
}

// Unit of this workgroup: (unit, key head), the heads of a unit side by side.
__device__ __forceinline__ PackedItem unit_of(const PackedArgs& a, int* kvh) {
  const int unit = divide((int)blockIdx.x, a.by_H_kv);
  *kvh = (int)blockIdx.x - unit * a.H_kv;
  return a.items[unit];
}
__device__ __forceinline__ const char* first_key(const void* x, const PackedItem& it, int64_t token,
                                                 int64_t head, int kvh) {
  return reinterpret_cast<const char*>(static_cast<const __bf16*>(x) + it.k_row * token +
                                       kvh * head);
}

// Where a row's output goes: bytes from o, elements from lse.
struct RowOut {
  int64_t at, lse;
};
__device__ __forceinline__ RowOut row_out(const PackedArgs& a, const PackedItem& it, const RowAt& at,
                                          int kvh) {
  RowOut r;
  r.at = 2 * row_offset(a, it, at, kvh, a.ot, a.oh);
  r.lse = 0;
  if (a.lse != nullptr) r.lse = (kvh * a.G + (int64_t)at.h) * a.lse_head + it.q_row + at.t;
  return r;
}

// The same of a row's partial result: elements of part_o and part_ml.
template <int D>
__device__ __forceinline__ RowOut part_out(const PackedArgs& a, const PackedItem& it, int r, int kvh) {
  const int64_t at = (int64_t)(it.part + r) * a.H_kv + kvh;
  return {at * D, 2 * at};
}

constexpr int NW = kPackedWaves[1];  // waves of a workgroup

// LDS of a workgroup.
template <int D>
struct PackedLds {
  // tile: the rings; few rows: each wave's K and V slot, then its O
  static constexpr int BYTES = 2 * FwdCfg<D, 32 * NW, 32>::RING;
  static_assert(BYTES == NW * 2 * FwdCfg<D, 32, 32>::SUB, "one size for both");
  __attribute__((aligned(1024))) char smem[BYTES];
  // where each row's output goes: found with its query, so that the end of the kernel
  // neither divides nor waits for the plan
  RowOut out[32 * NW];
  float ml[NW][32][2];
};

// A tile of 128 rows of one sequence against its keys or a part of them: four waves of 32
// rows.
template <int D>
__device__ __forceinline__ void tile_unit(const PackedArgs& a, PackedLds<D>& lds) {
  constexpr int BLK = 32 * NW, BK = 32;
  using C = FwdCfg<D, BLK, BK>;
  constexpr int R = C::R;
  char* const smem = lds.smem;
  RowOut* const out = lds.out;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);

  f32x16_t oacc[C::DB];
#pragma unroll
  for (int db = 0; db < C::DB; ++db) oacc[db] = f32x16_t{};
  float m_run = kNegBig;  // max used for exp2 (log2 units)
  float l_run = 0.f;      // this lane's share of the row sum
  int hidden;             // keys of the unit that some row does not see, if > 0
  int used;               // rows of the sequence from this wave's first on
  bool partial;           // not all of the sequence's keys: the result is joined later
  {
    const int lane = threadIdx.x & 63;
    const int g = lane >> 5;
    int kvh;
    const PackedItem it = unit_of(a, &kvh);
    if (!inside(a, it, BLK)) return;
    const int n = it.keys;
    hidden = n - it.seen;
    const int S = ((n + 31) / 32 + 1) & ~1;  // sub-tiles, a multiple of the loop's half
    const char* kb = first_key(a.k, it, a.kt, a.kh, kvh);
    const char* vb = first_key(a.v, it, a.vt, a.vh, kvh);
    const uint32_t ks = (uint32_t)a.kt * 2, vs = (uint32_t)a.vt * 2;
    const float scale_log2 = a.scale_log2;
    uint32_t koffs[C::LPW], voffs[C::LPW];
#pragma unroll
    for (int u = 0; u < C::LPW; ++u) {
      koffs[u] = k_offset<D>((w * C::LPW + u) * 1024 + lane * 16, ks);
      voffs[u] = v_offset<D>((w * C::LPW + u) * 1024 + lane * 16, vs);
    }
    if (S > 0) {
      Stream<D> kf(kb, n, ks, 0), vf(vb, n, vs, 0);
#pragma unroll
      for (int y = 0; y < R; ++y) {
        i32x4_t krs = kf.next(), vrs = vf.next();
        settle(krs, vrs);
#pragma unroll
        for (int u = 0; u < C::LPW; ++u) {
          dma16(lds0 + y * C::SUB + (w * C::LPW + u) * 1024, krs, koffs[u], 0);
          if (y < R - 2)
            dma16(lds0 + C::RING + y * C::SUB + (w * C::LPW + u) * 1024, vrs, voffs[u], 0);
        }
      }
    }
    const RowAt at = row_at(a, it, w * 32 + (lane & 31));
    const Row<D> row = row_of<D>(a, it, at, kvh, g);
    partial = it.part >= 0;
    if (g == 0)
      out[w * 32 + lane] = partial ? part_out<D>(a, it, w * 32 + lane, kvh) : row_out(a, it, at, kvh);
    used = it.rows - w * 32;
    const int left = row.left;
    const int whole = seen_from(a, it, w * 32);  // keys every row of the wave sees
    uint32_t ka[C::KS], va = v_operand<D>(lds0 + C::RING, lane);
#pragma unroll
    for (int st = 0; st < C::KS; ++st) ka[st] = k_operand<D>(lds0, lane, st);
    f32x16_t sc[2];
    bf16x8_t pb[2][2];

    if (S > 0) {
      for (int z = (w * 64 + lane) * 16; z < C::SUB; z += 64 * NW * 16)
        *reinterpret_cast<f32x4_t*>(smem + C::RING + (R - 1) * C::SUB + z) = f32x4_t{};
#pragma unroll
      for (int a2 = 0; a2 < 2; ++a2)
#pragma unroll
        for (int st = 0; st < 2; ++st) pb[a2][st] = bf16x8_t{};
      wait_vm_barrier<0>();
      mfma_pair<D, BLK, BK, true, false>(ka, 0, row.q, sc[0], va, 0, pb[1], oacc);
      // the first reference is the first sub-tile's max
      if (whole < 32) mask_left(sc[0], left, g);
      m_run = fmaxf(m_run, sub_max(sc[0]) * scale_log2);

      // sub-iteration s = R u + H of the block-sparse forward: scores of s + 1, softmax
      // of s, P V of s - 1; K slot H takes sub-tile s + R, V slot (H + R - 2) % R sub-tile
      // s + R - 2 (behind the end of the keys: zeros)
      Stream<D> kf(kb, n, ks, R), vf(vb, n, vs, R - 2);
      auto sub_iter = [&](auto hh, int u) {
        constexpr int H = decltype(hh)::value;
        const int s = R * u + H;
        f32x16_t& cur = sc[H & 1];
        f32x16_t& nxt = sc[(H + 1) & 1];
#pragma unroll
        for (int st = 0; st < C::KS; ++st) launder(ka[st]);
        launder(va);
        // (opaque, so that the loads' LDS addresses are not kept in a register each)
        uint32_t ring = lds0 + w * C::LPW * 1024;
        asm volatile("" : "+s"(ring));
        i32x4_t krs = kf.next(), vrs = vf.next();
        settle(krs, vrs);
        wait_vm_barrier<(R - 2) * 2 * C::LPW>();
        auto issue = [&](int t) {
          if (t < C::LPW) {
            dma16(ring + H * C::SUB + t * 1024, krs, koffs[t], 0);
          } else {
            const int z = t - C::LPW;
            dma16(ring + C::RING + ((H + R - 2) % R) * C::SUB + z * 1024, vrs, voffs[z], 0);
          }
        };
        if (whole < 32 * (s + 1)) mask_left(cur, left - 32 * s, g);
        __builtin_amdgcn_s_setprio(1);
        float ls = pipeline_step<D, BLK, BK, C::LEAD, 2 * C::LPW>(
            ka, ((H + 1) % R) * C::SUB, row.q, nxt, va, ((H + R - 1) % R) * C::SUB,
            pb[(H + 1) & 1], oacc, cur, scale_log2, m_run, pb[H & 1], issue);
        __builtin_amdgcn_s_setprio(0);
        if (__ballot(!(ls <= kSumBound)) != 0) {
          const float m_new = fmaxf(m_run, sub_max(cur) * scale_log2);
          const float alpha = fast_exp2(m_run - m_new);
          m_run = m_new;
          l_run *= alpha;
#pragma unroll
          for (int db = 0; db < C::DB; ++db) oacc[db] *= alpha;
          ls = softmax_sub(cur, scale_log2, m_run, pb[H & 1]);
        }
        l_run += ls;
      };
      using I0 = std::integral_constant<int, 0>;
      using I1 = std::integral_constant<int, 1>;
      using I2 = std::integral_constant<int, 2>;
      using I3 = std::integral_constant<int, 3>;
      static_assert(R == 4, "loop body written for a ring of 4");
      for (int u = 0;; ++u) {
        sub_iter(I0{}, u);
        sub_iter(I1{}, u);
        if (R * u + 2 >= S) break;
        sub_iter(I2{}, u);
        sub_iter(I3{}, u);
        if (R * (u + 1) >= S) break;
      }
      // P V of the last sub-tile (odd), whose slot the last two sub-iterations' loads are
      // not in; then those are waited out before LDS serves another purpose
      wait_vm_barrier<(R - 2) * 2 * C::LPW>();
      mfma_pair<D, BLK, BK, false, true>(ka, 0, row.q, sc[0], va,
                                         (uint32_t)(((S - 1) % R) * C::SUB), pb[1], oacc);
      wait_vm_barrier<0>();
    }
  }

  const int el = late_lane();
  const int er = el & 31, eg = el >> 5;
  if (hidden > 0) {
    // some row does not see some key of the unit: has a value that is not finite spread?
    const bool mine = not_finite<C::DB>(oacc);
    int* const flag = reinterpret_cast<int*>(smem + C::RING);  // (no output passes there)
    if (el == 0) flag[w] = mine;
    __syncthreads();
    bool redo = false;
#pragma unroll
    for (int z = 0; z < NW; ++z) redo = redo || flag[z] != 0;
    if (redo) {
      const PackedArgs b = late_args();
      int kvh;
      const PackedItem it = unit_of(b, &kvh);
      const Row<D> row = row_of<D>(b, it, row_at(b, it, w * 32 + er), kvh, eg);
      const int whole = seen_from(b, it, w * 32);
      const uint32_t ks = (uint32_t)b.kt * 2, vs = (uint32_t)b.vt * 2;
#pragma unroll
      for (int db = 0; db < C::DB; ++db) oacc[db] = f32x16_t{};
      m_run = kNegBig;
      l_run = 0.f;
      __bf16* const pw = reinterpret_cast<__bf16*>(smem + C::SUB) + w * 32 * 32;
      static_assert(C::SUB + NW * 2048 <= C::RING, "the probabilities fit behind K slot 0");
      Stream<D> kf(first_key(b.k, it, b.kt, b.kh, kvh), it.keys, ks, 0);
      Stream<D> vf(first_key(b.v, it, b.vt, b.vh, kvh), it.keys, vs, 0);
      for (int s = 0; 32 * s < it.keys; ++s) {
        i32x4_t krs = kf.next(), vrs = vf.next();
        settle(krs, vrs);
        lds_read_barrier();
#pragma unroll 1
        for (int u = 0; u < C::LPW; ++u) {
          const int o = (w * C::LPW + u) * 1024;
          dma16(lds0 + o, krs, k_offset<D>(o + el * 16, ks), 0);
          dma16(lds0 + C::RING + o, vrs, v_offset<D>(o + el * 16, vs), 0);
        }
        wait_vm_barrier<0>();
        slow_sub<D>(lds0, smem + C::RING, lds0 + C::RING, pw, row, 32 * s, whole, b.scale_log2, el,
                    oacc, m_run, l_run);
      }
      lds_read_barrier();
    }
  }

  const PackedArgs b = late_args();
  const float l_tot = add_partner(l_run);
  if (partial) {
    if (er >= used) return;
    const RowOut to = out[w * 32 + er];
    float* const po = b.part_o + to.at + 4 * eg;
#pragma unroll
    for (int db = 0; db < C::DB; ++db)
#pragma unroll
      for (int qd = 0; qd < 4; ++qd) {
        f32x4_t v;
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = oacc[db][qd * 4 + u];
        *reinterpret_cast<f32x4_t*>(po + db * 32 + qd * 8) = v;
      }
    if (eg == 0) *reinterpret_cast<f32x2_t*>(b.part_ml + to.lse) = f32x2_t{m_run, l_tot};
    return;
  }
  const float inv = l_tot == 0.f ? 0.f : 1.0f / l_tot;
  // O leaves through this wave's part of the K ring, which no wave reads any more, so
  // that a store instruction writes whole rows
  char* const ot = smem + w * 32 * C::KROW;
#pragma unroll
  for (int db = 0; db < C::DB; ++db)
#pragma unroll
    for (int qd = 0; qd < 4; ++qd) {
      f32x4_t v;
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = oacc[db][qd * 4 + u] * inv;
      *reinterpret_cast<bf16x4_t*>(ot + er * C::KROW +
                                   (kswz<D, BLK, BK>(er, db * 4 + qd) << 4) + eg * 8) =
          __builtin_convertvector(v, bf16x4_t);
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  // (a whole tile's stores are not tested, and a ragged one's last row is written once)
  const RowOut* const ro = out + w * 32 + el * 16 / C::KROW;
  char* const ob = static_cast<char*>(b.o) + (el * 16 % C::KROW);
  auto store = [&](int z) {
    const int r = (z + el * 16) / C::KROW, c = (el * 16 % C::KROW) >> 4;
    *reinterpret_cast<f32x4_t*>(ob + ro[z / C::KROW].at) = *reinterpret_cast<const f32x4_t*>(
        ot + r * C::KROW + (kswz<D, BLK, BK>(r, c) << 4));
  };
  if (used >= 32) {
#pragma unroll
    for (int z = 0; z < C::SUB; z += 1024) store(z);
  } else {
#pragma unroll
    for (int z = 0; z < C::SUB; z += 1024)
      if ((z + el * 16) / C::KROW < used) store(z);
  }
  if (b.lse != nullptr && eg == 0 && er < used)
    b.lse[out[w * 32 + er].lse] = l_tot == 0.f ? -INFINITY : (m_run + __log2f(l_tot)) * kLn2;
}

// A part of the keys of a sequence of few rows: its rows fit one 32-row tile, and four
// waves take the part's sub-tiles in turn, each through one K and one V slot of its own,
// so that the loop has no barrier: K's slot is refilled while the softmax runs, V's while
// the next scores do.  The waves' states are merged in LDS in wave order.
//
// Bound: HBM.  Two workgroups a CU (d = 128) keep 128 KiB in flight there.
template <int D>
__device__ __forceinline__ void few_unit(const PackedArgs& a, PackedLds<D>& lds) {
  using C = FwdCfg<D, 32, 32>;
  constexpr int LD = C::LPW;  // loads of a sub-tile
  char* const smem = lds.smem;
  RowOut* const out = lds.out;
  auto& ml = lds.ml;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int r32 = lane & 31, g = lane >> 5;
  const uint32_t lds0 =
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + w * 2 * C::SUB;
  char* const vptr = smem + w * 2 * C::SUB + C::SUB;
  int kvh;
  const PackedItem it = unit_of(a, &kvh);
  if (!inside(a, it, 32)) return;
  const int n = it.keys;
  const char* kb = first_key(a.k, it, a.kt, a.kh, kvh);
  const char* vb = first_key(a.v, it, a.vt, a.vh, kvh);
  const uint32_t ks = (uint32_t)a.kt * 2, vs = (uint32_t)a.vt * 2;
  uint32_t koffs[LD], voffs[LD];
#pragma unroll
  for (int u = 0; u < LD; ++u) {
    koffs[u] = k_offset<D>(u * 1024 + lane * 16, ks);
    voffs[u] = v_offset<D>(u * 1024 + lane * 16, vs);
  }
  auto load_k = [&](int s) {
    i32x4_t rs = Stream<D>(kb, n, ks, s).next();
    settle(rs);
#pragma unroll
    for (int u = 0; u < LD; ++u) dma16(lds0 + u * 1024, rs, koffs[u], 0);
  };
  auto load_v = [&](int s) {
    i32x4_t rs = Stream<D>(vb, n, vs, s).next();
    settle(rs);
#pragma unroll
    for (int u = 0; u < LD; ++u) dma16(lds0 + C::SUB + u * 1024, rs, voffs[u], 0);
  };
  if (32 * w < n) {
    load_k(w);
    load_v(w);
  }
  const RowAt row_in = row_at(a, it, r32);
  Row<D> row = row_of<D>(a, it, row_in, kvh, g);
  // (waited for here, not inside the loop, where the wait would cover the loads in flight)
#pragma unroll
  for (int st = 0; st < C::KS; ++st) asm volatile("" : "+v"(row.q[st]));
  if (w == 0 && g == 0) out[lane] = row_out(a, it, row_in, kvh);
  const int whole = seen_from(a, it, 0);
  f32x16_t oacc[C::DB];
#pragma unroll
  for (int db = 0; db < C::DB; ++db) oacc[db] = f32x16_t{};
  float m_run = kNegBig, l_run = 0.f;
  for (int s = w; 32 * s < n; s += NW) {
    wait_vm<LD>();  // K is there (V's loads are the last)
    f32x16_t cur = {};
#pragma unroll
    for (int st = 0; st < C::KS; ++st)
      cur = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read16(k_operand<D>(lds0, lane, st)),
                                                    row.q[st], cur, 0, 0, 0);
    lds_reads_done();
    load_k(s + NW);  // (behind the end: zeros)
    if (whole < 32 * (s + 1)) mask_left(cur, row.left - 32 * s, g);
    const float m_new = fmaxf(m_run, sub_max(cur) * a.scale_log2);
    if (__ballot(m_new > m_run) != 0) {
      const float alpha = fast_exp2(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < C::DB; ++db) oacc[db] *= alpha;
    }
    bf16x8_t pb[2];
    l_run += softmax_sub(cur, a.scale_log2, m_run, pb);
    wait_vm<LD>();  // V is there
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int db = 0; db < C::DB; ++db)
        oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            read_v<D, 32, 32>(v_operand<D>(lds0 + C::SUB, lane), st, db), pb[st], oacc[db], 0, 0, 0);
    lds_reads_done();
    load_v(s + NW);
  }
  wait_vm<0>();
  if (n > it.seen && not_finite<C::DB>(oacc)) {
    // some row does not see some key: this wave's sub-tiles again, see slow_sub
#pragma unroll
    for (int db = 0; db < C::DB; ++db) oacc[db] = f32x16_t{};
    m_run = kNegBig;
    l_run = 0.f;
    for (int s = w; 32 * s < n; s += NW) {
      lds_reads_done();
      load_k(s);
      load_v(s);
      wait_vm<0>();
      slow_sub<D>(lds0, vptr, lds0 + C::SUB, reinterpret_cast<__bf16*>(vptr - C::SUB), row, 32 * s,
                  whole, a.scale_log2, lane, oacc, m_run, l_run);
    }
    lds_reads_done();
  }

  // the waves' states through LDS: O of wave w, [row][d] in 16-byte chunks swizzled by
  // row, over its own slots
  const float l_tot = add_partner(l_run);
  const int rows = it.rows;
  constexpr int CH = D / 4;  // chunks of a row
  auto chunk = [&](int wave, int r, int c) {
    return reinterpret_cast<f32x4_t*>(smem + wave * 2 * C::SUB + (r * CH + (c ^ (r % CH))) * 16);
  };
  if (r32 < rows) {
#pragma unroll
    for (int db = 0; db < C::DB; ++db)
#pragma unroll
      for (int qd = 0; qd < 4; ++qd) {
        f32x4_t v;
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = oacc[db][qd * 4 + u];
        *chunk(w, r32, db * 8 + qd * 2 + g) = v;
      }
    if (g == 0) {
      ml[w][r32][0] = m_run;
      ml[w][r32][1] = l_tot;
    }
  }
  __syncthreads();
  const int used = rows < 32 ? rows : 32;
  for (int i = threadIdx.x; i < used * CH; i += 64 * NW) {
    const int r = i / CH, c = i % CH;
    float m = kNegBig, l = 0.f;
#pragma unroll
    for (int y = 0; y < NW; ++y) m = fmaxf(m, ml[y][r][0]);
    f32x4_t acc = {};
#pragma unroll
    for (int y = 0; y < NW; ++y) {
      const float f = fast_exp2(ml[y][r][0] - m);
      l = __builtin_fmaf(ml[y][r][1], f, l);
      const f32x4_t v = *chunk(y, r, c);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(v[e], f, acc[e]);
    }
    if (it.part >= 0) {
      const int64_t at = (int64_t)(it.part + r) * a.H_kv + kvh;
      *reinterpret_cast<f32x4_t*>(a.part_o + at * D + 4 * c) = acc;
      if (c == 0) *reinterpret_cast<f32x2_t*>(a.part_ml + 2 * at) = f32x2_t{m, l};
    } else {
      const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] *= inv;
      *reinterpret_cast<bf16x4_t*>(static_cast<char*>(a.o) + out[r].at + 8 * c) =
          __builtin_convertvector(acc, bf16x4_t);
      if (a.lse != nullptr && c == 0)
        a.lse[out[r].lse] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
    }
  }
}

// Waves per SIMD the registers are cut for, as in the block-sparse forward.
template <int D>
constexpr int packed_waves_per_simd() {
  return D == 64 ? 4 : 2;
}

// Tiles come first in a plan, then few-row parts: each kind in a kernel of its own, or
// both in one (kTogether).
constexpr int kTiles = 1, kFew = 2;
template <int D, int KINDS>
__global__ void __launch_bounds__(64 * NW)
    __attribute__((amdgpu_waves_per_eu(KINDS == kFew ? 2 : packed_waves_per_simd<D>())))
    packed_bf16_kernel(const PackedArgs a) {
  __shared__ PackedLds<D> lds;
  if (KINDS == kTiles || (KINDS != kFew && (int)blockIdx.x < a.n_tiles * a.H_kv))
    tile_unit<D>(a, lds);
  else
    few_unit<D>(a, lds);
}

// Rows whose keys were split: up to kFewParts parts a wave per row and key head, more
// (plan order: first) a workgroup, whose wave w takes parts w, w + 8, ... and whose states
// are then merged in order.  Lane t holds the max and sum of the wave's t-th part; the
// outputs, rescaled to the wave's max, are added in order, and their loads do not wait
// for the weights.
static_assert(kMostParts / kJoinWaves <= 64 && kFewParts <= 64, "a lane for each part of a wave");

// o (un-normalised), max and sum of parts at(0) .. at(n - 1); m, f: see above.
template <int D, typename At>
__device__ __forceinline__ float join_wave(const PackedArgs& a, At&& at, int n, int lane, float& m,
                                           float* acc) {
  constexpr int PL = D / 64;  // values per lane
  constexpr int U = 8;        // outputs in flight
  f32x2_t mine = {kNegBig, 0.f};
  if (lane < n) mine = *reinterpret_cast<const f32x2_t*>(a.part_ml + 2 * at(lane));
  m = kNegBig;
  float f = 0.f;
  for (int t0 = 0; t0 < n; t0 += U) {
    float po[U][PL];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* p = a.part_o + at(t0 + u < n ? t0 + u : 0) * D + lane * PL;
#pragma unroll
      for (int e = 0; e < PL; ++e) po[u][e] = p[e];
    }
    if (t0 == 0) {
      m = mine[0];
#pragma unroll
      for (int x = 32; x >= 1; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
      f = fast_exp2(mine[0] - m);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float g = __shfl(f, t0 + u);
      if (t0 + u < n) {
#pragma unroll
        for (int e = 0; e < PL; ++e) acc[e] = __builtin_fmaf(po[u][e], g, acc[e]);
      }
    }
  }
  return wave_sum(f * mine[1]);
}

template <typename T, int D>
__global__ void __launch_bounds__(64 * kJoinWaves) join_kernel(const PackedArgs a) {
  constexpr int PL = D / 64;
  __shared__ float ml[kJoinWaves][2];
  __shared__ float opart[kJoinWaves][D];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wide = a.n_wide * a.H_kv;  // rows with a workgroup each
  const bool own = (int)blockIdx.x >= wide;
  const int64_t x = own ? wide + ((int64_t)blockIdx.x - wide) * kJoinWaves + w : blockIdx.x;
  if (x >= (int64_t)a.n_joins * a.H_kv) return;  // (a whole wave of a workgroup without a barrier)
  const int unit = divide((int)x, a.by_H_kv);
  const int kvh = (int)x - unit * a.H_kv;
  const PackedJoin j = a.joins[unit];
  if (!inside(a, j) || (own && j.n > kFewParts)) return;
  const int64_t head = kvh * a.G + j.in_group;
  T* const op = static_cast<T*>(a.o) + j.q_row * a.ot + head * a.oh;
  float acc[PL] = {}, m;
  auto finish = [&](float l) {
    if (a.lse != nullptr && lane == 0 && (own || w == 0))
      a.lse[head * a.lse_head + j.q_row] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
    return l == 0.f ? 0.f : 1.0f / l;
  };
  if (own) {
    const float l = join_wave<D>(
        a, [&](int i) { return (int64_t)(j.part + (int64_t)i * j.step) * a.H_kv + kvh; }, j.n, lane, m, acc);
    const float inv = finish(l);
#pragma unroll
    for (int e = 0; e < PL; ++e) op[lane * PL + e] = (T)(acc[e] * inv);
    return;
  }
  const float lw = join_wave<D>(
      a,
      [&](int i) { return (int64_t)(j.part + (int64_t)(w + kJoinWaves * i) * j.step) * a.H_kv + kvh; },
      (j.n - w + kJoinWaves - 1) / kJoinWaves, lane, m, acc);
  if (lane == 0) {
    ml[w][0] = m;
    ml[w][1] = lw;
  }
#pragma unroll
  for (int e = 0; e < PL; ++e) opart[w][lane * PL + e] = acc[e];
  __syncthreads();
  m = kNegBig;
#pragma unroll
  for (int y = 0; y < kJoinWaves; ++y) m = fmaxf(m, ml[y][0]);
  float l = 0.f, wgt[kJoinWaves];
#pragma unroll
  for (int y = 0; y < kJoinWaves; ++y) {
    wgt[y] = fast_exp2(ml[y][0] - m);
    l = __builtin_fmaf(ml[y][1], wgt[y], l);
  }
  const float inv = finish(l);
  for (int e = threadIdx.x; e < D; e += 64 * kJoinWaves) {
    float o = 0.f;
#pragma unroll
    for (int y = 0; y < kJoinWaves; ++y) o = __builtin_fmaf(opart[y][e], wgt[y], o);
    op[e] = (T)(o * inv);
  }
}

template <int D, int KINDS>
void launch_units(const PackedArgs& a, int units, hipStream_t stream) {
  if (units > 0)
    hipLaunchKernelGGL((packed_bf16_kernel<D, KINDS>), dim3((uint32_t)units * a.H_kv),
                       dim3(64 * NW), 0, stream, a);
}

// Tiles of a call up to which both kinds share a launch at d = 128: it saves 3.4 us (10
// prompts of 1 to 1,024 tokens x 32 / 8 heads, 120 x 8 units: 31.3 us, in two launches
// 34.7), and the tiles are 2 % slower in it (12 heads x 8,192 dense: 370 / 361 us).  At
// d = 64, where a kernel of both spills, they are 10 to 15 % slower.
constexpr int64_t kTogether = 4096;

template <int D>
hipError_t launch(const PackedArgs& a, int n_few, hipStream_t stream) {
  if (D == 128 && a.n_tiles > 0 && n_few > 0 && (int64_t)a.n_tiles * a.H_kv <= kTogether) {
    launch_units<128, kTiles | kFew>(a, a.n_tiles + n_few, stream);
  } else {
    launch_units<D, kTiles>(a, a.n_tiles, stream);
    PackedArgs few = a;
    few.items += a.n_tiles;
    launch_units<D, kFew>(few, n_few, stream);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_bf16(int d, const PackedArgs& a, int n_few, hipStream_t stream) {
  if (d == 64) return launch<64>(a, n_few, stream);
  if (d == 128) return launch<128>(a, n_few, stream);
  return hipErrorInvalidValue;
}

hipError_t launch_packed_join(int d, bool bf16, const PackedArgs& a, hipStream_t stream) {
  if (a.n_joins == 0) return hipSuccess;
  const int64_t own = (int64_t)(a.n_joins - a.n_wide) * a.H_kv;
  const dim3 grid((uint32_t)(a.n_wide * a.H_kv + (own + kJoinWaves - 1) / kJoinWaves)),
      block(64 * kJoinWaves);
  if (bf16 && d == 64)
    hipLaunchKernelGGL((join_kernel<__bf16, 64>), grid, block, 0, stream, a);
  else if (bf16 && d == 128)
    hipLaunchKernelGGL((join_kernel<__bf16, 128>), grid, block, 0, stream, a);
  else if (d == 64)
    hipLaunchKernelGGL((join_kernel<float, 64>), grid, block, 0, stream, a);
  else if (d == 128)
    hipLaunchKernelGGL((join_kernel<float, 128>), grid, block, 0, stream, a);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace losa
