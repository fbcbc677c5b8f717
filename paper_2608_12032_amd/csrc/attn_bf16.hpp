// One wave's share of a bf16 attention stream on v_mfma_f32_32x32x16_bf16: shapes,
// LDS images, operand reads, and the sub-iteration that runs the scores of the next
// 32-key sub-tile and P V of the previous one in the shadow of the current one's
// softmax.  Used by the block-sparse forward and by the packed attention; the
// orientation, key order and images are explained in sparse_fwd.hip.
#pragma once

#include "common.hpp"

namespace losa {

namespace {

// Sub-tile slots per operand ring.
constexpr int kRing = 4;

template <int D, int BLK, int BK>
struct FwdCfg {
  static constexpr int NW = BLK / 32;                // waves per workgroup
  static constexpr int NT = NW * 64;                 // threads
  static constexpr int KS = D / 16;                  // k-steps of S^T = K Q^T
  static constexpr int DB = D / 32;                  // 32-row d sub-blocks of O^T
  static constexpr int NS = BK / 32;                 // 32-key sub-tiles per key block
  static constexpr int R = kRing;                    // slots per ring
  static constexpr int LEAD = 2;                     // MFMAs an LDS operand read leads by
  static constexpr int BPI = R / NS;                 // key blocks per unrolled loop pass
  static constexpr int SUB = 32 * D * 2;             // bytes of a K or V sub-tile
  static constexpr int RING = R * SUB;               // bytes of one ring
  static constexpr int LPW = SUB / (1024 * NW);      // 1 KiB wave loads per sub-tile
  static constexpr int KROW = D * 2;                 // bytes of a K row
  static constexpr int KCPR = KROW / 16;             // 16-byte chunks per K row
  static constexpr int KRPL = 256 / KROW;            // K rows per 256-byte line
  static constexpr int VPC = 8 * D;                  // bytes of a 4-key piece of a V sub-tile
  static_assert(SUB % (1024 * NW) == 0, "sub-tile must split into whole wave loads");
  static_assert(R % NS == 0 && R >= 4 && (R & 1) == 0, "ring holds whole key blocks");
  static_assert(KS == 2 * DB, "QK and PV steps alternate one to one");
};

// Swizzled chunk of K chunk c in sub-tile row `row`.
template <int D, int BLK, int BK>
__device__ __forceinline__ int kswz(int row, int c) {
  using C = FwdCfg<D, BLK, BK>;
  return c ^ ((row / C::KRPL) % C::KCPR);
}

// Keep a per-lane LDS base address opaque inside the loop, so that every
// operand read stays "base + immediate" instead of the compiler hoisting one
// precomputed address per (slot, k-step) into its own register.
__device__ __forceinline__ void launder(uint32_t& x) { asm volatile("" : "+v"(x)); }

// V^T operand (d rows 32 db .. + 31, 16-key step st) of the row-major V
// sub-tile at va.
template <int D, int BLK, int BK>
__device__ __forceinline__ bf16x8_t read_v(uint32_t va, int st, int db) {
  using C = FwdCfg<D, BLK, BK>;
  const uint32_t a = va + st * 4 * C::VPC + db * 256;
  return __builtin_shufflevector(lds_read_tr8(a), lds_read_tr8(a + 2 * C::VPC), 0, 1, 2, 3, 4, 5,
                                 6, 7);
}

// Unpipelined S^T = K Q^T of one sub-tile (QK) and/or O^T += V^T P^T of one
// sub-tile (PV); the prologue and the drain of the pipeline.  ka[st] is this
// lane's LDS address of its chunk for k-step st in K slot 0, va its address
// for key step 0, d block 0 in V slot 0; kimm / vimm select the slot.
template <int D, int BLK, int BK, bool QK, bool PV>
__device__ __forceinline__ void mfma_pair(const uint32_t* ka, uint32_t kimm, const bf16x8_t* qreg,
                                          f32x16_t& snext, uint32_t va, uint32_t vimm,
                                          const bf16x8_t* pprev, f32x16_t* o) {
  using C = FwdCfg<D, BLK, BK>;
  constexpr int NPV = 2 * C::DB;
#pragma unroll
  for (int i = 0; i < C::KS; ++i) {
    if constexpr (QK) {
      const bf16x8_t a = lds_read16(ka[i] + kimm);
      snext = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qreg[i], i == 0 ? f32x16_t{} : snext, 0,
                                                      0, 0);
    }
    if constexpr (PV) {
      if (i < NPV) {
        const int st = i / C::DB, db = i % C::DB;
        const bf16x8_t a = read_v<D, BLK, BK>(va + vimm, st, db);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pprev[st], o[db], 0, 0, 0);
      }
    }
  }
}

// Probabilities of one 32-key sub-tile for this lane's 16 scores against the
// running max m_run (log2 units): bf16-packed into pcur; returns their fp32 sum.
__device__ __forceinline__ float softmax_sub(const f32x16_t& cur, float scale_log2, float m_run,
                                             bf16x8_t* pcur) {
  f32x8_t p[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      p[h][e] = fast_exp2(__builtin_fmaf(cur[8 * h + e], scale_log2, -m_run));
    pcur[h] = __builtin_convertvector(p[h], bf16x8_t);
  }
  // two interleaved sums, started from the first two terms (the same values
  // and order as starting from +0, which the compiler cannot fold away)
  float ls0 = p[0][0], ls1 = p[0][1];
#pragma unroll
  for (int e = 2; e < 16; e += 2) {
    ls0 += p[e >> 3][e & 7];
    ls1 += p[e >> 3][(e & 7) + 1];
  }
  return ls0 + ls1;
}

// One pipelined sub-iteration, issued in a fixed order: NM = KS + 2*DB MFMAs
// alternate between S^T(next) = K Q^T (a KS-long dependent chain) and
// O^T += V^T P^T(prev) (2 k-steps x DB independent chains); each MFMA's LDS
// operand is read NPRE MFMAs ahead from a small register ring.  The softmax
// of the current sub-tile runs in their shadow: under each of the first NM/2
// MFMAs two scores are scaled (v_fma) and exponentiated (v_exp, a
// transcendental), under each of the last NM/2 the bf16 packs and the row
// sums.  The NL global->LDS loads of this sub-iteration (issue(t), t < NL)
// are spread evenly over the MFMAs instead of leaving in one burst, starting
// two MFMAs in, so that the sub-iteration's first operand reads reach LDS
// ahead of the loads' writes (1 % faster than starting at the first MFMA).
// sched_group_barrier fixes this order.
template <int D, int BLK, int BK, int NPRE, int NL, typename Issue>
__device__ __forceinline__ float pipeline_step(const uint32_t* ka, uint32_t kimm,
                                               const bf16x8_t* qreg, f32x16_t& snext,
                                               uint32_t va, uint32_t vimm,
                                               const bf16x8_t* pprev, f32x16_t* o, f32x16_t& cur,
                                               float scale_log2, float m_run, bf16x8_t* pcur,
                                               Issue&& issue) {
  using C = FwdCfg<D, BLK, BK>;
  constexpr int NM = C::KS + 2 * C::DB;
  static_assert(NM == 16 || NM == 8, "softmax split written for 8 or 16 MFMAs");
  static_assert(NL <= NM, "at most one load per MFMA");
  constexpr int EPM = 32 / NM;  // exponentials per MFMA in the first half
  auto read_op = [&](int i) -> bf16x8_t {
    if ((i & 1) == 0) return lds_read16(ka[i >> 1] + kimm);
    const int st = (i >> 1) / C::DB, db = (i >> 1) % C::DB;
    return read_v<D, BLK, BK>(va + vimm, st, db);
  };
  // load t is issued right after MFMA OFF + t * SP
  static_assert(NM % NL == 0, "loads spread evenly");
  constexpr int SP = NM / NL;
  constexpr int OFF = SP > 2 ? 2 : SP - 1;
  auto has_load = [&](int i) { return i >= OFF && (i - OFF) % SP == 0; };
  bf16x8_t ring[NPRE];
#pragma unroll
  for (int i = 0; i < NPRE; ++i) ring[i] = read_op(i);
  f32x8_t p[2];
#pragma unroll
  for (int i = 0; i < NM; ++i) {
    const bf16x8_t a = ring[i % NPRE];
    if ((i & 1) == 0) {
      const int st = i >> 1;
      snext = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qreg[st], st == 0 ? f32x16_t{} : snext,
                                                      0, 0, 0);
    } else {
      const int st = (i >> 1) / C::DB, db = (i >> 1) % C::DB;
      o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pprev[st], o[db], 0, 0, 0);
    }
    if (i + NPRE < NM) ring[i % NPRE] = read_op(i + NPRE);
    if (has_load(i)) issue((i - OFF) / SP);
    if (i < NM / 2) {
#pragma unroll
      for (int u = 0; u < EPM; ++u) {
        const int e = i * EPM + u;
        p[e >> 3][e & 7] = fast_exp2(__builtin_fmaf(cur[e], scale_log2, -m_run));
      }
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) pcur[h] = __builtin_convertvector(p[h], bf16x8_t);
  // two interleaved row sums, started from the first two terms (the same
  // values and order as starting from +0, which the compiler cannot fold)
  float ls0 = p[0][0], ls1 = p[0][1];
#pragma unroll
  for (int e = 2; e < 16; e += 2) {
    ls0 += p[e >> 3][e & 7];
    ls1 += p[e >> 3][(e & 7) + 1];
  }
  // fixed issue order: the NPRE lead reads; then per MFMA the next read, its
  // load if it has one, and either EPM (fma, exp) pairs or its share of the
  // 8 packs and 14 sums of the second half
  constexpr int TAIL = 22;
  __builtin_amdgcn_sched_group_barrier(0x100, NPRE + NPRE / 2, 0);
#pragma unroll
  for (int i = 0; i < NM; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (i + NPRE < NM) {  // a V operand takes two reads
      if (((i + NPRE) & 1) != 0)
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      else
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    if (has_load(i)) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);  // VMEM read
    if (i < NM / 2) {
      __builtin_amdgcn_sched_group_barrier(0x002, EPM, 0);  // v_fma
      __builtin_amdgcn_sched_group_barrier(0x400, EPM, 0);  // v_exp
    } else {
      __builtin_amdgcn_sched_group_barrier(0x002, (2 * TAIL + NM - 1) / NM, 0);  // packs / sums
    }
  }
  // pin the softmax results here: otherwise the compiler sinks the exp2 work
  // next to its consumers in the following sub-iteration, out of the shadow
  // of these MFMAs
  float ls = ls0 + ls1;
  asm volatile("" : "+v"(ls), "+v"(pcur[0]), "+v"(pcur[1]));
  return ls;
}

// Raw-score maximum of a 32-key sub-tile for this lane's query (both halves).
__device__ __forceinline__ float sub_max(const f32x16_t& s) {
  float m = s[0];
#pragma unroll
  for (int t = 1; t < 16; ++t) m = fmaxf(m, s[t]);
  return max_with_partner(m);
}

// Scores of sub-tile `part`'s keys at or beyond kvalid (block-relative) -> -inf.
__device__ __forceinline__ void mask_sub(f32x16_t& s, int part, int kvalid, int g) {
#pragma unroll
  for (int t = 0; t < 16; ++t) {
    const int key = part * 32 + ((t >> 2) << 3) + (g << 2) + (t & 3);
    if (key >= kvalid) s[t] = -INFINITY;
  }
}

}  // namespace

}  // namespace losa
