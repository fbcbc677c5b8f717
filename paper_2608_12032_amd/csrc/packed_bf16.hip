// Attention over packed sequences of different lengths, grouped heads, causal or
// not: bf16 in, fp32 accumulation on gfx950 MFMA.
//
// Mathematics.  Row (token i, head h) of a sequence with key head h / G:
//   O = sum_j softmax_j(scale q . k_j) v_j over the keys j it sees (causal:
//   j <= i + k_len - q_len), by the online softmax: running max, sum and O^T.
//
// Work unit.  One workgroup owns 32 NW rows of one sequence and key head and walks a
// range of its keys.  Rows are numbered token * G + head in group, so a tile's rows
// share their keys whatever G is: G heads of one token fill a tile where each alone
// would leave it nearly empty.  The plan lists the units, longest first.  Orientation,
// key order, LDS images, the two rings and the pipelined sub-iteration are those of
// the block-sparse forward (sparse_fwd.hip, attn_bf16.hpp); the stream is simply the
// unit's keys in order.
//
// Sequences of few rows (32 or fewer: single tokens with grouped heads) are bound by
// HBM, K and V read once, and have no rows to fill the chip with: their keys are split
// into parts (packed_plan.cpp), one wave each (NW = 1, its own rings), whose O, max and
// sum are joined in a fixed order by join_kernel.  How a sequence is split follows from
// its own lengths alone, so it gives the same bits alone and packed among others.
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

// Scores of sub-tile keys (this lane's 16) at or beyond `left` -> -inf.
__device__ __forceinline__ void mask_left(f32x16_t& s, int left, int g) {
#pragma unroll
  for (int t = 0; t < 16; ++t)
    if (((t >> 2) << 3) + (g << 2) + (t & 3) >= left) s[t] = -INFINITY;
}

// Bound on a lane's sum of 16 probabilities before the running max is raised, as in
// the block-sparse forward.
constexpr float kSumBound = 1048576.0f;

__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < INFINITY; }

// Buffer resource of sub-tile x (32 rows of D elements, `stride` bytes apart) of a
// range of n rows at base: rows at or beyond n read as 0.
template <int D>
__device__ __forceinline__ i32x4_t sub_rsrc(const char* base, uint32_t stride, int x, int n) {
  int left = n - 32 * x;
  left = left < 0 ? 0 : (left > 32 ? 32 : left);
  return rsrc_words(base + (int64_t)x * 32 * stride,
                    left == 0 ? 0u : (uint32_t)(left - 1) * stride + 2 * D);
}

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
__device__ __forceinline__ void settle(i32x4_t& rs) { asm volatile("s_nop 4" : "+s"(rs)); }

// A unit as its rows see it: keys that count, relative to c0.
struct Extent {
  int n;      // keys that some row sees
  int seen0;  // keys that every row sees
  int shift;  // causal: token i sees keys up to i + shift
};
template <int BLK>
__device__ __forceinline__ Extent extent(const PackedItem& it, int G, int causal) {
  Extent x;
  x.shift = it.k_len - it.q_len;
  int last = (it.row0 + BLK - 1) / G;
  last = last < it.q_len ? last : it.q_len - 1;
  const int top = causal && last + x.shift + 1 < it.c1 ? last + x.shift + 1 : it.c1;
  x.n = top > it.c0 ? top - it.c0 : 0;
  x.seen0 = causal ? it.row0 / G + x.shift + 1 - it.c0 : x.n;
  return x;
}

// A lane's row: its query operand, and how many of the unit's keys it sees.  Rows
// behind the last take Q = 0 and every key, and are not written.
template <int D>
struct Row {
  bf16x8_t q[D / 16];
  int left;
  bool valid;
};
template <int D>
__device__ __forceinline__ Row<D> row_of(const PackedArgs& a, const PackedItem& it, const Extent& x,
                                         int kvh, int row, int g) {
  Row<D> r;
  const int tok = row / a.G;
  r.valid = tok < it.q_len;
  r.left = x.n;
  if (a.causal && r.valid && tok + x.shift + 1 - it.c0 < x.n) r.left = tok + x.shift + 1 - it.c0;
  const int head = kvh * a.G + (r.valid ? row - tok * a.G : 0);
  const __bf16* qp = static_cast<const __bf16*>(a.q) + (it.q0 + (r.valid ? tok : 0)) * a.qt +
                     (int64_t)head * a.qh;
#pragma unroll
  for (int st = 0; st < D / 16; ++st)
    r.q[st] = r.valid ? *reinterpret_cast<const bf16x8_t*>(qp + 16 * st + 8 * g) : bf16x8_t{};
  return r;
}

// Keys seen by every row of the wave.
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) x = min(x, __shfl_xor(x, o));
  return __builtin_amdgcn_readfirstlane(x);
}

// Per-lane global offsets, inside a sub-tile, of the direct load that fills bytes
// o .. o + 15 of its LDS image (the images of sparse_fwd.hip, the caller's row strides).
template <int D, int BLK>
__device__ __forceinline__ uint32_t k_offset(int o, uint32_t stride) {
  using C = FwdCfg<D, BLK, 32>;
  const int r = o / C::KROW;
  return r * stride + (kswz<D, BLK, 32>(r, (o % C::KROW) >> 4) << 4);
}
template <int D, int BLK>
__device__ __forceinline__ uint32_t v_offset(int o, uint32_t stride) {
  using C = FwdCfg<D, BLK, 32>;
  const int rem = o % C::VPC;
  return (4 * (o / C::VPC) + ((rem >> 6) & 3)) * stride + (rem >> 8) * 64 + (rem & 63);
}

// LDS addresses of a lane's operand reads in K slot 0 (k-step st) and V slot 0.
template <int D, int BLK>
__device__ __forceinline__ uint32_t k_operand(uint32_t lds0, int lane, int st) {
  using C = FwdCfg<D, BLK, 32>;
  return lds0 + (lane & 31) * C::KROW + (kswz<D, BLK, 32>(lane & 31, 2 * st + (lane >> 5)) << 4);
}
template <int D, int BLK>
__device__ __forceinline__ uint32_t v_operand(uint32_t lds0, int lane) {
  using C = FwdCfg<D, BLK, 32>;
  return lds0 + C::RING + (lane >> 5) * C::VPC + ((lane >> 2) & 3) * 64 + ((lane >> 4) & 1) * 32 +
         (lane & 3) * 8;
}

// Waves per SIMD the registers are cut for, as in the block-sparse forward; the
// single waves of few-row units are limited by their rings (64 KiB at d = 128).
template <int D, int NW>
constexpr int packed_waves_per_simd() {
  return NW == 1 ? 1 : (D == 64 ? 4 : 2);
}

template <int D, int NW>
__global__ void __launch_bounds__(64 * NW)
    __attribute__((amdgpu_waves_per_eu(packed_waves_per_simd<D, NW>())))
    packed_bf16_kernel(const PackedArgs a) {
  constexpr int BLK = 32 * NW, BK = 32;
  using C = FwdCfg<D, BLK, BK>;
  constexpr int R = C::R;
  __shared__ __attribute__((aligned(1024))) char smem[2 * C::RING];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);

  f32x16_t oacc[C::DB];
#pragma unroll
  for (int db = 0; db < C::DB; ++db) oacc[db] = f32x16_t{};
  float m_run = kNegBig;  // max used for exp2 (log2 units)
  float l_run = 0.f;      // this lane's share of the row sum
  {
    const int lane = threadIdx.x & 63;
    const int g = lane >> 5;
    const int unit = (int)blockIdx.x / a.H_kv;
    const int kvh = (int)blockIdx.x - unit * a.H_kv;
    const PackedItem it = a.items[unit];
    // (a plan's units lie inside q and k; nothing is read or written for one that does not)
    if (it.q0 < 0 || it.q_len < 0 || it.q0 + it.q_len > a.q_rows || it.k0 < 0 || it.k_len < 0 ||
        it.k0 + it.k_len > a.k_rows || it.c0 < 0 || it.c1 > it.k_len || it.row0 < 0)
      return;
    const Extent x = extent<BLK>(it, a.G, a.causal);
    const int n = x.n;
    const int S = ((n + 31) / 32 + 1) & ~1;  // sub-tiles, a multiple of the loop's half
    const Row<D> row = row_of<D>(a, it, x, kvh, it.row0 + w * 32 + (lane & 31), g);
    const int left = row.left;
    const int whole = wave_min(left);
    const char* kb = reinterpret_cast<const char*>(static_cast<const __bf16*>(a.k) +
                                                   (it.k0 + it.c0) * a.kt + kvh * a.kh);
    const char* vb = reinterpret_cast<const char*>(static_cast<const __bf16*>(a.v) +
                                                   (it.k0 + it.c0) * a.vt + kvh * a.vh);
    const uint32_t ks = (uint32_t)a.kt * 2, vs = (uint32_t)a.vt * 2;
    const float scale_log2 = a.scale_log2;
    uint32_t ka[C::KS], va = v_operand<D, BLK>(lds0, lane);
#pragma unroll
    for (int st = 0; st < C::KS; ++st) ka[st] = k_operand<D, BLK>(lds0, lane, st);
    uint32_t koffs[C::LPW], voffs[C::LPW];
#pragma unroll
    for (int u = 0; u < C::LPW; ++u) {
      koffs[u] = k_offset<D, BLK>((w * C::LPW + u) * 1024 + lane * 16, ks);
      voffs[u] = v_offset<D, BLK>((w * C::LPW + u) * 1024 + lane * 16, vs);
    }
    f32x16_t sc[2];
    bf16x8_t pb[2][2];

    if (S > 0) {
#pragma unroll
      for (int y = 0; y < R; ++y) {
        i32x4_t krs = sub_rsrc<D>(kb, ks, y, n), vrs = sub_rsrc<D>(vb, vs, y, n);
        settle(krs);
        settle(vrs);
#pragma unroll
        for (int u = 0; u < C::LPW; ++u) {
          dma16(lds0 + y * C::SUB + (w * C::LPW + u) * 1024, krs, koffs[u], 0);
          if (y < R - 2)
            dma16(lds0 + C::RING + y * C::SUB + (w * C::LPW + u) * 1024, vrs, voffs[u], 0);
        }
      }
      for (int z = (w * 64 + lane) * 16; z < C::SUB; z += 64 * NW * 16)
        *reinterpret_cast<f32x4_t*>(smem + C::RING + (R - 1) * C::SUB + z) = f32x4_t{};
#pragma unroll
      for (int a2 = 0; a2 < 2; ++a2)
#pragma unroll
        for (int st = 0; st < 2; ++st) pb[a2][st] = bf16x8_t{};
      wait_vm_barrier<0>();
      mfma_pair<D, BLK, BK, true, false>(ka, 0, row.q, sc[0], va, 0, pb[1], oacc);

      // sub-iteration s = R u + H of the block-sparse forward: scores of s + 1, softmax
      // of s, P V of s - 1; K slot H takes sub-tile s + R, V slot (H + R - 2) % R sub-tile
      // s + R - 2 (behind the end of the keys: zeros)
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
        i32x4_t krs = sub_rsrc<D>(kb, ks, s + R, n);
        i32x4_t vrs = sub_rsrc<D>(vb, vs, s + R - 2, n);
        settle(krs);
        settle(vrs);
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

  const PackedArgs b = late_args();
  const int el = late_lane();
  const int er = el & 31, eg = el >> 5;
  const int unit = (int)blockIdx.x / b.H_kv;
  const int kvh = (int)blockIdx.x - unit * b.H_kv;
  const PackedItem it = b.items[unit];
  const Extent x = extent<BLK>(it, b.G, b.causal);
  const int rows = it.q_len * b.G - it.row0 - w * 32;  // rows from this wave's first on

  if (x.seen0 < x.n) {
    // some row does not see some key of the unit: has a value that is not finite spread?
    float bad = 0.f;  // becomes NaN
#pragma unroll
    for (int db = 0; db < C::DB; ++db)
#pragma unroll
      for (int t = 0; t < 16; ++t) bad = __builtin_fmaf(oacc[db][t], 0.f, bad);
    bool redo = __ballot(er < rows && bad != 0.f) != 0;
    if constexpr (NW > 1) {
      int* const flag = reinterpret_cast<int*>(smem + C::RING);  // (no output passes there)
      if (el == 0) flag[w] = redo;
      __syncthreads();
      redo = false;
#pragma unroll
      for (int z = 0; z < NW; ++z) redo = redo || flag[z] != 0;
    }
    if (redo) {
      const Row<D> row = row_of<D>(b, it, x, kvh, it.row0 + w * 32 + er, eg);
      const int left = row.left, whole = wave_min(left);
      const char* kb = reinterpret_cast<const char*>(static_cast<const __bf16*>(b.k) +
                                                     (it.k0 + it.c0) * b.kt + kvh * b.kh);
      const char* vb = reinterpret_cast<const char*>(static_cast<const __bf16*>(b.v) +
                                                     (it.k0 + it.c0) * b.vt + kvh * b.vh);
      const uint32_t va = v_operand<D, BLK>(lds0, el);
#pragma unroll
      for (int db = 0; db < C::DB; ++db) oacc[db] = f32x16_t{};
      m_run = kNegBig;
      l_run = 0.f;
      // this wave's probabilities of a sub-tile, [key][row], behind K slot 0
      __bf16* const pw = reinterpret_cast<__bf16*>(smem + C::SUB) + w * 32 * 32;
      static_assert(C::SUB + NW * 2048 <= C::RING, "the probabilities fit the K ring");
      for (int s = 0; 32 * s < x.n; ++s) {
        i32x4_t krs = sub_rsrc<D>(kb, (uint32_t)b.kt * 2, s, x.n);
        i32x4_t vrs = sub_rsrc<D>(vb, (uint32_t)b.vt * 2, s, x.n);
        settle(krs);
        settle(vrs);
        lds_read_barrier();
#pragma unroll 1
        for (int u = 0; u < C::LPW; ++u) {
          const int o = (w * C::LPW + u) * 1024;
          dma16(lds0 + o, krs, k_offset<D, BLK>(o + el * 16, (uint32_t)b.kt * 2), 0);
          dma16(lds0 + C::RING + o, vrs, v_offset<D, BLK>(o + el * 16, (uint32_t)b.vt * 2), 0);
        }
        wait_vm_barrier<0>();
        f32x16_t cur = {};
        bf16x8_t pb[2];
#pragma unroll
        for (int st = 0; st < C::KS; ++st) {
          cur = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              lds_read16(k_operand<D, BLK>(lds0, el, st)), row.q[st], cur, 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        mask_left(cur, left - 32 * s, eg);
        const float m_new = fmaxf(m_run, sub_max(cur) * b.scale_log2);
        const float alpha = fast_exp2(m_run - m_new);
        m_run = m_new;
#pragma unroll
        for (int db = 0; db < C::DB; ++db) oacc[db] *= alpha;
        l_run = l_run * alpha + softmax_sub(cur, b.scale_log2, m_run, pb);
        const bool all = whole >= 32 * (s + 1);  // every row sees every key of the sub-tile
#pragma unroll
        for (int st = 0; st < 2; ++st) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            pw[(16 * st + 4 * eg + (e & 3) + 8 * (e >> 2)) * 32 + er] = pb[st][e];
#pragma unroll
          for (int db = 0; db < C::DB; ++db) {
            bf16x8_t v = read_v<D, BLK, BK>(va, st, db);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = all || finite((float)v[e]) ? v[e] : (__bf16)0.f;
            oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pb[st], oacc[db], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        if (all) continue;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int key = 0; key < 32; ++key) {
          const float p = (float)pw[key * 32 + er];
          const bool sees = 32 * s + key < left;
          const char* vrow = smem + C::RING + (key >> 2) * C::VPC + (key & 3) * 64 + eg * 8;
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
      lds_read_barrier();
    }
  }

  const float l_tot = add_partner(l_run);
  if (it.part >= 0) {
    if (er < rows) {
      const int64_t at = (int64_t)(it.part + w * 32 + er) * b.H_kv + kvh;
      float* const po = b.part_o + at * D + 4 * eg;
#pragma unroll
      for (int db = 0; db < C::DB; ++db)
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
          f32x4_t v;
#pragma unroll
          for (int u = 0; u < 4; ++u) v[u] = oacc[db][qd * 4 + u];
          *reinterpret_cast<f32x4_t*>(po + db * 32 + qd * 8) = v;
        }
      if (eg == 0) *reinterpret_cast<f32x2_t*>(b.part_ml + 2 * at) = f32x2_t{m_run, l_tot};
    }
    return;
  }
  // O leaves through this wave's part of the K ring, which no wave reads any more, so
  // that a store instruction writes whole rows
  const float inv = l_tot == 0.f ? 0.f : 1.0f / l_tot;
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
#pragma unroll
  for (int z = 0; z < C::SUB; z += 1024) {
    const int r = (z + el * 16) / C::KROW, c = (el * 16 % C::KROW) >> 4;
    if (r >= rows) continue;
    const int gr = it.row0 + w * 32 + r, t = gr / b.G;
    __bf16* const op = static_cast<__bf16*>(b.o) + (it.q0 + t) * b.ot +
                       (int64_t)(kvh * b.G + (gr - t * b.G)) * b.oh;
    *reinterpret_cast<f32x4_t*>(op + 8 * c) =
        *reinterpret_cast<const f32x4_t*>(ot + r * C::KROW + (kswz<D, BLK, BK>(r, c) << 4));
  }
  if (b.lse != nullptr && eg == 0 && er < rows) {
    const int gr = it.row0 + w * 32 + er, t = gr / b.G;
    b.lse[(int64_t)(kvh * b.G + (gr - t * b.G)) * b.lse_head + it.q0 + t] =
        l_tot == 0.f ? -INFINITY : (m_run + __log2f(l_tot)) * kLn2;
  }
}

// Rows whose keys were split: one workgroup per row and key head takes the parts'
// common max, then their sums and outputs rescaled to it, each wave every fourth
// part, the waves added in order.
constexpr int kJoinWaves = 4;

template <typename T, int D>
__global__ void __launch_bounds__(64 * kJoinWaves) join_kernel(const PackedArgs a) {
  constexpr int PL = D / 64;  // values per lane
  __shared__ float red[kJoinWaves];
  __shared__ float lpart[kJoinWaves];
  __shared__ float opart[kJoinWaves][D];
  const int unit = (int)blockIdx.x / a.H_kv;
  const int kvh = (int)blockIdx.x - unit * a.H_kv;
  const PackedJoin j = a.joins[unit];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  auto at = [&](int i) { return (int64_t)(j.part + (int64_t)i * j.step) * a.H_kv + kvh; };
  float m = kNegBig;
  for (int i = threadIdx.x; i < j.n; i += 64 * kJoinWaves) m = fmaxf(m, a.part_ml[2 * at(i)]);
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
  if (lane == 0) red[w] = m;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kJoinWaves; ++x) m = fmaxf(m, red[x]);
  float l = 0.f, acc[PL] = {};
#pragma unroll 4
  for (int i = w; i < j.n; i += kJoinWaves) {
    const f32x2_t ml = *reinterpret_cast<const f32x2_t*>(a.part_ml + 2 * at(i));
    const float* po = a.part_o + at(i) * D + lane * PL;
    const float f = fast_exp2(ml[0] - m);
    l = __builtin_fmaf(ml[1], f, l);
#pragma unroll
    for (int e = 0; e < PL; ++e) acc[e] = __builtin_fmaf(po[e], f, acc[e]);
  }
  if (lane == 0) lpart[w] = l;
#pragma unroll
  for (int e = 0; e < PL; ++e) opart[w][lane * PL + e] = acc[e];
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int x = 0; x < kJoinWaves; ++x) l += lpart[x];
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const int64_t head = kvh * a.G + j.in_group;
  for (int e = threadIdx.x; e < D; e += 64 * kJoinWaves) {
    float o = 0.f;
#pragma unroll
    for (int x = 0; x < kJoinWaves; ++x) o += opart[x][e];
    static_cast<T*>(a.o)[j.q_row * a.ot + head * a.oh + e] = (T)(o * inv);
  }
  if (a.lse != nullptr && threadIdx.x == 0)
    a.lse[head * a.lse_head + j.q_row] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

template <int D>
hipError_t launch(const PackedArgs& a, int n_tiles, int n_few, hipStream_t stream) {
  if (n_tiles > 0)
    hipLaunchKernelGGL((packed_bf16_kernel<D, 4>), dim3((uint32_t)n_tiles * a.H_kv), dim3(256), 0,
                       stream, a);
  if (n_few > 0) {
    PackedArgs few = a;
    few.items += n_tiles;
    hipLaunchKernelGGL((packed_bf16_kernel<D, 1>), dim3((uint32_t)n_few * a.H_kv), dim3(64), 0,
                       stream, few);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_bf16(int d, const PackedArgs& a, int n_tiles, int n_few,
                              hipStream_t stream) {
  if (d == 64) return launch<64>(a, n_tiles, n_few, stream);
  if (d == 128) return launch<128>(a, n_tiles, n_few, stream);
  return hipErrorInvalidValue;
}

hipError_t launch_packed_join(int d, bool bf16, const PackedArgs& a, int n_joins,
                              hipStream_t stream) {
  if (n_joins == 0) return hipSuccess;
  const dim3 grid((uint32_t)n_joins * a.H_kv), block(64 * kJoinWaves);
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
