// Attention over packed sequences, fp32 inputs, on the fp32 matrix instructions: the
// mathematics, units and plan of packed_bf16.hip with the tiles of the fp32 path
// (f32_path.hip).  A wave takes one or two groups of 16 rows; the waves of a row set, all
// eight of a workgroup or, over few keys, 4, 2 or 1 of them (packed_plan.cpp), take the
// unit's 32-key sub-tiles in turn and merge their softmax states (max, sum in fp64, O)
// in a fixed order through LDS.  K and V come straight to registers through
// buffer resources of one sub-tile each, cut at the unit's last key: rows behind it
// read as 0, and no offset passes 32 bits.
//
// Values that are not finite, in causal units: as in packed_bf16.hip a wave whose
// result is not finite does its sub-tiles again, slowly, with such values of the
// diagonal kept out of the matrix products and added to the rows that see them.
#include <algorithm>

#include "attn_f32.hpp"
#include "common.hpp"
#include "packed.hpp"

namespace losa {

namespace {

constexpr int kWaves = kPackedWaves[0];  // of a workgroup: two per SIMD
constexpr int M = 16;

__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < INFINITY; }

// Sub-tile x (32 rows of D floats, `stride` bytes apart) of n rows at base.
template <int D>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t sub_rsrc(const char* base, uint32_t stride, int x,
                                                           int n) {
  int left = n - CK * x;
  left = left < 0 ? 0 : (left > CK ? CK : left);
  return make_rsrc(base + (int64_t)x * CK * stride,
                   left == 0 ? 0u : (uint32_t)(left - 1) * stride + 4 * D);
}
__device__ __forceinline__ f32x4_t load4(__amdgpu_buffer_rsrc_t rs, uint32_t off) {
  typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(f32x4_t, (u32x4_t)__builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0));
}

// Chunk c of a sub-tile's stream of K, then of V (f32_path.hip), as a byte offset.
template <int D>
__device__ __forceinline__ uint32_t k_at(int c, int lm, int g, uint32_t stride) {
  using T = F32Tile<D, M>;
  return (c % T::KT * M + lm) * stride + 4 * (4 * g + 4 * T::G * (c / T::KT));
}
template <int D>
__device__ __forceinline__ uint32_t v_at(int c, int lm, int g, uint32_t stride) {
  using T = F32Tile<D, M>;
  const int t = c / T::VP % T::SR, kt = c / T::VP / T::SR;
  return (kt * M + score_key<M>(t, g)) * stride + 4 * (lm * 4 + c % T::VP * 4 * M);
}

// RG groups of 16 rows a row set.
template <int D, int RG>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2)))
    packed_f32_kernel(const PackedArgs a) {
  constexpr int ROWS = M * RG;
  using T = F32Tile<D, M>;
  using A = F32Acc<M>;
  constexpr int NT = 64 * kWaves;
  constexpr int LD = D + 4;
  __shared__ float mpart[kWaves * ROWS];
  __shared__ double lpart[kWaves * ROWS];
  __shared__ __attribute__((aligned(16))) float opart[kWaves * ROWS * LD];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lm = lane % M, g = lane / M;
  const int unit = divide((int)blockIdx.x, a.by_H_kv);
  const int kvh = (int)blockIdx.x - unit * a.H_kv;
  const PackedItem it = a.items[unit];
  const int by = it.split & 3;  // 2^by waves share a row set
  const int KS = 1 << by;
  if (!inside(a, it, ROWS * kWaves >> by)) return;
  const int G = a.G;
  const int n = it.keys;
  const int set = w >> by, part = w & (KS - 1);
  const int first = set * ROWS;  // this wave's rows, from the unit's first on
  const int used = it.rows - first < ROWS ? it.rows - first : ROWS;
  // keys that every row of the wave sees, sub-tiles that some row does
  int whole = 0, S = 0;
  if (used > 0) {
    const int lo = it.seen + divide(it.head0 + first, a.by_G);
    const int hi = it.seen + divide(it.head0 + first + used - 1, a.by_G);
    whole = lo < n ? lo : n;
    S = ((hi < n ? hi : n) + CK - 1) / CK;
  }

  f32x4_t qr[RG * T::QI];
  int left[RG];  // keys this lane's row of each group sees
  bool valid[RG];
#pragma unroll
  for (int rg = 0; rg < RG; ++rg) {
    const int r = first + rg * M + lm;
    valid[rg] = r < it.rows;
    const int x = it.head0 + (valid[rg] ? r : 0);
    const int tok = divide(x, a.by_G);
    left[rg] = valid[rg] && it.seen + tok < n ? it.seen + tok : n;
    const float* qp = static_cast<const float*>(a.q) + (it.q_row + tok) * a.qt +
                      (int64_t)(kvh * G + x - tok * G) * a.qh + 4 * g;
#pragma unroll
    for (int i = 0; i < T::QI; ++i) {
      const f32x4_t q4 = *reinterpret_cast<const f32x4_t*>(qp + 4 * T::G * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) qr[rg * T::QI + i][e] = valid[rg] ? q4[e] * a.scale_log2 : 0.f;
    }
  }
  const char* kb = reinterpret_cast<const char*>(static_cast<const float*>(a.k) +
                                                 it.k_row * a.kt + kvh * a.kh);
  const char* vb = reinterpret_cast<const char*>(static_cast<const float*>(a.v) +
                                                 it.k_row * a.vt + kvh * a.vh);
  const uint32_t ks = (uint32_t)a.kt * 4, vs = (uint32_t)a.vt * 4;

  float m[RG];
  double l[RG];
  typename A::type o[RG][T::DB];
  auto clear = [&]() {
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
      m[rg] = kNegBig;
      l[rg] = 0.0;
#pragma unroll
      for (int b = 0; b < T::DB; ++b) o[rg][b] = typename A::type{};
    }
  };
  // scores of sub-tile x -> probabilities against the running max, sums
  auto softmax = [&](typename A::type* s, int x) {
    if (whole < CK * (x + 1)) {
#pragma unroll
      for (int rg = 0; rg < RG; ++rg)
#pragma unroll
        for (int kt = 0; kt < T::KT; ++kt)
#pragma unroll
          for (int t = 0; t < T::SR; ++t)
            if (CK * x + kt * M + score_key<M>(t, g) >= left[rg]) s[rg * T::KT + kt][t] = -INFINITY;
    }
    float mx[RG];
    bool raise = false;
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
      mx[rg] = tile_max<D, M>(s + rg * T::KT);
      raise = raise || mx[rg] > m[rg];
    }
    if (__ballot(raise) != 0) {
#pragma unroll
      for (int rg = 0; rg < RG; ++rg) {
        const float m_new = fmaxf(m[rg], mx[rg]);
        const float alpha = fast_exp2(m[rg] - m_new);  // 1 where the max stays
        m[rg] = m_new;
        l[rg] *= (double)alpha;
#pragma unroll
        for (int b = 0; b < T::DB; ++b) o[rg][b] *= alpha;
      }
    }
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) l[rg] += (double)tile_exp<D, M>(s + rg * T::KT, m[rg]);
  };

  clear();
  {
    constexpr int NC = T::KC + T::VN;  // chunks of a sub-tile
    f32x4_t ring[kLead];
    __amdgpu_buffer_rsrc_t krs = sub_rsrc<D>(kb, ks, part, n);
    if (part < S) {
#pragma unroll
      for (int c = 0; c < kLead; ++c) ring[c] = load4(krs, k_at<D>(c, lm, g, ks));
    }
    for (int x = part; x < S; x += KS) {
      const __amdgpu_buffer_rsrc_t vrs = sub_rsrc<D>(vb, vs, x, n);
      const __amdgpu_buffer_rsrc_t next = sub_rsrc<D>(kb, ks, x + KS, n);  // past the end: zeros
      auto issue = [&](int c) {
        const int y = c + kLead;
        if (y < T::KC)
          ring[c % kLead] = load4(krs, k_at<D>(y, lm, g, ks));
        else if (y < NC)
          ring[c % kLead] = load4(vrs, v_at<D>(y - T::KC, lm, g, vs));
        else
          ring[c % kLead] = load4(next, k_at<D>(y - NC, lm, g, ks));
      };
      typename A::type s[RG * T::KT];
      scores<D, M, RG>(ring, qr, g, CK, s, issue);
      softmax(s, x);
#pragma unroll
      for (int c = 0; c < T::VN; ++c) {
        const int p = c % T::VP, t = c / T::VP % T::SR, kt = c / T::VP / T::SR;
        const f32x4_t v = ring[(T::KC + c) % kLead];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int rg = 0; rg < RG; ++rg)
            o[rg][p * 4 + e] = A::mfma(v[e], s[rg * T::KT + kt][t], o[rg][p * 4 + e]);
        issue(T::KC + c);
        __builtin_amdgcn_sched_barrier(0);
      }
      krs = next;
    }
  }

  if (whole < n) {
    // some row does not see some key of the unit: has a value that is not finite spread?
    float bad = 0.f;  // becomes NaN
#pragma unroll
    for (int rg = 0; rg < RG; ++rg)
#pragma unroll
      for (int b = 0; b < T::DB; ++b)
#pragma unroll
        for (int t = 0; t < T::SR; ++t)
          bad = __builtin_fmaf(valid[rg] ? o[rg][b][t] : 0.f, 0.f, bad);
    if (__ballot(bad != 0.f) != 0) {
      clear();
      for (int x = part; x < S; x += KS) {
        const __amdgpu_buffer_rsrc_t krs = sub_rsrc<D>(kb, ks, x, n), vrs = sub_rsrc<D>(vb, vs, x, n);
        const bool all = whole >= CK * (x + 1);
        f32x4_t ring[kLead];
#pragma unroll
        for (int c = 0; c < kLead; ++c) ring[c] = load4(krs, k_at<D>(c, lm, g, ks));
        typename A::type s[RG * T::KT];
        scores<D, M, RG>(ring, qr, g, CK, s, [&](int c) {
          if (c + kLead < T::KC) ring[c % kLead] = load4(krs, k_at<D>(c + kLead, lm, g, ks));
        });
        softmax(s, x);
#pragma unroll
        for (int c = 0; c < T::VN; ++c) {
          const int p = c % T::VP, t = c / T::VP % T::SR, kt = c / T::VP / T::SR;
          const f32x4_t v = load4(vrs, v_at<D>(c, lm, g, vs));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float f = all || finite(v[e]) ? v[e] : 0.f;
#pragma unroll
            for (int rg = 0; rg < RG; ++rg)
              o[rg][p * 4 + e] = A::mfma(f, s[rg * T::KT + kt][t], o[rg][p * 4 + e]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (all) continue;
        // register t2 of d blocks 4 p .. 4 p + 3 holds d = 4 (16 p + score_key(t2, g)) .. + 3
#pragma unroll 1
        for (int kg = 0; kg < T::G; ++kg)
#pragma unroll
          for (int kt = 0; kt < T::KT; ++kt)
#pragma unroll
            for (int t = 0; t < T::SR; ++t) {
              const int key = kt * M + score_key<M>(t, kg);
#pragma unroll
              for (int rg = 0; rg < RG; ++rg) {
                const float p = __shfl(s[rg * T::KT + kt][t], kg * M + lm);
                const bool sees = CK * x + key < left[rg];
#pragma unroll
                for (int b = 0; b < T::DB; b += 4)
#pragma unroll
                  for (int t2 = 0; t2 < T::SR; ++t2) {
                    const f32x4_t v =
                        load4(vrs, key * vs + 16 * (b / 4 * M + score_key<M>(t2, g)));
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                      if (sees && !finite(v[e])) o[rg][b + e][t2] += p * v[e];
                  }
              }
              __builtin_amdgcn_sched_barrier(0);
            }
      }
    }
  }

  // merge the waves' states: the common max, then sums and outputs rescaled to it,
  // added in wave order
#pragma unroll
  for (int rg = 0; rg < RG; ++rg) {
    const int at = w * ROWS + rg * M + lm;
    const double lw = group_sum<M>(l[rg]);
    if (g == 0) {
      mpart[at] = m[rg];
      lpart[at] = lw;
    }
#pragma unroll
    for (int t = 0; t < T::SR; ++t)
#pragma unroll
      for (int b = 0; b < T::DB; ++b)
        opart[at * LD + 4 * (b / 4 * M + score_key<M>(t, g)) + b % 4] = o[rg][b][t];
  }
  __syncthreads();
  // where row r's state of the first of its waves lies
  auto state = [&](int r) { return (r / ROWS << by) * ROWS + r % ROWS; };
  const int all = ROWS * kWaves >> by, rows = it.rows < all ? it.rows : all;
  if (tid < rows) {
    // the weight of each wave takes its max's place, what the sum is divided by the first sum's
    const int at = state(tid);
    float mw[kWaves], mm = kNegBig;
#pragma unroll
    for (int y = 0; y < kWaves; ++y)
      if (y < KS) mm = fmaxf(mm, mw[y] = mpart[at + y * ROWS]);
    double lt = 0.0;
#pragma unroll
    for (int y = 0; y < kWaves; ++y)
      if (y < KS) {
        const float wgt = fast_exp2(mw[y] - mm);
        lt += lpart[at + y * ROWS] * (double)wgt;
        mpart[at + y * ROWS] = wgt;
      }
    // (in fp32 from here on: half a step, 2^-24, of a sum of positive terms, also of a part's)
    const float lf = (float)lt;
    lpart[at] = it.part >= 0 ? 1.f : (lf == 0.f ? 0.f : 1.0f / lf);
    if (it.part >= 0) {
      const int64_t to = (int64_t)(it.part + tid) * a.H_kv + kvh;
      *reinterpret_cast<f32x2_t*>(a.part_ml + 2 * to) = f32x2_t{mm, lf};
    } else if (a.lse != nullptr) {
      const int row = it.head0 + tid, tok = divide(row, a.by_G);
      a.lse[(int64_t)(kvh * G + (row - tok * G)) * a.lse_head + it.q_row + tok] =
          lf == 0.f ? -INFINITY : (mm + __log2f(lf)) * kLn2;
    }
  }
  __syncthreads();
#pragma unroll 2
  for (int idx = tid; idx < rows * D / 4; idx += NT) {
    const int r = idx / (D / 4), d4 = (idx % (D / 4)) * 4;
    const int at = state(r);
    const float inv = (float)lpart[at];
    f32x4_t acc = f32x4_t{};
#pragma unroll
    for (int y = 0; y < kWaves; ++y)
      if (y < KS) {
        const float wgt = mpart[at + y * ROWS];
        const f32x4_t p = *reinterpret_cast<const f32x4_t*>(opart + (at + y * ROWS) * LD + d4);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(p[e], wgt, acc[e]);
      }
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] *= inv;
    const int row = it.head0 + r, tok = divide(row, a.by_G);
    float* const op = it.part >= 0
                          ? a.part_o + ((int64_t)(it.part + r) * a.H_kv + kvh) * D
                          : static_cast<float*>(a.o) + (it.q_row + tok) * a.ot +
                                (int64_t)(kvh * G + (row - tok * G)) * a.oh;
    *reinterpret_cast<f32x4_t*>(op + d4) = acc;
  }
}

template <int D, int RG>
void launch_units(const PackedArgs& a, int units, hipStream_t stream) {
  if (units > 0)
    hipLaunchKernelGGL((packed_f32_kernel<D, RG>), dim3((uint32_t)units * a.H_kv),
                       dim3(64 * kWaves), 0, stream, a);
}

template <int D>
hipError_t launch(const PackedArgs& a, int n_few, hipStream_t stream) {
  if (a.tile_rows == kPackedNarrow) {  // tiles and few-row parts alike
    launch_units<D, 1>(a, a.n_tiles + n_few, stream);
    return hipGetLastError();
  }
  launch_units<D, 2>(a, a.n_tiles, stream);
  PackedArgs few = a;
  few.items += a.n_tiles;
  launch_units<D, 1>(few, n_few, stream);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_f32(int d, const PackedArgs& a, int n_few, hipStream_t stream) {
  if (d == 64) return launch<64>(a, n_few, stream);
  if (d == 128) return launch<128>(a, n_few, stream);
  return hipErrorInvalidValue;
}

}  // namespace losa
