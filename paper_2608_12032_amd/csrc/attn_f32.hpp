// One wave's share of an fp32 attention stream on the fp32 matrix instructions:
// shapes, scores of a 32-key sub-tile, its softmax.  Used by the fp32 path and by
// the packed attention; the tiles are explained in f32_path.hip.
#pragma once

#include "common.hpp"

namespace losa {

namespace {

constexpr int CK = 32;    // keys per sub-tile
constexpr int kLead = 8;  // loads in flight ahead of their use, per wave

// Shapes of a wave's groups of M query rows.  A sub-tile's operands arrive as a
// stream of KC chunks of K, then (M = 16) VN of V, 16 bytes a lane.
template <int D, int M>
struct F32Tile {
  static constexpr int G = 64 / M;             // lane groups
  static constexpr int SR = M * M / 64;        // score registers per M-key tile
  static constexpr int KT = CK / M;            // M-key tiles per sub-tile
  static constexpr int QI = D / (4 * G);       // 16-byte chunks of a row per lane
  static constexpr int DB = D / M;             // d blocks of O^T
  static constexpr int VP = DB / 4;            // V loads per score register
  static constexpr int KC = KT * QI;
  static constexpr int VN = KT * SR * VP;
  static_assert(KC % kLead == 0 && VN % kLead == 0, "the stream fills the ring evenly");
};

template <int M>
struct F32Acc;
template <>
struct F32Acc<32> {
  typedef f32x16_t type;
  static __device__ __forceinline__ type mfma(float a, float b, type c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
  }
};
template <>
struct F32Acc<16> {
  typedef f32x4_t type;
  static __device__ __forceinline__ type mfma(float a, float b, type c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
  }
};

// Key of score register t in lane group g, inside an M-key tile.
template <int M>
__device__ __forceinline__ int score_key(int t, int g) {
  return (t >> 2) * (256 / M) + 4 * g + (t & 3);
}

// Scores of a sub-tile in log2 units: chunk c of K, in ring[c % kLead], against
// the query operands of RG row groups (group r's at qr[r * QI], its scores at
// s[r * KT]; two accumulation chains each, so that no product waits for the one
// before it).  issue(c) refills the slot just used.  Keys at or beyond kvalid get
// -inf.
template <int D, int M, int RG, typename Issue>
__device__ __forceinline__ void scores(f32x4_t* ring, const f32x4_t* qr, int g, int kvalid,
                                       typename F32Acc<M>::type* s, Issue&& issue) {
  using T = F32Tile<D, M>;
  using A = F32Acc<M>;
  typename A::type odd[RG * T::KT];
#pragma unroll
  for (int x = 0; x < RG * T::KT; ++x) {
    s[x] = typename A::type{};
    odd[x] = typename A::type{};
  }
#pragma unroll
  for (int c = 0; c < T::KC; ++c) {
    const int kt = c % T::KT, i = c / T::KT;
    const f32x4_t a = ring[c % kLead];
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int r = 0; r < RG; ++r) {
        typename A::type& x = (e & 1) == 0 ? s[r * T::KT + kt] : odd[r * T::KT + kt];
        x = A::mfma(a[e], qr[r * T::QI + i][e], x);
      }
    issue(c);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int x = 0; x < RG * T::KT; ++x) s[x] += odd[x];
  if (kvalid < CK) {
#pragma unroll
    for (int x = 0; x < RG * T::KT; ++x)
#pragma unroll
      for (int t = 0; t < T::SR; ++t)
        if (x % T::KT * M + score_key<M>(t, g) >= kvalid) s[x][t] = -INFINITY;
  }
}

template <int M>
__device__ __forceinline__ float group_max(float x) {
  x = max_with_partner(x);
  if constexpr (M == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return x;
}
template <int M>
__device__ __forceinline__ double group_sum(double x) {
  x += __shfl_xor(x, 32);
  if constexpr (M == 16) x += __shfl_xor(x, 16);
  return x;
}

// Maximum of the sub-tile's scores of this lane's query.
template <int D, int M>
__device__ __forceinline__ float tile_max(const typename F32Acc<M>::type* s) {
  using T = F32Tile<D, M>;
  float mx = s[0][0];
#pragma unroll
  for (int kt = 0; kt < T::KT; ++kt)
#pragma unroll
    for (int t = 0; t < T::SR; ++t) mx = fmaxf(mx, s[kt][t]);
  return group_max<M>(mx);
}

// s <- 2^(s - m); returns this lane's sum.
template <int D, int M>
__device__ __forceinline__ float tile_exp(typename F32Acc<M>::type* s, float m) {
  using T = F32Tile<D, M>;
  float part = 0.f;
#pragma unroll
  for (int kt = 0; kt < T::KT; ++kt)
#pragma unroll
    for (int t = 0; t < T::SR; ++t) {
      s[kt][t] = fast_exp2(s[kt][t] - m);
      part += s[kt][t];
    }
  return part;
}

}  // namespace

}  // namespace losa
