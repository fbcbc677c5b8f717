// Rotary positions with several axes, alone or with the norms of queries and
// keys in the same pass; also lays values out beside them.
//
// Mathematics.  A row x is the d values of one token and head.  With a norm,
//   RMS    y = x / sqrt(mean(x^2) + eps) * w
//   layer  y = (x - mean(x)) / sqrt(var(x) + eps) * w + b
// over the row or over the token's H rows together (w, b: d or H*d values).  Pair i
// of the rotated dims belongs to one axis and turns by the angle of the token's
// position on it: (u, v) -> (u c - v s, u s + v c), with (c, s) from the caller's
// table (pairs: neighbours, or halves rot / 2 apart).  All in fp32 from the input to
// the single rounding of the output; the variance is taken about the mean.
//
// Bound: HBM.  Each element is read once and written once; a table by axis and
// position (a few KiB) stays in L1 where one by token would be 8 bytes per pair.
//
// Layout.  d / 8 lanes hold a row, 8 values a lane, so 64 / (d / 8) tokens share a
// wave and a row's sums are exchanges inside 8 or 16 lanes (DPP, no LDS).  A lane
// keeps its four pairs' (c, s) and loops over heads, kUnroll rows in flight.
// Input rows of a token lie side by side (token-major projections), output rows of
// a head (head-major attention layout): a wave's load takes whole rows, its store 1
// KiB (bf16) in one run.
#include "common.hpp"
#include "rope.hpp"

namespace losa {

namespace {

constexpr int kWaves = 4;   // waves of a workgroup
constexpr int kUnroll = 4;  // heads in flight per lane
// Heads up to which a wave holds a token's for their norm: no barrier, loads not
// repeated (121 us where the workgroup's waves share them: 138).  Up to kUnroll heads
// take a form for those (2 heads x 32,760 x 128, fp32: 35 us, in the one for 16 heads 48),
// and one head's is its row's.
constexpr int kAlone = 16;

// Output bytes of a call from which it is streamed: stores, and bf16 loads of 16 bytes
// that are not repeated, go past the caches (the L2s hold 32 MiB).  32,760 tokens x 12
// heads x 128, bf16, one tensor 48.5 -> 41.7 us, q, k, v with one norm over all heads
// 143 -> 121 (stores alone 134); 55 MB of fp32 29.7 -> 26.8 (its loads too: 29.4).
constexpr int64_t kStreamBytes = (int64_t)32 << 20;

// Whose norm: each row's; a token's, its heads over the workgroup's waves; a token's, all
// its heads in one wave, kAlone at most or kUnroll.
enum Norm { kEach, kShared, kOwn, kOwnFew };

// Eight values of a row as they lie in memory, in two groups of four.
template <typename T>
struct Raw;
template <>
struct Raw<__bf16> {
  bf16x4_t h[2];
};
template <>
struct Raw<float> {
  f32x4_t h[2];
};

// Groups at e0 and e1; neighbours (!HALVES, e1 = e0 + 4) move as 16 bytes, past the
// caches where the call is large and reads them once (ONCE).
template <bool HALVES, bool ONCE>
__device__ __forceinline__ Raw<__bf16> load_raw(const __bf16* p, int e0, int e1) {
  Raw<__bf16> r;
  if constexpr (HALVES) {
    r.h[0] = *reinterpret_cast<const bf16x4_t*>(p + e0);
    r.h[1] = *reinterpret_cast<const bf16x4_t*>(p + e1);
  } else {
    const bf16x8_t* const at = reinterpret_cast<const bf16x8_t*>(p + e0);
    const bf16x8_t v = ONCE ? __builtin_nontemporal_load(at) : *at;
    r.h[0] = __builtin_shufflevector(v, v, 0, 1, 2, 3);
    r.h[1] = __builtin_shufflevector(v, v, 4, 5, 6, 7);
  }
  return r;
}
template <bool HALVES, bool ONCE>
__device__ __forceinline__ Raw<float> load_raw(const float* p, int e0, int e1) {
  Raw<float> r;
  r.h[0] = *reinterpret_cast<const f32x4_t*>(p + e0);
  r.h[1] = *reinterpret_cast<const f32x4_t*>(p + e1);
  return r;
}
// Stores go past the caches (STREAM) where the call's outputs are too large to stay in
// them (kStreamBytes).
template <bool STREAM, typename V>
__device__ __forceinline__ void put(void* p, V v) {
  if constexpr (STREAM)
    __builtin_nontemporal_store(v, static_cast<V*>(p));
  else
    *static_cast<V*>(p) = v;
}
template <bool HALVES, bool STREAM>
__device__ __forceinline__ void store_raw(__bf16* p, int e0, int e1, const Raw<__bf16>& r) {
  if constexpr (HALVES) {
    put<STREAM, bf16x4_t>(p + e0, r.h[0]);
    put<STREAM, bf16x4_t>(p + e1, r.h[1]);
  } else {
    put<STREAM, bf16x8_t>(p + e0,
                          __builtin_shufflevector(r.h[0], r.h[1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
}
template <bool HALVES, bool STREAM>
__device__ __forceinline__ void store_raw(float* p, int e0, int e1, const Raw<float>& r) {
  put<STREAM, f32x4_t>(p + e0, r.h[0]);
  put<STREAM, f32x4_t>(p + e1, r.h[1]);
}

template <typename T>
__device__ __forceinline__ void widen(const Raw<T>& r, float* x) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (float)r.h[e >> 2][e & 3];
}
template <typename T>
__device__ __forceinline__ Raw<T> narrow(const float* x) {
  Raw<T> r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r.h[e >> 2][e & 3] = (T)x[e];
  return r;
}

template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
// Sum over the L = 8 or 16 lanes of a row, in every one of them.
template <int L>
__device__ __forceinline__ float row_sum(float x) {
  x = add_dpp<0xB1>(x);   // lane ^ 1
  x = add_dpp<0x4E>(x);   // lane ^ 2
  x = add_dpp<0x141>(x);  // 7 - lane: the other four
  if constexpr (L == 16) x = add_dpp<0x140>(x);  // 15 - lane: the other eight
  return x;
}

// Workgroup -> tensor, batch, token tile, heads.  kEach: a wave owns a tile of tokens
// and `hc` heads, the workgroup's waves neighbouring tiles.  kOwn, kOwnFew: the same with
// all of the 16 heads or fewer, which the wave holds in registers between their sum and
// their output.  kShared: a workgroup owns a tile, its waves take the heads in turn and add
// their sums in LDS; with more than 16 heads a pass reads them again.
template <typename T, int D, bool HALVES, bool STREAM, Norm WHOSE>
__global__ void __launch_bounds__(64 * kWaves) rows_kernel(const RowsArgs a) {
  constexpr int L = D / 8;    // lanes per row
  constexpr int TW = 64 / L;  // tokens per wave
  constexpr bool ALL = WHOSE != kEach, SHARED = WHOSE == kShared;
  constexpr int U = WHOSE == kOwn ? kAlone : kUnroll;  // heads in flight
  __shared__ float part[SHARED ? 2 : 1][kWaves][TW];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int l = lane % L, tk = lane / L;
  int ti = 0;
  int64_t j = blockIdx.x;
  while (ti < 2 && j >= a.blocks[ti]) j -= a.blocks[ti++];
  const RowsTensor& t = a.t[ti];
  const int64_t tw = j / t.chunks;  // tile (kShared) or group of kWaves tiles
  const int chunk = (int)(j - tw * t.chunks);
  const int b = (int)(tw / a.tiles);
  const int tile = (int)(tw - (int64_t)b * a.tiles);
  const int n = (SHARED ? tile : tile * kWaves + w) * TW + tk;
  const bool real = n < a.N;       // else a padding row (0), or none
  const bool there = n < a.n_pad;
  const int nr = real ? n : 0;     // a token whose row and positions may be read

  // this lane's values of a row
  int e0 = 8 * l, e1 = e0 + 4;
  const bool turned = t.rotate && l < a.rot8;
  if (HALVES && l < a.rot8) {
    e0 = 4 * l;
    e1 = 4 * a.rot8 + 4 * l;
  }
  // its pairs' (cos, sin): pair 4 l + i of the rotated dims
  float c[4], s[4];
  if (t.rotate) {
    int at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) at[i] = -1;
    const int32_t* pos = a.pos + b * a.pos_batch + nr;
#pragma unroll
    for (int x = 0; x < kMaxAxes; ++x) {
      if (x < a.axes) {
        const int p = pos[(int64_t)x * a.N];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int q = 4 * l + i - a.pair0[x];
          if (q >= 0 && q < a.dim[x] / 2)
            at[i] = p < 0 ? -1 : (p >= a.len[x] ? -2 : a.off[x] + p * a.dim[x] + 2 * q);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2_t v = *reinterpret_cast<const f32x2_t*>(a.table + (at[i] < 0 ? 0 : at[i]));
      c[i] = at[i] == -1 ? 1.f : (at[i] == -2 ? __builtin_nanf("") : v[0]);
      s[i] = at[i] == -1 ? 0.f : (at[i] == -2 ? __builtin_nanf("") : v[1]);
    }
  }

  const T* xp = static_cast<const T*>(t.x) + b * t.xb + nr * t.xt;
  T* yp = static_cast<T*>(t.y) + b * t.yb + (int64_t)n * t.yt;
  const int h0 = SHARED ? w * U : chunk * t.hc;
  const int h1 = SHARED ? t.H : (h0 + t.hc < t.H ? h0 + t.hc : t.H);
  const int step = SHARED ? kWaves * U : U;  // heads a pass of the loops below

  Raw<T> raw[U];
  auto load = [&](int h) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      raw[u] = Raw<T>{};
      if (h + u < h1 && real) raw[u] = load_raw<HALVES, STREAM && !SHARED>(xp + (h + u) * t.xh, e0, e1);
    }
  };
  float mean = 0.f, inv = 1.f;
  const bool once = h0 + step >= h1;  // every head of this wave is held in raw
  // sum of a token's lanes' (and, shared, waves') values, in every lane
  auto token_sum = [&](float x, int which) {
    x = row_sum<L>(x);
    if constexpr (SHARED) {
      if (l == 0) part[which][w][tk] = x;
      __syncthreads();
      x = 0.f;
#pragma unroll
      for (int y = 0; y < kWaves; ++y) x += part[which][y][tk];
    }
    return x;
  };
  if constexpr (ALL) {
    if (t.norm != kNormNone) {
      if (once) load(h0);
      const float count = (float)t.H * D;
      if (t.norm == kNormLayer) {
        float sum = 0.f;
        for (int h = h0; h < h1; h += step) {
          if (!once) load(h);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            float x[8];
            widen<T>(raw[u], x);
            sum += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
          }
        }
        mean = token_sum(sum, 0) / count;
      }
      float sq = 0.f;
      for (int h = h0; h < h1; h += step) {
        if (!once) load(h);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float x[8];
          widen<T>(raw[u], x);
          if (h + u < h1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float z = x[e] - mean;
              sq = __builtin_fmaf(z, z, sq);
            }
          }
        }
      }
      inv = 1.0f / sqrtf(token_sum(sq, 1) / count + a.eps);
    }
  }

  float wt[8], bs[8];  // weights and biases of a norm over each head
  auto load8 = [&](const float* p, float* v) {
    const f32x4_t v0 = *reinterpret_cast<const f32x4_t*>(p + e0);
    const f32x4_t v1 = *reinterpret_cast<const f32x4_t*>(p + e1);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = v0[e];
      v[4 + e] = v1[e];
    }
  };
  if (!ALL && t.norm != kNormNone) {
    if (t.w != nullptr) load8(t.w, wt);
    if (t.b != nullptr) load8(t.b, bs);
  }

  for (int h = h0; h < h1; h += step) {
    if (!(ALL && once && t.norm != kNormNone)) load(h);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (h + u >= h1) break;
      if (t.norm != kNormNone || t.rotate) {
        float x[8];
        widen<T>(raw[u], x);
        if (t.norm != kNormNone) {
          if constexpr (ALL) {
            if (t.w != nullptr) load8(t.w + (h + u) * D, wt);
            if (t.b != nullptr) load8(t.b + (h + u) * D, bs);
          } else {
            mean = 0.f;
            if (t.norm == kNormLayer)
              mean = row_sum<L>(((x[0] + x[1]) + (x[2] + x[3])) +
                                ((x[4] + x[5]) + (x[6] + x[7]))) * (1.0f / D);
            float sq = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float z = x[e] - mean;
              sq = __builtin_fmaf(z, z, sq);
            }
            inv = 1.0f / sqrtf(row_sum<L>(sq) * (1.0f / D) + a.eps);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] = (x[e] - mean) * inv;
            if (t.w != nullptr) x[e] *= wt[e];
            if (t.b != nullptr) x[e] += bs[e];
          }
        }
        if (turned) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = x[HALVES ? i : 2 * i], q = x[HALVES ? 4 + i : 2 * i + 1];
            // an angle of 0 leaves the pair as it is, its infinities too
            const bool still = s[i] == 0.f;
            x[HALVES ? i : 2 * i] = still ? p * c[i] : p * c[i] - q * s[i];
            x[HALVES ? 4 + i : 2 * i + 1] = still ? q * c[i] : p * s[i] + q * c[i];
          }
        }
        raw[u] = narrow<T>(x);
        if (!real) raw[u] = Raw<T>{};
      }
      if (there) store_raw<HALVES, STREAM>(yp + (h + u) * t.yh, e0, e1, raw[u]);
    }
  }
}

// Heads that a wave takes one after another: all of a token's, so that its (c, s)
// are fetched once, unless the call is too small to give every SIMD a few waves.
int heads_per_wave(int H, int64_t groups_heads) {
  const int64_t want = groups_heads / 1024;
  const int hc = (int)(want < kUnroll ? kUnroll : (want > H ? H : want));
  return (hc + kUnroll - 1) / kUnroll * kUnroll;
}

template <typename T, int D, bool HALVES, bool STREAM>
void launch_rows_of(const RowsArgs& a, Norm whose, uint32_t groups, hipStream_t stream) {
  const dim3 grid(groups), block(64 * kWaves);
  if (whose == kEach)
    hipLaunchKernelGGL((rows_kernel<T, D, HALVES, STREAM, kEach>), grid, block, 0, stream, a);
  else if (whose == kOwn)
    hipLaunchKernelGGL((rows_kernel<T, D, HALVES, STREAM, kOwn>), grid, block, 0, stream, a);
  else if (whose == kOwnFew)
    hipLaunchKernelGGL((rows_kernel<T, D, HALVES, STREAM, kOwnFew>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((rows_kernel<T, D, HALVES, STREAM, kShared>), grid, block, 0, stream, a);
}

template <typename T, int D, bool HALVES>
hipError_t launch(RowsArgs& a, int tensors, bool all, hipStream_t stream) {
  constexpr int TW = 64 / (D / 8);
  int64_t heads = 0, total = 0;
  int normed = 0;  // most heads of a tensor with a norm
  for (int i = 0; i < tensors; ++i) {
    heads += a.t[i].H;
    if (a.t[i].norm != kNormNone && a.t[i].H > normed) normed = a.t[i].H;
  }
  const Norm whose = !all || normed <= 1 ? kEach  // (over one head it is the head's)
                     : normed <= kUnroll ? kOwnFew
                     : normed <= kAlone  ? kOwn
                                         : kShared;
  const int64_t tiles = (a.n_pad + TW - 1) / TW;
  a.tiles = (int)(whose == kShared ? tiles : (tiles + kWaves - 1) / kWaves);
  for (int i = 0; i < 3; ++i) {
    a.blocks[i] = 0;
    if (i >= tensors) continue;
    RowsTensor& t = a.t[i];
    t.hc = whose == kEach ? heads_per_wave(t.H, heads * a.B * a.tiles) : t.H;
    t.chunks = (t.H + t.hc - 1) / t.hc;
    a.blocks[i] = (int64_t)a.B * a.tiles * t.chunks;
    total += a.blocks[i];
  }
  // (a launch counts its threads in 32 bits)
  if (total * 64 * kWaves >= ((int64_t)1 << 32)) return hipErrorInvalidConfiguration;
  if (heads * a.B * a.n_pad * D * (int64_t)sizeof(T) >= kStreamBytes)
    launch_rows_of<T, D, HALVES, true>(a, whose, (uint32_t)total, stream);
  else
    launch_rows_of<T, D, HALVES, false>(a, whose, (uint32_t)total, stream);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rows(int d, bool bf16, bool halves, RowsArgs& a, int tensors, bool all,
                       hipStream_t stream) {
#define LOSA_ROWS(TT, DD)                                                        \
  if (bf16 == (sizeof(TT) == 2) && d == DD)                                      \
    return halves ? launch<TT, DD, true>(a, tensors, all, stream)                \
                  : launch<TT, DD, false>(a, tensors, all, stream);
  LOSA_ROWS(__bf16, 64)
  LOSA_ROWS(__bf16, 128)
  LOSA_ROWS(float, 64)
  LOSA_ROWS(float, 128)
#undef LOSA_ROWS
  return hipErrorInvalidValue;
}

}  // namespace losa
