// Decode attention with a sliding window and a few first tokens: the page waves of
// decode_mha.h and decode_gqa_common.h over the pages that hold visible tokens
// (WindowPages), whose other slots are masked, and the ring 64 slots at a time.
//
// The kernels take pages of any k_pad up to 8 KP8 (spare groups, load_page), for KP8 of
// window_tier(): a page pays for its tier at most.
#pragma once

#include "decode_mha.h"
#include "swan_layer_ops.h"

namespace swan {

// the kernels' KP8 serving a k_pad of 8 kp8
inline int window_tier(int kp8) { return kp8 <= 12 ? (kp8 + 1) & ~1 : 16; }

// The token of ring slot s (s < min(L, bb))
__device__ __forceinline__ int ring_token(int L, int bb, int s) {
  if (L <= bb) return s;
  const int at = L % bb;
  return L - at + s - (s >= at ? bb : 0);
}

// One wave: ring slots 64 piece .. + 63 of (sequence b, kv head h) for GH query heads from
// hq0 on.  Lane t scores slot t, then lane l sums dims 2 l and 2 l + 1.  q: [kD][GH] floats of
// scratch, p: [GH][64].
template <typename E, int GH>
__device__ void ring_wave(const WindowLaunch& a, int b, int h, int hq0, int piece, float* q,
                          float* p, int lane) {
  const int L = a.len[b], nb = min(L, a.bb);
  const int64_t ring = (((int64_t)b * a.Hkv + h) * a.bb + 64 * piece) * kD;
  const int count = min(64, nb - 64 * piece);
  const float* qh = a.qhat + ((int64_t)b * a.Hq + hq0) * kD;
#pragma unroll
  for (int x = 0; x < 2 * GH; ++x) q[(lane + 64 * (x & 1)) * GH + (x >> 1)] = qh[64 * x + lane];
  wave_lds_fence();
  const int token = ring_token(L, a.bb, 64 * piece + min(lane, count - 1));
  const bool seen = lane < count && (token >= a.lo[b] || token < a.sink[b]);
  constexpr int N = 16 / (int)sizeof(E);
  float s[GH];
#pragma unroll
  for (int g = 0; g < GH; ++g) s[g] = 0.f;
  const E* row = (const E*)a.k_ring + ring + (int64_t)min(lane, count - 1) * kD;
#pragma unroll 4
  for (int c = 0; c < kD / N; ++c) {
    struct alignas(16) {
      E v[N];
    } k = *(const decltype(k)*)(row + N * c);
#pragma unroll
    for (int e = 0; e < N; ++e)
#pragma unroll
      for (int g = 0; g < GH; ++g) s[g] = fmaf(q[(N * c + e) * GH + g], (float)k.v[e], s[g]);
  }
  float* part = a.part + (((int64_t)b * a.Hq + hq0) * a.slots + a.nsplit[b] + piece) * kPartFloats;
  const int64_t step = (int64_t)a.slots * kPartFloats;  // from a query head's part to the next's
#pragma unroll
  for (int g = 0; g < GH; ++g) {
    const float m = wave_max(seen ? s[g] : -INFINITY);
    const float w = seen ? exp2f(s[g] - m) : 0.f;
    const float l = wave_sum(w);
    p[g * 64 + lane] = w;
    if (lane == 0) {
      part[g * step] = m;
      part[g * step + 1] = l;
    }
  }
  wave_lds_fence();
  const uint64_t mask = __ballot(seen);
  float o[GH][2];
#pragma unroll
  for (int g = 0; g < GH; ++g) o[g][0] = o[g][1] = 0.f;
  const E* col = (const E*)a.v_ring + ring + 2 * lane;
#pragma unroll 8
  for (int t = 0; t < count; ++t) {
    struct alignas(2 * sizeof(E)) {
      E v[2];
    } v = *(const decltype(v)*)(col + t * kD);
    const bool on = (mask >> t) & 1;  // (a hidden token's value may be no number)
    const float v0 = on ? (float)v.v[0] : 0.f, v1 = on ? (float)v.v[1] : 0.f;
#pragma unroll
    for (int g = 0; g < GH; ++g) {
      const float w = p[g * 64 + t];
      o[g][0] = fmaf(w, v0, o[g][0]);
      o[g][1] = fmaf(w, v1, o[g][1]);
    }
  }
#pragma unroll
  for (int g = 0; g < GH; ++g) {
    part[g * step + 4 + 2 * lane] = o[g][0];
    part[g * step + 4 + 2 * lane + 1] = o[g][1];
  }
}

// whether the wave's lane has a visible token in page p
__device__ __forceinline__ bool seen_slot(const WindowLaunch& a, int b, const WindowPages& w, int p,
                                          int lane) {
  const int t = p * kPage + lane;
  return t < w.S && (t >= a.lo[b] || t < a.sink[b]);
}

}  // namespace swan
