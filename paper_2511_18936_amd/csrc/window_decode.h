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

// One wave: ring slots 64 piece .. + 63 of (sequence b, kv head h) for query head hq.  Lane t
// scores slot t; then a row of the values goes to 16 lanes (float32: 32), 16 bytes each, 4 (2)
// rows at a time, and the lanes' sums of the same dims meet at the end.  What bounds it is the
// latency of its loads, so 16 of them are in flight at a time, the first values' before the
// scores.  One query head a wave, the rows of a group's others coming from L2: two need more
// registers than the page waves, whose kernel it is.  q: its rotated query in LDS; p: 64 floats
// of scratch.
template <typename E>
__device__ void ring_wave(const WindowLaunch& a, int b, int h, int hq, int piece, const float* q,
                          float* p, int lane) {
  constexpr int N = 16 / (int)sizeof(E);  // elements of 16 bytes
  constexpr int kLanes = kD / N, kAtOnce = 64 / kLanes, kLoads = 16;
  struct alignas(16) Vec {
    E v[N];
  };
  const int L = a.len[b], nb = min(L, a.bb);
  const int64_t ring = (((int64_t)b * a.Hkv + h) * a.bb + 64 * piece) * kD;
  const int count = min(64, nb - 64 * piece), mine = min(lane, count - 1);
  Vec k[kLoads], v[kLoads];
  const E* row = (const E*)a.k_ring + ring + (int64_t)mine * kD;
  const E* col = (const E*)a.v_ring + ring + N * (lane % kLanes);
  const int first = lane / kLanes;  // row first + kAtOnce i is this lane's i-th
  auto load_k = [&](int x0) {
#pragma unroll
    for (int x = 0; x < kLoads; ++x) k[x] = *(const Vec*)(row + N * (x0 + x));
  };
  auto load_v = [&](int x0) {
#pragma unroll
    for (int x = 0; x < kLoads; ++x)
      v[x] = *(const Vec*)(col + (int64_t)min(first + kAtOnce * (x0 + x), count - 1) * kD);
  };
  load_k(0);
  load_v(0);
  const int token = ring_token(L, a.bb, 64 * piece + mine);
  const bool seen = lane < count && (token >= a.lo[b] || token < a.sink[b]);
  float s0 = 0.f, s1 = 0.f;
#pragma unroll
  for (int x0 = 0; x0 < kLanes; x0 += kLoads) {
    if (x0 > 0) load_k(x0);
#pragma unroll
    for (int x = 0; x < kLoads; ++x)
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        s0 = fmaf(q[N * (x0 + x) + e], (float)k[x].v[e], s0);
        s1 = fmaf(q[N * (x0 + x) + e + 1], (float)k[x].v[e + 1], s1);
      }
  }
  float* part = a.part + (((int64_t)b * a.Hq + hq) * a.slots + a.nsplit[b] + piece) * kPartFloats;
  const float s = seen ? s0 + s1 : -INFINITY, m = wave_max(s);
  const float w = seen ? exp2f(s - m) : 0.f, l = wave_sum(w);
  p[lane] = w;
  if (lane == 0) {
    part[0] = m;
    part[1] = l;
  }
  wave_lds_fence();
  const uint64_t mask = __ballot(seen) >> first;
  float o[N];
#pragma unroll
  for (int e = 0; e < N; ++e) o[e] = 0.f;
#pragma unroll
  for (int x0 = 0; x0 < 64 / kAtOnce; x0 += kLoads) {
    if (x0 > 0) load_v(x0);
#pragma unroll
    for (int x = 0; x < kLoads; ++x) {
      const int t = kAtOnce * (x0 + x);
      const bool on = (mask >> t) & 1;  // (a hidden token's value may be no number)
      const float pt = p[t + first];
#pragma unroll
      for (int e = 0; e < N; ++e) o[e] = fmaf(pt, on ? (float)v[x].v[e] : 0.f, o[e]);
    }
  }
#pragma unroll
  for (int d = kLanes; d < 64; d *= 2)
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] += __shfl_xor(o[e], d, 64);
  if (lane < kLanes) {
#pragma unroll
    for (int e = 0; e < N; e += 4)
      *(float4*)(part + 4 + N * lane + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
  }
}

// whether the wave's lane has a visible token in page p
__device__ __forceinline__ bool seen_slot(const WindowLaunch& a, int b, const WindowPages& w, int p,
                                          int lane) {
  const int t = p * kPage + lane;
  return t < w.S && (t >= a.lo[b] || t < a.sink[b]);
}

}  // namespace swan
