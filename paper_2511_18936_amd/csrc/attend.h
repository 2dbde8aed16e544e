// Attention of many query rows over tiles of 64 keys, one pass with a running softmax.
//
// Per tile and wave (32 query rows, one per lane and half wave):
//   S^T[64 keys][32 rows] = K . Q^T      MFMA, K from LDS, Q in registers
//   p = exp2(S - ref), row by row        a lane holds its row's scores of 32 of the keys
//   O^T[128 dims][32 rows] += V^T . P^T  MFMA, V^T from LDS, p straight from the registers
//
// The products are taken transposed because the result layout of the first (a lane has one
// column, its query row, and rows 8 (i / 4) + 4 (lane / 32) + i % 4) is then the operand
// layout of the second up to the order of the keys, which both operands of a product may
// permute alike: no exchange between lanes and no LDS for p.  A row's maximum takes one
// exchange with lane +- 32, its sum one at the end.
//
// The reference `ref` lags behind the maximum: it moves when a score exceeds it by more
// than kLag, and is set kHead below the maximum, so that the binary16 p of the 16-bit path
// (2^kLag at most) uses the upper part of its range: p below 2^-14 of the largest would be
// subnormal without it.  p is rounded to binary16 there (2^-11 relative, and the sum is
// taken of the rounded values, so the weights still sum to one); everything else is float32.
#pragma once

#include "swan_device.h"
#include "swan_layer_ops.h"

namespace swan {

typedef _Float16 h2v __attribute__((ext_vector_type(2)));
typedef _Float16 h4v __attribute__((ext_vector_type(4)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));

constexpr float kHead = 7.f;
constexpr float kLag = 15.f;  // 2^15 < 65504
constexpr float kLog2e = 1.4426950408889634f;

// v of this lane and of lane +- 32: {the lower half's, the upper half's}
__device__ __forceinline__ f4v both_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return f4v{__uint_as_float(r[0]), __uint_as_float(r[1]), 0.f, 0.f};
}
__device__ __forceinline__ float max_halves(float v) {
  const f4v b = both_halves(v);
  return fmaxf(b.x, b.y);
}
__device__ __forceinline__ float sum_halves(float v) {
  const f4v b = both_halves(v);
  return b.x + b.y;
}

// The tile in LDS and its products, by element type.  K [key][dim] and V^T [dim][key], with
// row strides that put 16-byte reads of consecutive rows on distinct banks; key t of a
// binary16 V^T is at column col(t), which swaps the middle two quads of every 16 so that a
// lane's 8 keys (8 (i / 4) + 4 (lane / 32) + i % 4, i = 0..7) are contiguous.
template <typename T>
struct Tile;

template <>
struct Tile<_Float16> {
  static constexpr int KS = 136, VS = 72;
  struct alignas(16) Buf {
    _Float16 k[kTileKeys * KS];
    _Float16 v[kD * VS];
  };
  __device__ static __forceinline__ int col(int t) {
    return (t & ~12) | ((t & 4) << 1) | ((t & 8) >> 1);
  }
  // Q of the wave's rows: dims 16 s + 8 (lane / 32) .. + 7 of row lane % 32; kLow: a second
  // part for what the first rounds off
  template <bool kLow>
  struct Q {
    h8v hi[8], lo[kLow ? 8 : 1];
  };
  template <bool kLow>
  __device__ static __forceinline__ void scores(const Buf& b, const Q<kLow>& q, int lane,
                                                f16v (&S)[2]) {
    const _Float16* k0 = b.k + (lane & 31) * KS + 8 * (lane >> 5);
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const h8v k = *(const h8v*)(k0 + 32 * t * KS + 16 * s);
        S[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q.hi[s], S[t], 0, 0, 0);
        if constexpr (kLow) S[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q.lo[s], S[t], 0, 0, 0);
      }
  }
  // p = exp2(S c - ref) into S's place (rounded), O += V^T . p; returns the lane's sum of p
  __device__ static __forceinline__ float values(const Buf& b, f16v (&S)[2], float c, float ref,
                                                 int lane, f16v (&O)[4]) {
    const _Float16* v0 = b.v + (lane & 31) * VS + 8 * (lane >> 5);
    const h2v one = {(_Float16)1.f, (_Float16)1.f};
    float l = 0.f;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      h8v p;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const int i = 8 * (s & 1) + e;
        const h2v two = {
            (_Float16)__builtin_amdgcn_exp2f(fmaf(S[s >> 1][i], c, -ref)),
            (_Float16)__builtin_amdgcn_exp2f(fmaf(S[s >> 1][i + 1], c, -ref))};
        l = __builtin_amdgcn_fdot2(two, one, l, false);
        p[e] = two.x;
        p[e + 1] = two.y;
      }
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const h8v v = *(const h8v*)(v0 + 32 * d * VS + 16 * s);
        O[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p, O[d], 0, 0, 0);
      }
    }
    return l;
  }
};

template <>
struct Tile<float> {
  static constexpr int KS = 132, VS = 68;
  struct alignas(16) Buf {
    float k[kTileKeys * KS];
    float v[kD * VS];
  };
  __device__ static __forceinline__ int col(int t) { return t; }
  template <bool kLow>
  struct Q {
    f4v hi[16];  // dims 8 s + 4 (lane / 32) .. + 3
  };
  template <bool kLow>
  __device__ static __forceinline__ void scores(const Buf& b, const Q<kLow>& q, int lane,
                                                f16v (&S)[2]) {
    const float* k0 = b.k + (lane & 31) * KS + 4 * (lane >> 5);
#pragma unroll
    for (int s = 0; s < 16; ++s)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const f4v k = *(const f4v*)(k0 + 32 * t * KS + 8 * s);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          S[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], q.hi[s][e], S[t], 0, 0, 0);
      }
  }
  __device__ static __forceinline__ float values(const Buf& b, f16v (&S)[2], float c, float ref,
                                                 int lane, f16v (&O)[4]) {
    const float* v0 = b.v + (lane & 31) * VS + 4 * (lane >> 5);
    float l = 0.f;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      f4v p;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(S[s >> 2][4 * (s & 3) + e], c, -ref));
        l += p[e];
      }
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const f4v v = *(const f4v*)(v0 + 32 * d * VS + 8 * s);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          O[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e], p[e], O[d], 0, 0, 0);
      }
    }
    return l;
  }
};

// key of element i of S[t], from the tile's first
__device__ __forceinline__ int key_of(int t, int i, int lane) {
  return 32 * t + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
}

// A wave's running softmax: a lane's row, dims 32 d + 8 (i / 4) + 4 (lane / 32) + i % 4
struct RowState {
  float ref;  // log2 units; -inf: no key yet
  float l;    // this lane's half of the sum
  f16v O[4];
  __device__ __forceinline__ void clear() {
    ref = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) O[d][i] = 0.f;
  }
  // moves the reference of the rows in which a score of this tile exceeds it by more than
  // kLag (of no other row: a row's bits do not depend on its neighbours'); mx: the
  // maximum of the row's scores x c
  __device__ __forceinline__ void raise(float mx) {
    const bool up = mx - ref > kLag;
    if (__any(up)) {
      const float to = up ? mx - kHead : ref;
      const float f = up ? __builtin_amdgcn_exp2f(ref - to) : 1.f;
      ref = to;
      l *= f;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[d][i] *= f;
    }
  }
  __device__ __forceinline__ float safe_ref() const { return ref == -INFINITY ? 0.f : ref; }
};

__device__ __forceinline__ float tile_max(const f16v (&S)[2]) {
  float m = S[0][0];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(m, S[t][i]);
  return max_halves(m);
}

// the group of a unit (uniform)
__device__ __forceinline__ int group_of(const AttendLaunch& a, int unit) {
  int lo = 0, hi = a.groups;  // unit0[lo] <= unit < unit0[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (unit >= a.unit0[mid]) lo = mid;
    else hi = mid;
  }
  return lo;
}

// sequence b and row i of it that token `tok` of group j is
__device__ __forceinline__ void token_at(const AttendLaunch& a, int j, int tok, int& b, int& i) {
  int lo = a.first[j], hi = a.first[j + 1];
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (tok >= a.tok0[mid]) lo = mid;
    else hi = mid;
  }
  b = a.seq[lo];
  i = tok - a.tok0[lo];
}

// the row's partial: reference, sum, accumulator
__device__ __forceinline__ void write_partial(const AttendLaunch& a, const RowState& st,
                                              int64_t row, int split, bool live, int lane) {
  const float l = sum_halves(st.l);
  if (!live) return;
  float* part = a.part + (row * a.slots + a.slot0 + split) * kPartFloats;
  if (lane < 32) {
    part[0] = st.ref;
    part[1] = l;
  }
  part += 4 + 4 * (lane >> 5);
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(f4v*)(part + 32 * d + 8 * i) = f4v{st.O[d][4 * i], st.O[d][4 * i + 1], st.O[d][4 * i + 2],
                                           st.O[d][4 * i + 3]};
}

}  // namespace swan
