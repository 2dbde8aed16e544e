// How the rows of RoPE are turned: kForm
//   0  the whole head, dims k and k + 64 a pair, base^(-2k/128) radians a position
//   1  the first 2 half dims, dims k and k + half a pair, given frequencies and a magnitude
//   2  the same with dims 2k and 2k + 1 as pairs
// In forms 1 and 2 the dims from 2 half on are pairs too, the k-th for k >= half, which are
// left as they are.  half is a multiple of 4, so that a lane's pairs (4 at most) are of one
// kind and its accesses aligned.
#pragma once

#include <type_traits>

#include "swan_layer_ops.h"

namespace swan {

struct WholeHead {};
template <int kForm>
using FormArg = typename std::conditional<kForm == 0, WholeHead, RotaryForm>::type;

template <int kForm>
__device__ __forceinline__ double pair_freq(const FormArg<kForm>& f, double base, int k) {
  if constexpr (kForm == 0) return pow(base, -(2.0 * k) / kD);
  else return f.freq[k];
}

template <int kForm>
__device__ __forceinline__ void pair_turn(const FormArg<kForm>& f, double angle, double& s,
                                          double& c) {
  sincos(angle, &s, &c);
  if constexpr (kForm != 0) {
    s *= f.magnitude;
    c *= f.magnitude;
  }
}

// whether pair k is turned
template <int kForm>
__device__ __forceinline__ bool turned(const FormArg<kForm>& f, int k) {
  if constexpr (kForm == 0) return true;
  else return k < f.half;
}

// Where the N elements that a lane loads first, and second, begin for its pairs k .. k + N - 1
template <int kForm, int N>
__device__ __forceinline__ int place(const FormArg<kForm>& f, int k, bool second) {
  if constexpr (kForm == 0) return k + (second ? kD / 2 : 0);
  else if constexpr (kForm == 1) {
    const bool t = k < f.half;
    return (t ? k : f.half + k) + (second ? (t ? f.half : kD / 2 - f.half) : 0);
  } else {
    return 2 * k + (second ? N : 0);
  }
}

// What was loaded as the pairs' first and second elements, and back
template <int kForm, int N, typename T>
__device__ __forceinline__ void to_pairs(T (&a)[N], T (&b)[N]) {
  if constexpr (kForm == 2) {
    T all[2 * N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      all[e] = a[e];
      all[N + e] = b[e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      a[e] = all[2 * e];
      b[e] = all[2 * e + 1];
    }
  }
}
template <int kForm, int N, typename T>
__device__ __forceinline__ void from_pairs(T (&a)[N], T (&b)[N]) {
  if constexpr (kForm == 2) {
    T all[2 * N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      all[2 * e] = a[e];
      all[2 * e + 1] = b[e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      a[e] = all[e];
      b[e] = all[N + e];
    }
  }
}

}  // namespace swan
