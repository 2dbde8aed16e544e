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
// than Lag::kBy, and is set Lag::kHead below the maximum.  Binary16: by more than 15, then 7
// below, so p (2^15 at most, below 65504) uses the upper part of its type's range.  It goes to
// the second product as two parts, p rounded and what that left: within 2^-23 of p (and 2^-25
// absolutely, where a row's largest p is 2^7 at least).  So the weights are float32's but for a
// bit, and the sum is taken of the float32 p.  One part alone leaves an error of up to 2^-11 in
// each weight, as much as the rounding of a binary16 result, for less time (32 query heads on
// 8, 4096 causal rows: 161 us against 217; 4 x 256 rows over 4 x 8192 cached keys 230 against
// 277; 32 tokens behind 32768 keys 86 against 93).  Float32: whenever a score exceeds it, then
// 15 above the score, so p is 1 at most and the sums reach no further than the values do.
//
// Why 32 rows a wave and 64 keys a tile: the accumulator (64 registers a lane), the queries
// (32, or 64 in two parts) and the scores of a tile (32) fill the 256 registers that two
// waves per SIMD leave each, so one wave's products run while the other takes exponentials;
// the wider MFMA shape halves the operand reads of the 16 x 16 one; and 64 keys are a page.
#pragma once

#include "swan_device.h"
#include "swan_layer_ops.h"

namespace swan {

typedef _Float16 h2v __attribute__((ext_vector_type(2)));
typedef _Float16 h4v __attribute__((ext_vector_type(4)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));

template <typename T>
struct Lag {
  static constexpr float kHead = sizeof(T) == 2 ? 7.f : -15.f, kBy = sizeof(T) == 2 ? 15.f : 0.f;
};
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

// What numbers with this largest magnitude are multiplied by before they are split into two
// binary16 parts (within 2^-23 of them, and 2^-38 of the largest: its parts would be subnormal
// as they are), and c, what that leaves to multiply results by: 2^(13 - exponent) and the
// inverse; 1 for zeros, infinities or NaNs.
__device__ __forceinline__ float split_scale(float top, float& c) {
  const int ex = (int)((__float_as_uint(top) >> 23) & 0xFF) - 127;
  const int up = top > 0.f && ex < 128 ? 13 - (ex < -100 ? -100 : ex) : 0;
  c = __builtin_ldexpf(1.f, -up);
  return __builtin_ldexpf(1.f, up);
}

#define SWAN_LDS __attribute__((address_space(3)))

// A tile in LDS: 64 keys' rows of K or V, row-major as in memory, so that they can be
// loaded without passing through registers.  The 16-byte pieces of row `key` are permuted,
// piece c at place c ^ turn(key), which puts on distinct banks what the products read
// together: the same piece of 16 keys (K), and of V the 4 x 2 pieces that a transposing
// read takes from 4 keys (binary16) or one dim group of two keys (float32).
template <typename T>
struct Rows {
  static constexpr int kBytes = kD * (int)sizeof(T);        // of a row
  static constexpr int kTile = kTileKeys * kBytes;          // of a tile
  static constexpr int kPieces = kBytes / 16;               // of a row
  __device__ static __forceinline__ int turn(int key) {
    if constexpr (sizeof(T) == 2) return (key & 3) << 2 | (key >> 2 & 3);
    else return (key >> 2 & 1) << 3 | (key & 3) << 1 | (key >> 3 & 1);
  }
  // byte of element d of row `key`
  __device__ static __forceinline__ int at(int key, int d) {
    constexpr int N = 16 / (int)sizeof(T);
    return key * kBytes + ((d / N) ^ turn(key)) * 16 + d % N * (int)sizeof(T);
  }
};

// Loads a tile's first `rows` rows (at most 64) from p, zeros in the place of the others;
// dma_wait() and a barrier before it is read.  Wave w has rows 16 w .. + 15, 1 KiB at a
// time in the order of the places; `from` are the lane's places in memory (dma_from).
// Binary16: asynchronous, straight to LDS, in assembly because the compiler would have
// every later read of LDS wait for it.  Float32, whose tiles lie beyond the 64 KiB that such
// loads reach: through registers.
template <typename T>
struct DmaFrom {
  static constexpr int N = Rows<T>::kTile / 4096;
  uint32_t at[N];
};
template <typename T>
__device__ __forceinline__ DmaFrom<T> dma_from(int wave, int lane) {
  using R = Rows<T>;
  DmaFrom<T> f;
#pragma unroll
  for (int x = 0; x < DmaFrom<T>::N; ++x) {
    const int key = 16 * wave + x * (1024 / R::kBytes) + lane / R::kPieces;
    f.at[x] = (uint32_t)(key * R::kBytes + ((lane % R::kPieces) ^ R::turn(key)) * 16);
  }
  return f;
}
template <typename T, bool kAsync = sizeof(T) == 2>
__device__ __forceinline__ void dma_tile(char* lds, const T* p, int rows, const DmaFrom<T>& from,
                                         int wave) {
  typedef int i4v __attribute__((ext_vector_type(4)));
  const uint64_t base = (uint64_t)p;
  rows = rows > kTileKeys ? kTileKeys : rows < 0 ? 0 : rows;
  if constexpr (!kAsync) {
    u32x4 r[DmaFrom<T>::N];
#pragma unroll
    for (int x = 0; x < DmaFrom<T>::N; ++x)
      r[x] = from.at[x] < (uint32_t)(rows * Rows<T>::kBytes)
                 ? *(const u32x4*)((const char*)p + from.at[x]) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int x = 0; x < DmaFrom<T>::N; ++x)
      *(u32x4*)(lds + wave * (Rows<T>::kTile / 4) + 1024 * x + 16 * __lane_id()) = r[x];
    return;
  }
  const i4v rsrc = {__builtin_amdgcn_readfirstlane((int)(uint32_t)base),
                    __builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32)),
                    __builtin_amdgcn_readfirstlane(rows * Rows<T>::kBytes), 0x00020000};
  const uint32_t to = __builtin_amdgcn_readfirstlane(
      (uint32_t)(uintptr_t)(SWAN_LDS char*)lds + wave * (Rows<T>::kTile / 4));
  // (wait states: 5 from v_readfirstlane's SGPRs to a load that reads them, 1 from M0's write)
#pragma unroll
  for (int x = 0; x < DmaFrom<T>::N; ++x)
    asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(from.at[x]), "s"(rsrc),
                 "{m0}"(to + 1024 * x)
                 : "memory");
}
__device__ __forceinline__ void dma_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// The products, by element type.
template <typename T>
struct Tile;

template <>
struct Tile<_Float16> {
  using R = Rows<_Float16>;
  // Q of the wave's rows: dims 16 s + 8 (lane / 32) .. + 7 of row lane % 32; kLow: a second
  // part for what the first rounds off
  template <bool kLow>
  struct Q {
    h8v hi[8], lo[kLow ? 8 : 1];
  };
  static constexpr int kSteps = 16;  // of scores()
  // S += K . Q^T, the steps (16 dims of one half of the keys) from s0 to s1; the first two
  // start from zero
  template <bool kLow>
  __device__ static __forceinline__ void scores(const char* kb, const Q<kLow>& q, int lane,
                                                f16v (&S)[2], int s0 = 0, int s1 = kSteps) {
    const int key = lane & 31;
#pragma unroll
    for (int x = s0; x < s1; ++x) {
      const int t = x & 1, s = x >> 1;
      const h8v k = *(const SWAN_LDS h8v*)((SWAN_LDS const char*)kb + 32 * t * R::kBytes +
                                           R::at(key, 16 * s + 8 * (lane >> 5)));
      if (s == 0) S[t] = f16v{};
      S[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q.hi[s], S[t], 0, 0, 0);
      if constexpr (kLow) S[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q.lo[s], S[t], 0, 0, 0);
    }
  }
  // V^T of dims 32 d .. + 31 (lane % 32) and the lane's 8 keys of 16 s .. + 15, as the
  // scores' layout has them: 4 (lane / 32) + {0..3, 8..11}
  __device__ static __forceinline__ h8v value(const char* vb, int lane, int d, int s) {
    typedef short s4v __attribute__((ext_vector_type(4)));
    const int j = lane & 15, dim = 32 * d + 16 * (lane >> 4 & 1) + 4 * (j & 3);
    const int key = 4 * (lane >> 5) + (j >> 2);
    s4v x[2];
#pragma unroll
    for (int w = 0; w < 2; ++w)
      x[w] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (SWAN_LDS s4v*)((SWAN_LDS char*)vb + 16 * s * R::kBytes + R::at(8 * w + key, dim)));
    const u32x2 a = __builtin_bit_cast(u32x2, x[0]), b = __builtin_bit_cast(u32x2, x[1]);
    return __builtin_bit_cast(h8v, u32x4{a.x, a.y, b.x, b.y});
  }
  // p = exp2(S c - ref), O += V^T . p; returns the lane's sum of p.  kNext: the scores of
  // the next tile are taken in between, so that its products run while the exponentials
  // are computed.  kOdd: some value may be infinite, whose product with a part of p that is 0
  // or negative would make a NaN: the parts meet it cut to the finite range, and what was cut
  // off (0 of the finite ones, whose sums keep their bits) is added for a p above 0.
  template <bool kNext, bool kOdd, bool kLow>
  __device__ static __forceinline__ float values(const char* vb, const f16v (&S)[2], float c,
                                                 float ref, int lane, f16v (&O)[4],
                                                 const char* next_k, const Q<kLow>& q,
                                                 f16v (&next)[2]) {
    float l = 0.f;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if constexpr (kNext) scores<kLow>(next_k, q, lane, next, 4 * s, 4 * s + 4);
      h8v hi, lo, some;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = __builtin_amdgcn_exp2f(fmaf(S[s >> 1][8 * (s & 1) + e], c, -ref));
        l += p;
        hi[e] = (_Float16)p;
        lo[e] = (_Float16)(p - (float)hi[e]);
        if constexpr (kOdd) some[e] = p > 0.f ? (_Float16)1.f : (_Float16)0.f;
      }
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        h8v v = value(vb, lane, d, s);
        if constexpr (kOdd) {
          const h8v all = v;
          v = __builtin_elementwise_max(
              __builtin_elementwise_min(v, (h8v)(_Float16)65504.f), (h8v)(_Float16)-65504.f);
          O[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(all - v, some, O[d], 0, 0, 0);
        }
        O[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, hi, O[d], 0, 0, 0);
        O[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, lo, O[d], 0, 0, 0);
      }
    }
    return l;
  }
};

template <>
struct Tile<float> {
  using R = Rows<float>;
  template <bool kLow>
  struct Q {
    f4v hi[16];  // dims 8 s + 4 (lane / 32) .. + 3
  };
  static constexpr int kSteps = 32;
  template <bool kLow>
  __device__ static __forceinline__ void scores(const char* kb, const Q<kLow>& q, int lane,
                                                f16v (&S)[2], int s0 = 0, int s1 = kSteps) {
    const int key = lane & 31;
#pragma unroll
    for (int x = s0; x < s1; ++x) {
      const int t = x & 1, s = x >> 1;
      const f4v k = *(const SWAN_LDS f4v*)((SWAN_LDS const char*)kb + 32 * t * R::kBytes +
                                           R::at(key, 8 * s + 4 * (lane >> 5)));
      if (s == 0) S[t] = f16v{};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        S[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], q.hi[s][e], S[t], 0, 0, 0);
    }
  }
  template <bool kNext, bool kOdd, bool kLow>
  __device__ static __forceinline__ float values(const char* vb, const f16v (&S)[2], float c,
                                                 float ref, int lane, f16v (&O)[4],
                                                 const char* next_k, const Q<kLow>& q,
                                                 f16v (&next)[2]) {
    float l = 0.f;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      if constexpr (kNext) scores<kLow>(next_k, q, lane, next, 4 * s, 4 * s + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(fmaf(S[s >> 2][4 * (s & 3) + e], c, -ref));
        l += p;
        const int key = 8 * s + 4 * (lane >> 5) + e;
#pragma unroll
        for (int d = 0; d < 4; ++d)
          O[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(
              *(const SWAN_LDS float*)((SWAN_LDS const char*)vb + R::at(key, 32 * d + (lane & 31))),
              p, O[d], 0, 0, 0);
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
template <typename T>
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
  // Lag::kBy (of no other row: a row's bits do not depend on its neighbours'); mx: the
  // maximum of the row's scores x c
  __device__ __forceinline__ void raise(float mx) {
#pragma clang fp contract(off)
    const bool up = mx - ref > Lag<T>::kBy;
    if (__any(up)) {
      const float to = up ? mx - Lag<T>::kHead : ref;
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
  // whether some sum is no number (0 times it is none)
  __device__ __forceinline__ bool odd() const {
    f4v z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) z[d] = fmaf(O[d][i], 0.f, z[d]);
    return !(z[0] + z[1] + z[2] + z[3] == 0.f);
  }
};

__device__ __forceinline__ float tile_max(const f16v (&S)[2]) {
  float m = S[0][0];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(m, S[t][i]);
  return max_halves(m);
}

// Raises the reference for the scores S x c of a tile, of which values() takes S c - ref: c and
// ref as it needs them.  It rounds the difference once, the reference is made of rounded
// products; from 2^28 on these are further apart than Lag::kHead, so where they pass kFar S itself
// becomes the difference of the rounded product (a power of two as c has none to round).
constexpr float kFar = 0x1p20f;
template <typename T>
__device__ __forceinline__ float take_scores(RowState<T>& rs, f16v (&S)[2], float& c) {
#pragma clang fp contract(off)
  const float mx = tile_max(S) * c;
  rs.raise(mx);
  float ref = rs.safe_ref();
  const bool far = fabsf(mx) > kFar && mx != -INFINITY;  // (of this row alone)
  if (__any(far)) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x = S[t][i] * c;
        S[t][i] = far ? x - ref : S[t][i];
      }
    c = far ? 1.f : c;
    ref = far ? 0.f : ref;
  }
  return ref;
}

// A unit: kv head, split and row tile (in grid order) of group j
struct Unit {
  int j, h, split, nsplit, tile;
};
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

// Unit u of a group: kv head u % Hkv (so that a head's tiles fall to few of the 8 XCDs and
// its keys stay in their L2), then the split, then the row tile.
__device__ __forceinline__ Unit unit_at(const AttendLaunch& a, int block) {
  Unit n;
  n.j = group_of(a, block);
  const uint32_t u = (uint32_t)(block - a.unit0[n.j]), rest = a.by_hkv.of(u);
  n.h = (int)(u - rest * a.by_hkv.d);
  n.nsplit = a.nsplit[n.j];
  n.tile = (int)rest;
  n.split = 0;
  if (n.nsplit > 1) {
    n.tile = (int)(rest / (uint32_t)n.nsplit);
    n.split = (int)(rest - (uint32_t)n.tile * (uint32_t)n.nsplit);
  }
  return n;
}
// first of nt tiles of a split: nt / nsplit of them each, the first ones one more
__device__ __forceinline__ int split_first(int nt, int split, int nsplit) {
  if (nsplit == 1) return split * nt;
  const int each = nt / nsplit;
  return each * split + min(split, nt - each * nsplit);
}

// The sequence and row that a group's tokens are.  Lane l holds list entry l, read once: a
// search through the launch's table itself would be a chain of loads, each with the whole
// latency of memory.
struct Tokens {
  int tok0, seq;
  __device__ __forceinline__ Tokens(const AttendLaunch& a, int lane)
      : tok0(a.tok0[lane]), seq(a.seq[lane]) {}
  // token tok of group j: sequence b and row i of it (every lane of the wave asks)
  __device__ __forceinline__ void at(const AttendLaunch& a, int j, int tok, int& b, int& i) const {
    int lo = a.first[j], hi = a.first[j + 1];  // uniform
    while (__any(hi - lo > 1)) {
      const int mid = (lo + hi) >> 1;
      const int first = __shfl(tok0, mid, 64);  // (by every lane: each is read from)
      const bool up = hi - lo > 1 && tok >= first;
      lo = up ? mid : lo;
      hi = up ? hi : mid > lo ? mid : lo + 1;
    }
    b = __shfl(seq, lo, 64);
    i = tok - __shfl(tok0, lo, 64);
  }
};

// the row's partial: reference, sum, accumulator
template <typename T>
__device__ __forceinline__ void write_partial(const AttendLaunch& a, const RowState<T>& st,
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
