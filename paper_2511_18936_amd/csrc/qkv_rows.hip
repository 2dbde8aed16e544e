// A layer's projections to the rows its cache and attention take: [q | k | v] of a token
// split into heads, each head of q and k divided by its root mean square and weighted
// (optional), then rotated to the token's position as swan_rope does it; v as it is.
//   r = 1 / sqrt(mean_j x_j^2 + eps),  y_j = x_j r w_j,
//   (y_j, y_{j+64}) turned by pos base^(-2j/128)
// in float64 and rounded once, so that without weights the bits are swan_rope's.
#include "swan_cache_ops.h"
#include "swan_layer_ops.h"

namespace swan {

typedef double f64x2 __attribute__((ext_vector_type(2)));

template <typename T>
__device__ __forceinline__ T stored(double y) {
  if constexpr (sizeof(T) == 2) return __builtin_bit_cast(T, f64_to_f16_bits_fast(y));
  else return (T)y;
}

template <typename T>
__device__ __forceinline__ void one_nan_of(T& y) {
  if constexpr (sizeof(T) == 2) y = __builtin_bit_cast(T, one_nan(__builtin_bit_cast(uint16_t, y)));
}

// 1 / sqrt(ms).  Binary16 rows: their mean square lies within float32's range, so the
// float32 estimate and one step of Newton's method (error squared, below 2^-44).
template <typename T>
__device__ __forceinline__ double inv_root(double ms) {
  if constexpr (sizeof(T) == 2) {
    const double r = (double)__builtin_amdgcn_rsqf((float)ms);
    return r == 0.0 ? 0.0 : r * (1.5 - 0.5 * ms * r * r);  // an infinity in the row: 0
  } else {
    return 1.0 / sqrt(ms);
  }
}

// N weights of role from element i on (16-byte aligned for N = 4)
template <typename T, int N>
__device__ __forceinline__ void weights_at(const QkvRowsLaunch& a, int role, int64_t i,
                                           double (&w)[N]) {
  struct alignas(N * 4) V32 {
    float v[N];
  };
  struct alignas(N * sizeof(T)) VT {
    T v[N];
  };
  if (sizeof(T) == 4 || a.w32) {
    const V32 x = *(const V32*)((const float*)a.w[role] + i);
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = (double)x.v[e];
  } else {
    const VT x = *(const VT*)((const T*)a.w[role] + i);
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = (double)(float)x.v[e];
  }
}

// sum over the `N` (16 or 64) lanes that hold a row
template <int N>
__device__ __forceinline__ double row_sum(double v) {
#pragma unroll
  for (int d = N / 2; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}

constexpr int kTilePos = 4;  // positions of a workgroup

// A workgroup takes 4 positions at a time: its 256 threads compute their 4 x 64 sines and
// cosines once for all heads, then a quarter wave (16 lanes of 4 pairs, 8-byte accesses for
// binary16) has a head's row of one position, wave w heads w, w + 4, ...
template <typename T>
__global__ __launch_bounds__(256) void qkv_rows_kernel(QkvRowsLaunch a) {
  __shared__ f64x2 cs[kTilePos][kD / 2];
  struct alignas(4 * sizeof(T)) Vec {
    T v[4];
  };
  const int t = threadIdx.x, wave = t >> 6, p = (t >> 4) & 3, l = t & 15;
  const int H = a.Hq + 2 * a.Hkv;
  const uint32_t n = (uint32_t)a.n, positions = (uint32_t)a.B * n;  // below 2^31
  const uint32_t tiles = (positions + kTilePos - 1) / kTilePos;
  const double freq = pow(a.base, -(2.0 * (t & 63)) / kD);
  for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    {
      const uint32_t at = tile * kTilePos + wave;
      if (at < positions) {
        const uint32_t b = at / n;
        double s, c;
        sincos(((double)a.pos0[b] + (double)(at - b * n)) * freq, &s, &c);
        cs[wave][t & 63] = f64x2{c, s};
      }
    }
    __syncthreads();
    const uint32_t at = tile * kTilePos + p;
    const bool live = at < positions;
    const int b = live ? (int)(at / n) : 0, i = live ? (int)(at - b * n) : 0;
    double c[4], s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f64x2 v = cs[p][4 * l + e];
      c[e] = v.x;
      s[e] = v.y;
    }
    const T* row = (const T*)a.x + b * a.seq + i * a.row + 4 * l;
    if (live) {
      for (int h = wave; h < H; h += 4) {
        const Vec lo = *(const Vec*)(row + h * kD), hi = *(const Vec*)(row + h * kD + kD / 2);
        const int role = h < a.Hq ? 0 : h < a.Hq + a.Hkv ? 1 : 2;
        const int hr = role == 0 ? h : role == 1 ? h - a.Hq : h - a.Hq - a.Hkv;
        T* to = (T*)a.out[role] +
                (((int64_t)b * (role == 0 ? a.Hq : a.Hkv) + hr) * a.n + i) * kD + 4 * l;
        Vec y = lo, z = hi;
        if (role < 2) {
          double x0[4], x1[4];
          bool nan = false;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x0[e] = (double)(float)lo.v[e];
            x1[e] = (double)(float)hi.v[e];
            nan |= __builtin_isunordered((float)lo.v[e], (float)hi.v[e]);
          }
          if (a.w[role]) {
            double ss = 0.0;
#pragma unroll
            for (int e = 0; e < 4; ++e) ss += x0[e] * x0[e] + x1[e] * x1[e];
            const double r = inv_root<T>(row_sum<16>(ss) * (1.0 / kD) + a.eps);
            double w0[4], w1[4];
            weights_at<T>(a, role, (int64_t)hr * a.wstep + 4 * l, w0);
            weights_at<T>(a, role, (int64_t)hr * a.wstep + 4 * l + kD / 2, w1);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              x0[e] *= r * w0[e];
              x1[e] *= r * w1[e];
            }
            nan |= !(r - r == 0.0);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            y.v[e] = stored<T>(x0[e] * c[e] - x1[e] * s[e]);
            z.v[e] = stored<T>(x1[e] * c[e] + x0[e] * s[e]);
          }
          if (nan)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              one_nan_of(y.v[e]);
              one_nan_of(z.v[e]);
            }
        }
        *(Vec*)to = y;
        *(Vec*)(to + kD / 2) = z;
      }
    }
    __syncthreads();
  }
}

// Few rows: a wave per (position, head), lane l the pair (l, l + 64); the row and its
// weights are loaded before the chain of pow and sincos, which bounds it.
template <typename T>
__global__ __launch_bounds__(64) void qkv_rows_few_kernel(QkvRowsLaunch a) {
  const int l = threadIdx.x, i = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const T* row = (const T*)a.x + b * a.seq + i * a.row + (int64_t)h * kD + l;
  const T lo = row[0], hi = row[kD / 2];
  const int role = h < a.Hq ? 0 : h < a.Hq + a.Hkv ? 1 : 2;
  const int hr = role == 0 ? h : role == 1 ? h - a.Hq : h - a.Hq - a.Hkv;
  T* to = (T*)a.out[role] + (((int64_t)b * (role == 0 ? a.Hq : a.Hkv) + hr) * a.n + i) * kD + l;
  if (role == 2) {
    to[0] = lo;
    to[kD / 2] = hi;
    return;
  }
  double x0 = (double)(float)lo, x1 = (double)(float)hi;
  bool nan = x0 != x0 || x1 != x1;
  if (a.w[role]) {
    double w0[1], w1[1];
    weights_at<T>(a, role, (int64_t)hr * a.wstep + l, w0);
    weights_at<T>(a, role, (int64_t)hr * a.wstep + l + kD / 2, w1);
    const double r = inv_root<T>(row_sum<64>(x0 * x0 + x1 * x1) * (1.0 / kD) + a.eps);
    x0 *= r * w0[0];
    x1 *= r * w1[0];
    nan |= !(r - r == 0.0);
  }
  double s, c;
  sincos(((double)a.pos0[b] + (double)i) * pow(a.base, -(2.0 * l) / kD), &s, &c);
  T y = stored<T>(x0 * c - x1 * s), z = stored<T>(x1 * c + x0 * s);
  if (nan) {
    one_nan_of(y);
    one_nan_of(z);
  }
  to[0] = y;
  to[kD / 2] = z;
}

template <typename T>
static hipError_t launch_qkv_rows_t(const QkvRowsLaunch& a) {
  const int64_t positions = (int64_t)a.B * a.n;
  const int H = a.Hq + 2 * a.Hkv;
  if (positions * H <= 4096 && H <= 65535) {
    hipLaunchKernelGGL(qkv_rows_few_kernel<T>, dim3(a.n, H, a.B), dim3(64), 0, a.stream, a);
    return hipGetLastError();
  }
  const int64_t tiles = (positions + kTilePos - 1) / kTilePos;
  const dim3 grid((unsigned)(tiles < 2048 ? tiles : 2048));
  hipLaunchKernelGGL(qkv_rows_kernel<T>, grid, dim3(256), 0, a.stream, a);
  return hipGetLastError();
}

hipError_t launch_qkv_rows(const QkvRowsLaunch& a) {
  return a.dtype == SWAN_F32 ? launch_qkv_rows_t<float>(a) : launch_qkv_rows_t<_Float16>(a);
}

}  // namespace swan
