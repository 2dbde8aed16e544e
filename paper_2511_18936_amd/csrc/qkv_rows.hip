// A layer's projections to the rows its cache and attention take: [q | k | v] of a token
// split into heads, each head of q and k divided by its root mean square and weighted
// (optional), then rotated to the token's position as swan_rope does it; v as it is.
//   r = 1 / sqrt(mean_j x_j^2 + eps),  y_j = x_j r w_j,
//   (y_j, y_{j+64}) turned by pos base^(-2j/128)
// in float64 and rounded once, so that without weights the bits are swan_rope's.
//
// Bound by memory for long prompts: 8 x 8190 positions of 32 + 2 x 32 heads without norms
// 615 us, 5.2 TB/s read and written (a large copy: 4.8).  In between latency counts: 1999
// positions of 32 + 2 x 8 heads with norms 13.7 us, 3.6 TB/s, where waves wait for half of
// their time (pow, sincos and a barrier come before a row's load, and the workgroups are few)
// and vector instructions, most of them float64, are issued in 28 % of the cycles; 16 lanes
// have a row and 4 pairs each, and the sines are shared by the heads; 3 x 517 positions of
// 12 + 2 x 4 float32 heads 9.6 us.  Single tokens (4 x 48 heads) 3 us, the chain of pow and
// sincos.
#include "swan_cache_ops.h"
#include "swan_layer_ops.h"

namespace swan {

typedef double f64x2 __attribute__((ext_vector_type(2)));

// y rounded once.  Binary16: y cut to float32's 24 bits, the last one set if anything was
// cut off (round to odd), is a float32 number that rounds to binary16 as y does.  (The same
// as f64_to_f16_bits_fast, half the instructions, no branch.)
template <typename T>
__device__ __forceinline__ T stored(double y) {
  if constexpr (sizeof(T) == 2) {
    const uint64_t bits = (uint64_t)__double_as_longlong(y);
    const uint32_t lo = (uint32_t)bits, cut = (lo & 0x1FFFFFFFu) + 0x1FFFFFFFu;
    const uint64_t odd = (bits & 0xFFFFFFFF00000000ull) | ((lo | cut) & 0xE0000000u);
    return (T)(float)__longlong_as_double((long long)odd);
  } else {
    return (T)y;
  }
}

template <typename T>
__device__ __forceinline__ void one_nan_of(T& y) {
  if constexpr (sizeof(T) == 2) y = __builtin_bit_cast(T, one_nan(__builtin_bit_cast(uint16_t, y)));
}

// 1 / sqrt(ms).  Binary16 rows: the float64 estimate, within 2^-22, and one step of Newton's
// method (error squared, below 2^-43).  Not the float32 one: ms may be below or above its
// range, for a row of zeros with a tiny eps or any row with a huge one.
template <typename T>
__device__ __forceinline__ double inv_root(double ms) {
  if constexpr (sizeof(T) == 2) {
    const double r = __builtin_amdgcn_rsq(ms);
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

// sum over the 16 lanes of a row of lanes, then (N = 64) over the wave
template <int CTRL>
__device__ __forceinline__ double rotated(double v) {
  const uint64_t x = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, 0xF, 0xF, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, 0xF, 0xF, true);
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
template <int N>
__device__ __forceinline__ double row_sum(double v) {
  v += rotated<0x128>(v);
  v += rotated<0x124>(v);
  v += rotated<0x122>(v);
  v += rotated<0x121>(v);
  if constexpr (N == 64) {
    v += __shfl_xor(v, 16, 64);
    v += __shfl_xor(v, 32, 64);
  }
  return v;
}

constexpr int kTilePos = 4;  // positions of a workgroup

template <typename T>
struct alignas(4 * sizeof(T)) Four {
  T v[4];
};

// One row's 4 + 4 elements of a lane (of 16): norm with weights w (NULL: none), rotation
template <typename T>
__device__ __forceinline__ void turn_row(Four<T>& lo, Four<T>& hi, const double* w, double eps,
                                         const double (&c)[4], const double (&s)[4]) {
  double x0[4], x1[4];
  bool nan = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x0[e] = (double)(float)lo.v[e];
    x1[e] = (double)(float)hi.v[e];
    nan |= __builtin_isunordered((float)lo.v[e], (float)hi.v[e]);
  }
  if (w) {
    double ss = 0.0;
#pragma unroll
    for (int e = 0; e < 4; ++e) ss += x0[e] * x0[e] + x1[e] * x1[e];
    const double r = inv_root<T>(row_sum<16>(ss) * (1.0 / kD) + eps);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x0[e] *= r * w[e];
      x1[e] *= r * w[4 + e];
    }
    nan |= !(r - r == 0.0);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    lo.v[e] = stored<T>(x0[e] * c[e] - x1[e] * s[e]);
    hi.v[e] = stored<T>(x1[e] * c[e] + x0[e] * s[e]);
  }
  if (nan)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      one_nan_of(lo.v[e]);
      one_nan_of(hi.v[e]);
    }
}

// A workgroup takes 4 positions at a time and `heads` of their heads (grid: positions,
// chunks of heads): its 256 threads compute the 4 x 64 sines and cosines once for all of
// them, then a quarter wave (16 lanes of 4 pairs, 8-byte accesses for binary16) has a head's
// row of one position, wave w every fourth head, two at a time.
template <typename T>
__global__ __launch_bounds__(256) void qkv_rows_kernel(QkvRowsLaunch a, int heads) {
  __shared__ f64x2 cs[kTilePos][kD / 2];
  using Vec = Four<T>;
  const int t = threadIdx.x, wave = t >> 6, p = (t >> 4) & 3, l = t & 15;
  const int h0 = blockIdx.y * heads, h1 = min(a.Hq + 2 * a.Hkv, h0 + heads);
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
    if (at < positions) {
      const int b = (int)(at / n), i = (int)(at - b * n);
      const T* row = (const T*)a.x + b * a.seq + i * a.row + 4 * l;
      double c[4], s[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f64x2 v = cs[p][4 * l + e];
        c[e] = v.x;
        s[e] = v.y;
      }
      int first = 0;
#pragma unroll
      for (int role = 0; role < 3; ++role) {
        const int count = role == 0 ? a.Hq : a.Hkv, last = min(first + count, h1);
        T* out = (T*)a.out[role] + (((int64_t)b * count - first) * a.n + i) * kD + 4 * l;
        const bool norm = role < 2 && a.w[role] != nullptr;
        double w[8];
        if (norm && a.wstep == 0) {
          weights_at<T>(a, role, 4 * l, *(double(*)[4])w);
          weights_at<T>(a, role, 4 * l + kD / 2, *(double(*)[4])(w + 4));
        }
        // the first of this wave's heads that is the chunk's and this role's
        for (int h = max(first, h0) + wave; h < last; h += 8) {
          const bool two = h + 4 < last;
          Vec lo[2], hi[2];
          lo[0] = *(const Vec*)(row + h * kD);
          hi[0] = *(const Vec*)(row + h * kD + kD / 2);
          if (two) {
            lo[1] = *(const Vec*)(row + (h + 4) * kD);
            hi[1] = *(const Vec*)(row + (h + 4) * kD + kD / 2);
          }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (x == 1 && !two) break;
            if (role < 2) {
              if (norm && a.wstep) {
                const int64_t at = (int64_t)(h + 4 * x - first) * a.wstep + 4 * l;
                weights_at<T>(a, role, at, *(double(*)[4])w);
                weights_at<T>(a, role, at + kD / 2, *(double(*)[4])(w + 4));
              }
              turn_row<T>(lo[x], hi[x], norm ? w : nullptr, a.eps, c, s);
            }
            T* to = out + (int64_t)(h + 4 * x) * a.n * kD;
            *(Vec*)to = lo[x];
            *(Vec*)(to + kD / 2) = hi[x];
          }
        }
        first += count;
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
  // Few positions split their heads, 4 at least to each, over 768 workgroups: fewer leave
  // processors idle, more repeat the sines and cosines.  Binary16 with norms, us with 512, 768
  // and 1024: 32 + 2 x 8 heads x 300 positions 5.4, 5.4, 7.0, x 1100 12.9, 11.4, 12.3, x 1999
  // 13.7, 13.7, 15.2; 32 + 2 x 32 heads x 500 9.7, 9.3, 10.8, x 1500 19.6, 16.5, 16.5; 16 + 2
  // heads x 1000 6.4, 6.8, 6.9; float32, 12 + 2 x 4 heads, 3 x 517 9.6, 9.6, 10.4.
  const int64_t tiles = (positions + kTilePos - 1) / kTilePos;
  int64_t chunks = 768 / tiles;
  chunks = chunks < 1 ? 1 : chunks > (H + 3) / 4 ? (H + 3) / 4 : chunks;
  const int heads = (int)(((H + chunks - 1) / chunks + 3) / 4 * 4);
  const dim3 grid((unsigned)(tiles < 2048 ? tiles : 2048), (unsigned)((H + heads - 1) / heads));
  hipLaunchKernelGGL(qkv_rows_kernel<T>, grid, dim3(256), 0, a.stream, a, heads);
  return hipGetLastError();
}

hipError_t launch_qkv_rows(const QkvRowsLaunch& a) {
  return a.dtype == SWAN_F32 ? launch_qkv_rows_t<float>(a) : launch_qkv_rows_t<_Float16>(a);
}

}  // namespace swan
