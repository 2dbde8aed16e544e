// What runs before and after the attention of attend.h: rows times a head's 128 x 128
// rotation, and the partial results of a row joined to one.
#include "attend.h"

namespace swan {

// y = mult * x . M, M = P (or its transpose) of the row's kv head, as M^T . x^T on MFMA: a
// workgroup takes 128 rows of one (sequence, head), wave w has dims 32 w .. + 31 of the
// result and holds that part of M^T.  Binary16 rows: M as two binary16 parts (22 bits);
// float32 rows: float32 MFMA.
template <typename T>
__global__ __launch_bounds__(256) void rotate_rows_kernel(RotateLaunch a) {
  const int tid = threadIdx.x, lane = tid & 63, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.x, b = bh / a.H, rows = a.rows[b];
  const int row0 = blockIdx.y * kTileRows;
  if (row0 >= rows) return;
  const float* P = a.P + (int64_t)(bh % a.H / (a.H / a.Hkv)) * kD * kD;
  const int j = 32 * wave + (lane & 31);  // the dim of the result that this lane's M^T row is
  auto m = [&](int i) { return a.transposed ? P[j * kD + i] : P[i * kD + j]; };
  constexpr bool k16 = sizeof(T) == 2;
  h8v mh[k16 ? 8 : 1], ml[k16 ? 8 : 1];
  f4v mf[k16 ? 1 : 16];
  if constexpr (k16) {
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = m(16 * s + 8 * hi + e);
        mh[s][e] = (_Float16)x;
        ml[s][e] = (_Float16)(x - (float)mh[s][e]);
      }
  } else {
#pragma unroll
    for (int s = 0; s < 16; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) mf[s][e] = m(8 * s + 4 * hi + e);
  }
#pragma unroll 1
  for (int t = 0; t < kTileRows / 32; ++t) {
    const int i = row0 + 32 * t + (lane & 31);
    if (row0 + 32 * t >= rows) return;
    const int64_t at = ((int64_t)bh * a.n + (i < rows ? i : rows - 1)) * kD;
    f16v acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    if constexpr (k16) {
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const h8v x = *(const h8v*)((const _Float16*)a.x + at + 16 * s + 8 * hi);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(mh[s], x, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ml[s], x, acc, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 16; ++s) {
        const f4v x = *(const f4v*)((const float*)a.x + at + 8 * s + 4 * hi);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc = __builtin_amdgcn_mfma_f32_32x32x2f32(mf[s][e], x[e], acc, 0, 0, 0);
      }
    }
    if (i < rows) {
      float* y = a.y + at + 32 * wave + 4 * hi;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *(f4v*)(y + 8 * e) = f4v{acc[4 * e] * a.mult, acc[4 * e + 1] * a.mult,
                                 acc[4 * e + 2] * a.mult, acc[4 * e + 3] * a.mult};
    }
  }
}

hipError_t launch_rotate_rows(const RotateLaunch& a) {
  const dim3 grid(a.B * a.H, (a.n + kTileRows - 1) / kTileRows);
  if (a.x_dtype == SWAN_F32)
    hipLaunchKernelGGL(rotate_rows_kernel<float>, grid, dim3(256), 0, a.stream, a);
  else
    hipLaunchKernelGGL(rotate_rows_kernel<_Float16>, grid, dim3(256), 0, a.stream, a);
  return hipGetLastError();
}

// One workgroup per row, thread t the dim t: out of partials (m, l, acc) the sums
// l = sum_i 2^(m_i - m) l_i, o = sum_i 2^(m_i - m) acc_i / l in fixed order.  The partials:
// those of swan_decode_attention's kernels (a decode step's own cache), then of each
// source, then the state (lse, 1, o).
constexpr int kMaxJoin = kMaxSplits + 1 + 2 * kMaxSlots + 1;
template <typename T>
__global__ __launch_bounds__(128) void join_kernel(JoinLaunch a) {
  __shared__ float wts[kMaxJoin];
  __shared__ float oh[kD];
  __shared__ float red[4];
  const int t = threadIdx.x, i = blockIdx.x % a.n, bh = blockIdx.x / a.n;
  const int b = bh / a.H;
  if (i >= a.rows[b]) return;
  const int64_t row = blockIdx.x;
  int own_ns = 0, own_n = 0;  // splits; with the buffer's partial (slot own_slots)
  if (a.own) {
    const int L = a.own_tab.len[b];
    const int np = pages_for(L > a.own_bb ? L - a.own_bb : 0);
    own_ns = np < a.own_tab.nsplit[b] ? np : a.own_tab.nsplit[b];
    own_n = own_ns + (min(L, a.own_bb) > 0 ? 1 : 0);
  }
  const int n0 = own_n, n1 = n0 + a.used[0][b], n2 = n1 + a.used[1][b];
  const int total = n2 + (a.o0 ? 1 : 0);
  const float* own = a.own + row * (a.own_slots + 1) * kPartFloats;
  const float* part = a.part + row * a.slots * kPartFloats;
  auto at = [&](int x) {  // x < n2
    if (x < n0) return own + (x < own_ns ? x : a.own_slots) * kPartFloats;
    return part + (x < n1 ? a.base[0] + x - n0 : a.base[1] + x - n1) * kPartFloats;
  };
  float mloc = -INFINITY;
  for (int x = t; x < total; x += 128)
    mloc = fmaxf(mloc, x < n2 ? at(x)[0] : a.lse0[row] * kLog2e);
  mloc = wave_max(mloc);
  if ((t & 63) == 0) red[t >> 6] = mloc;
  __syncthreads();
  const float m = fmaxf(red[0], red[1]);
  float lloc = 0.f;
  for (int x = t; x < total; x += 128) {
    const float mx = x < n2 ? at(x)[0] : a.lse0[row] * kLog2e;
    const float w = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx - m);
    wts[x] = w;
    lloc += w * (x < n2 ? at(x)[1] : 1.f);
  }
  lloc = wave_sum(lloc);
  if ((t & 63) == 0) red[2 + (t >> 6)] = lloc;
  __syncthreads();
  const float l = red[2] + red[3];
  float o = 0.f;
  for (int x = 0; x < n2; ++x) o = fmaf(wts[x], at(x)[4 + t], o);  // (an empty part's are 0)
  if (n2 < total && wts[n2] != 0.f) o = fmaf(wts[n2], a.o0[row * kD + t], o);
  o = l == 0.f ? 0.f : o / l;
  if (!a.out) {
    a.o[row * kD + t] = o;
    if (t == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) / kLog2e;
    return;
  }
  if (!a.P_vo) {
    ((T*)a.out)[row * kD + t] = (T)o;
    return;
  }
  oh[t] = o;
  __syncthreads();
  const float4* P = (const float4*)(a.P_vo + ((int64_t)(bh % a.H / (a.H / a.Hkv)) * kD + t) * kD);
  float r = 0.f;
#pragma unroll 8
  for (int j4 = 0; j4 < kD / 4; ++j4) {
    const float4 p = P[j4];
    r = fmaf(p.x, oh[4 * j4], r);
    r = fmaf(p.y, oh[4 * j4 + 1], r);
    r = fmaf(p.z, oh[4 * j4 + 2], r);
    r = fmaf(p.w, oh[4 * j4 + 3], r);
  }
  ((T*)a.out)[row * kD + t] = (T)r;
}

hipError_t launch_join(const JoinLaunch& a) {
  const dim3 grid((unsigned)((int64_t)a.B * a.H * a.n));
  if (a.dtype == SWAN_F32)
    hipLaunchKernelGGL(join_kernel<float>, grid, dim3(128), 0, a.stream, a);
  else
    hipLaunchKernelGGL(join_kernel<_Float16>, grid, dim3(128), 0, a.stream, a);
  return hipGetLastError();
}

}  // namespace swan
