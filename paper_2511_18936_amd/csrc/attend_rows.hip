// What runs before and after the attention of attend.h: rows times a head's 128 x 128
// rotation, and the partial results of a row joined to one.
#include "attend.h"

namespace swan {

// y = mult * x . M, M = P (or its transpose) of the row's kv head, as M^T . x^T on MFMA: a
// workgroup takes 128 rows of one (sequence, head), wave w has dims 32 w .. + 31 of the
// result and holds that part of M^T.  Binary16 rows: M as two binary16 parts (split_scale by
// the largest entry of the wave's part); float32 rows: float32 MFMA.  The matrix is read once
// per 128 rows, strided, as its 64 KiB stay in L2; the rows' float32 results are most of the
// traffic: 32768 binary16 rows 11 us, 2.2 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void rotate_rows_kernel(RotateLaunch a) {
  const int tid = threadIdx.x, lane = tid & 63, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.x % (a.B * a.H), b = bh / a.H, rows = a.rows[b];
  const int row0 = blockIdx.x / (a.B * a.H) * kTileRows;
  if (row0 >= rows) return;
  const float* P = a.P + (int64_t)(bh % a.H / (a.H / a.Hkv)) * kD * kD;
  const int j = 32 * wave + (lane & 31);  // the dim of the result that this lane's M^T row is
  auto m = [&](int i) { return a.transposed ? P[j * kD + i] : P[i * kD + j]; };
  constexpr bool k16 = sizeof(T) == 2;
  h8v mh[k16 ? 8 : 1], ml[k16 ? 8 : 1];
  f4v mf[k16 ? 1 : 16];
  float c = 1.f;
  if constexpr (k16) {
    float top = 0.f, x[kD / 2];
#pragma unroll
    for (int i = 0; i < kD / 2; ++i) {
      x[i] = m(16 * (i >> 3) + 8 * hi + (i & 7));
      top = fmaxf(top, fabsf(x[i]));
    }
    const float f = split_scale(wave_max(top), c);
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = x[8 * s + e] * f;
        mh[s][e] = (_Float16)y;
        ml[s][e] = (_Float16)(y - (float)mh[s][e]);
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
        *(f4v*)(y + 8 * e) = f4v{acc[4 * e] * c * a.mult, acc[4 * e + 1] * c * a.mult,
                                 acc[4 * e + 2] * c * a.mult, acc[4 * e + 3] * c * a.mult};
    }
  }
}

hipError_t launch_rotate_rows(const RotateLaunch& a) {
  const dim3 grid(a.B * a.H * ((a.n + kTileRows - 1) / kTileRows));  // at most B H n
  if (a.x_dtype == SWAN_F32)
    hipLaunchKernelGGL(rotate_rows_kernel<float>, grid, dim3(256), 0, a.stream, a);
  else
    hipLaunchKernelGGL(rotate_rows_kernel<_Float16>, grid, dim3(256), 0, a.stream, a);
  return hipGetLastError();
}

// The parts of a row: (m, l, acc) of swan_decode_attention's kernels over a decode step's
// own cache, then those of each source, then the state (lse, 1, o).  Their sum is
//   l = sum_i 2^(m_i - m) l_i,  o = sum_i 2^(m_i - m) acc_i / l
// (an empty part has m = -inf, l = 0 and a zero accumulator).
struct Parts {
  const float* own;
  const float* part;
  const float* lse0;
  int own_ns, own_slots, n0, n1, n2, total, base0, base1;
  __device__ __forceinline__ Parts(const JoinLaunch& a, int b, int64_t row) {
    own_slots = a.own_slots;
    own_ns = n0 = 0;
    if (a.own) {
      const int L = a.own_tab.len[b];
      const int np = pages_for(L > a.own_bb ? L - a.own_bb : 0);
      own_ns = np < a.own_tab.nsplit[b] ? np : a.own_tab.nsplit[b];
      n0 = own_ns + (min(L, a.own_bb) > 0 ? 1 : 0);  // the last: the buffer's, in slot own_slots
    }
    n1 = n0 + a.used[0][b];
    n2 = n1 + a.used[1][b];
    total = n2 + (a.o0 ? 1 : 0);
    base0 = a.base[0] - n0;
    base1 = a.base[1] - n1;
    own = a.own + row * (a.own_slots + 1) * kPartFloats;
    part = a.part + row * a.slots * kPartFloats;
    lse0 = a.lse0 + row;
  }
  __device__ __forceinline__ const float* at(int x) const {  // x < n2
    if (x < n0) return own + (x < own_ns ? x : own_slots) * kPartFloats;
    return part + (x < n1 ? base0 + x : base1 + x) * kPartFloats;
  }
  __device__ __forceinline__ float m_of(int x) const {  // x < total
#pragma clang fp contract(off)  // (rounded, as the maximum of all that it is compared with)
    return x < n2 ? at(x)[0] : *lse0 * kLog2e;
  }
};

// Decode: a workgroup per row.  The weights of its parts once, in LDS; then each of the groups
// of 32 threads (lanes of 4 dims) adds up its share of the parts, and the result is turned
// back.  P_vo is read in whole rows, on their way while the parts are added; its products
// are summed over a group's lanes through LDS (1024 rows: 4 us less than a row of P_vo per
// thread, 18 less than exchanges between the lanes).  Twice the threads gain nothing.  1024 rows of 67
// parts 11 us (3.3 TB/s of parts), 128 rows of 18 4.7 us: the latencies of the parts'
// references, of their accumulators, of P_vo, one after another.
constexpr int kMaxJoin = kMaxSplits + 1 + 2 * kMaxSlots + 1;
constexpr int kJoinGroups = 4;
constexpr int kJoinThreads = 32 * kJoinGroups;
template <typename T>
__global__ __launch_bounds__(kJoinThreads) void join_decode_kernel(JoinLaunch a) {
  constexpr int NG = kJoinGroups, NT = kJoinThreads, NR = kD / NG;
  __shared__ float wts[kMaxJoin];
  __shared__ f4v sums[NG][kD / 4];
  __shared__ __align__(16) float oh[kD];
  __shared__ float red[2 * NG];
  __shared__ float turn[kD][33];
  const int t = threadIdx.x, g = t >> 5, lane = t & 31, bh = blockIdx.x, b = bh / a.H;
  const Parts ps(a, b, bh);
  float m = -INFINITY;
  for (int x = t; x < ps.n2; x += NT) m = fmaxf(m, ps.at(x)[0]);
  m = wave_max(m);
  if (lane == 0) red[g] = m;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < NG; ++x) m = fmaxf(m, red[x]);
  float l = 0.f;
  for (int x = t; x < ps.n2; x += NT) {
    const float* part = ps.at(x);
    const float w = part[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(part[0] - m);
    wts[x] = w;
    l += w * part[1];
  }
  l = wave_sum(l);
  if (lane == 0) red[NG + g] = l;  // (both halves of a wave have its sum)
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int x = 0; x < NG; x += 2) l += red[NG + x];
  f4v o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int x = g; x < ps.n2; x += NG) {
    const f4v acc = *(const f4v*)(ps.at(x) + 4 + 4 * lane);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(wts[x], acc[e], o[e]);
  }
  f4v P[NR];
  if (a.P_vo) {
    const float* p0 = a.P_vo + ((int64_t)(bh % a.H / (a.H / a.Hkv)) * kD + NR * g) * kD + 4 * lane;
#pragma unroll
    for (int i = 0; i < NR; ++i) P[i] = *(const f4v*)(p0 + i * kD);
  }
  sums[g][lane] = o;
  __syncthreads();
  if (t < kD) {
    const float* s = (const float*)sums + t;
    float mine = 0.f;
#pragma unroll
    for (int x = 0; x < NG; x += 2) mine += s[x * kD] + s[(x + 1) * kD];
    mine *= l == 0.f ? 0.f : 1.f / l;
    if (!a.P_vo) ((T*)a.out)[(int64_t)bh * kD + t] = (T)mine;
    oh[t] = mine;
  }
  if (!a.P_vo) return;
  __syncthreads();
  const f4v o4 = *(const f4v*)(oh + 4 * lane);
#pragma unroll
  for (int i = 0; i < NR; ++i)
    turn[NR * g + i][lane] =
        fmaf(P[i].w, o4.w, fmaf(P[i].z, o4.z, fmaf(P[i].y, o4.y, P[i].x * o4.x)));
  __syncthreads();
  if (t >= kD) return;
  float r[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 32; ++i) r[i & 3] += turn[t][i];
  ((T*)a.out)[(int64_t)bh * kD + t] = (T)((r[0] + r[1]) + (r[2] + r[3]));
}

// Many rows: half a wave per row, a lane 4 dims; 32 parts' weights at a time are the lanes'.
// Bound by the parts' bytes: 32768 rows of 2 parts 12 us, 4.2 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void join_rows_kernel(JoinLaunch a) {
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= (int64_t)a.B * a.H * a.n) return;
  const int i = (int)(row % a.n), b = (int)(row / a.n / a.H);
  if (i >= a.rows[b]) return;
  const Parts ps(a, b, row);
  float m = -INFINITY;
  for (int x = lane; x < ps.total; x += 32) m = fmaxf(m, ps.m_of(x));
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 32));
  float l = 0.f;
  f4v o = {0.f, 0.f, 0.f, 0.f};
  for (int x0 = 0; x0 < ps.total; x0 += 32) {
    float w = 0.f;
    if (x0 + lane < ps.total) {
      const float mx = ps.m_of(x0 + lane);
      w = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx - m);
      l += w * (x0 + lane < ps.n2 ? ps.at(x0 + lane)[1] : 1.f);
    }
    const int count = min(32, ps.n2 - x0);
#pragma unroll 4
    for (int x = 0; x < count; ++x) {
      const f4v acc = *(const f4v*)(ps.at(x0 + x) + 4 + 4 * lane);
      const float wx = __shfl(w, x, 32);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(wx, acc[e], o[e]);
    }
    if (ps.n2 < ps.total && ps.n2 >= x0 && ps.n2 < x0 + 32) {  // the state
      const float wx = __shfl(w, ps.n2 - x0, 32);
      if (wx != 0.f) {  // (the o of a row that has none is not looked at)
        const f4v acc = *(const f4v*)(a.o0 + row * kD + 4 * lane);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(wx, acc[e], o[e]);
      }
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) l += __shfl_xor(l, d, 32);
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] *= inv;
  if (!a.out) {
    *(f4v*)(a.o + row * kD + 4 * lane) = o;
    if (lane == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) / kLog2e;
    return;
  }
  struct alignas(4 * sizeof(T)) {
    T v[4];
  } y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y.v[e] = (T)o[e];
  *(decltype(y)*)((T*)a.out + row * kD + 4 * lane) = y;
}

template <typename T>
static hipError_t launch_join_t(const JoinLaunch& a) {
  const int64_t rows = (int64_t)a.B * a.H * a.n;
  if (a.decode)
    hipLaunchKernelGGL(join_decode_kernel<T>, dim3((unsigned)rows), dim3(kJoinThreads), 0, a.stream,
                       a);
  else
    hipLaunchKernelGGL(join_rows_kernel<T>, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0,
                       a.stream, a);
  return hipGetLastError();
}

hipError_t launch_join(const JoinLaunch& a) {
  return a.dtype == SWAN_F32 ? launch_join_t<float>(a) : launch_join_t<_Float16>(a);
}

}  // namespace swan
