// Decode attention with a sliding window: the query rotation, the launch of one query head a
// wave (the others: window_decode_gqa.hip), and the choice between them.
#include "window_decode.h"

namespace swan {

// q_hat[b][h] = mult * q[b][h] . P_qk of the head's kv head, the sums as qrot_kernel takes them
// (decode.hip), so that a step's results are those of its two parts
template <typename T>
__global__ __launch_bounds__(512) void window_rotate_kernel(WindowLaunch a) {
  __shared__ float qs[kD];
  __shared__ float part[4][kD];
  const int bh = blockIdx.x, h = bh % a.Hq / (a.Hq / a.Hkv);
  const int j = threadIdx.x & (kD - 1), sq = threadIdx.x / kD;
  const float* P = a.P_qk + (int64_t)h * kD * kD + (int64_t)(32 * sq) * kD + j;
  float m[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) m[i] = P[i * kD];
  if (sq == 0) qs[j] = (float)((const T*)a.q)[(int64_t)bh * kD + j];
  __syncthreads();
  float a0 = 0.f, a1 = 0.f;
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    a0 = fmaf(qs[32 * sq + i], m[i], a0);
    a1 = fmaf(qs[32 * sq + i + 1], m[i + 1], a1);
  }
  part[sq][j] = a0 + a1;
  __syncthreads();
  if (sq == 0)
    a.qhat[(int64_t)bh * kD + j] =
        ((part[0][j] + part[1][j]) + (part[2][j] + part[3][j])) * a.qmult;
}

// Grid: n * Hq * g.n_splits waves over pages, then n * Hq * ring pieces, a wave for 64 rows, last:
// they start beside the last page waves.
//
// The online softmax over pages of decode_mha.h, whose slots outside the window are no tokens,
// two pages' loads in flight.  Bound by memory: 16 sequences of 32 heads over windows of 4096 of
// up to 6000 tokens (k = 48, 444 MB of pages and rings) 73 us, 6.1 TB/s (a streaming read reaches
// 6.8), with the queries' rotation and the join 83.  Groups of odd size, and float32 ones, take it
// too, a wave for each of their heads: 16 sequences of 24 heads on 8 over windows of 4096 (k = 64,
// 204 MB) 113 us, where a page is loaded three times.
template <typename T, int KP8>
__global__ __launch_bounds__(64) void window_kernel(WindowLaunch a, SeqGroup g) {
  constexpr int kRows = kD + 1;  // and the spare row
  __shared__ __attribute__((aligned(16))) float qrep[kRows * kQRep];
  __shared__ __attribute__((aligned(16))) float acc[kRows * kAccCols];
  using E = typename Fmt<T>::Elem;
  const int lane = threadIdx.x, U = g.n * a.Hq;
  int w = blockIdx.x;
  const int b = g.seq[w % U / a.Hq], hq = w % U % a.Hq, h = hq / (a.Hq / a.Hkv);
  w /= U;
  if (w >= g.n_splits) {
    w -= g.n_splits;
    if (64 * w >= min(a.len[b], a.bb)) return;
    const float* qh = a.qhat + ((int64_t)b * a.Hq + hq) * kD;
    qrep[lane] = qh[lane];
    qrep[lane + 64] = qh[lane + 64];
    wave_lds_fence();
    ring_wave<E>(a, b, h, hq, w, qrep, acc, lane);
    return;
  }
  const int split = w, ns = a.nsplit[b];
  if (split >= ns) return;
  const WindowPages list(a.len[b], a.bb, a.lo[b], a.sink[b]);
  const int x0 = split_begin(split, ns, list.count, true);
  const int x1 = split_begin(split + 1, ns, list.count, true);
  UnitPages u;
  u.kbytes = page_bytes_of(Fmt<T>::kValBytes, a.kact[0][b]);
  u.vbytes = page_bytes_of(Fmt<T>::kValBytes, a.kact[1][b]);
  u.nk8 = kpad_of(a.kact[0][b]) / 8;
  u.nv8 = kpad_of(a.kact[1][b]) / 8;
  u.kbase = (const char*)a.k_pages + a.off[0][b] + (int64_t)h * a.npc * u.kbytes;
  u.vbase = (const char*)a.v_pages + a.off[1][b] + (int64_t)h * a.npc * u.vbytes;
  PageRegs<T, KP8> ka, va;
  // (past the split's last page: the resident spare arrays)
  auto load = [&](PageRegs<T, KP8>& k, PageRegs<T, KP8>& v, int x) {
    const bool in = x < x1;
    const int64_t p = list.page(in ? x : x1 - 1);
    load_page<T, KP8>(k, u.kbase + p * u.kbytes, lane, in ? u.nk8 : 0);
    load_page<T, KP8>(v, u.vbase + p * u.vbytes, lane, in ? u.nv8 : 0);
  };
  load(ka, va, x0);
  const float* qh = a.qhat + ((int64_t)b * a.Hq + hq) * kD;
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    const int r = lane + 64 * hh;
    const float v = qh[r];
    float4* row = (float4*)(qrep + r * kQRep);
    row[0] = make_float4(v, v, v, v);
    row[1] = make_float4(v, v, v, v);
  }
  if (lane < 2) ((float4*)(qrep + kSpareRow * kQRep))[lane] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int c = 0; c < kAccCols / 2; ++c)
    ((float4*)acc)[c * 64 + lane] = make_float4(0.f, 0.f, 0.f, 0.f);
  wave_lds_fence();
  const float* qrep_l = qrep + (lane & (kQRep - 1));
  float* acc_l = acc + lane;
  SoftmaxState st{0.f, 0.f, true};
  auto process = [&](const PageRegs<T, KP8>& k, const PageRegs<T, KP8>& v, int x) {
    process_page<T, KP8>(k, v, seen_slot(a, b, list, list.page(x), lane), qrep_l, acc_l, acc, lane,
                         st);
  };
  if constexpr (two_page_sets<T, KP8>()) {
    PageRegs<T, KP8> kb, vb;
    for (int x = x0; x < x1; x += 2) {
      load(kb, vb, x + 1);
      process(ka, va, x);
      load(ka, va, x + 2);
      if (x + 1 < x1) process(kb, vb, x + 1);
    }
  } else {
    for (int x = x0; x < x1; ++x) {
      if (x > x0) load(ka, va, x);
      process(ka, va, x);
    }
  }
  float* part = a.part + (((int64_t)b * a.Hq + hq) * a.slots + split) * kPartFloats;
  const float l = wave_sum(st.l);
  wave_lds_fence();
  reduce_acc(acc, lane, part);
  if (lane == 0) {
    part[0] = st.m;
    part[1] = l;
  }
}

template <typename T, int KP8>
static hipError_t launch_window_k(const WindowLaunch& a, const SeqGroup& g) {
  const dim3 grid(g.n * a.Hq * (g.n_splits + pages_for(a.bb)));
  hipLaunchKernelGGL((window_kernel<T, KP8>), grid, dim3(64), 0, a.stream, a, g);
  return hipGetLastError();
}

template <typename T>
static hipError_t launch_window_t(const WindowLaunch& a) {
  using E = typename Fmt<T>::Elem;
  hipError_t e = hipSuccess;
  if (!a.qhat_ready && !a.rotate_here) {
    hipLaunchKernelGGL(window_rotate_kernel<E>, dim3(a.B * a.Hq), dim3(512), 0, a.stream, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  for (int tier = 16; tier >= 2; tier -= 2) {  // one launch per tier among the sequences
    SeqGroup g;
    g.n = g.n_splits = 0;
    for (int b = 0; b < a.B; ++b) {
      const int k = a.kact[0][b] > a.kact[1][b] ? a.kact[0][b] : a.kact[1][b];
      if (a.len[b] == 0 || window_tier(kpad_of(k) / 8) != tier) continue;
      g.seq[g.n++] = b;
      g.n_splits = a.nsplit[b] > g.n_splits ? a.nsplit[b] : g.n_splits;
    }
    if (g.n == 0) continue;
    if (decode_heads_per_wave(a.dtype, a.Hq, a.Hkv) > 1) {
      e = launch_window_gqa(a, g, tier);
    } else {
      switch (tier) {
#define SWAN_TIER(n)                   \
  case n:                              \
    e = launch_window_k<T, n>(a, g);   \
    break;
        SWAN_TIER(2) SWAN_TIER(4) SWAN_TIER(6) SWAN_TIER(8) SWAN_TIER(10) SWAN_TIER(12) SWAN_TIER(16)
#undef SWAN_TIER
        default:
          e = hipErrorInvalidValue;
      }
    }
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_window(const WindowLaunch& a) {
  if (a.dtype == SWAN_F16) return launch_window_t<_Float16>(a);
  if (a.dtype == SWAN_F16_E4M3) return launch_window_t<E4M3V>(a);
  return launch_window_t<float>(a);
}

}  // namespace swan
