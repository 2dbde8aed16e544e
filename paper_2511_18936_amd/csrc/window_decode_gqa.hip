// Decode attention with a sliding window for grouped-query heads (binary16 storage): the
// score wave and the value wave of decode_gqa.h over the pages that hold visible tokens.
#include "decode_gqa.h"
#include "window_decode.h"

namespace swan {

// The rotated queries of N heads from hq0 on of kv head h, dim threadIdx.x of them in `out`, by
// the 128 threads of a block; the sums as window_rotate_kernel takes them, which this replaces:
// 32 lanes have a quarter of P_qk's rows, 16 bytes of each (one sequence of 8 kv heads 13.9 us a
// call; with a dim of all rows a thread, for four times the loads and reads of LDS, 15.1).  q: [5 N][kD] of scratch.
template <int N>
__device__ __forceinline__ void rotate_here(const WindowLaunch& a, int b, int h, int hq0, float* q,
                                            float (&out)[N]) {
  constexpr int kLoads = 16;
  const int t = threadIdx.x, sq = t >> 5, d = 4 * (t & 31);
  float* part = q + N * kD;
  const float* P = a.P_qk + (int64_t)h * kD * kD + 32 * sq * kD + d;
  f4 m[kLoads], a0[N], a1[N];
  auto load = [&](int i0) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) m[i] = *(const f4*)(P + (i0 + i) * kD);
  };
  load(0);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    q[j * kD + t] = (float)((const _Float16*)a.q)[((int64_t)b * a.Hq + hq0 + j) * kD + t];
    a0[j] = a1[j] = f4{0.f, 0.f, 0.f, 0.f};
  }
  __syncthreads();
#pragma unroll
  for (int i0 = 0; i0 < 32; i0 += kLoads) {
    if (i0 > 0) load(i0);
#pragma unroll
    for (int i = 0; i < kLoads; i += 2)
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a0[j][e] = fmaf(q[j * kD + 32 * sq + i0 + i], m[i][e], a0[j][e]);
          a1[j][e] = fmaf(q[j * kD + 32 * sq + i0 + i + 1], m[i + 1][e], a1[j][e]);
        }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) *(f4*)(part + (4 * j + sq) * kD + d) = a0[j] + a1[j];
  __syncthreads();
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float* p = part + 4 * j * kD + t;
    out[j] = ((p[0] + p[kD]) + (p[2 * kD] + p[3 * kD])) * a.qmult;
  }
}

// Grid: units * g.n_splits blocks over pages, then units * ring pieces * GH / 2, of a ring wave
// per query head; a unit is GH query heads of one kv head of a sequence.  Two waves a SIMD, as
// LDS allows four blocks a CU (the largest pages: one).
//
// Few sequences are bound by latency: one of 8 kv heads over 1024 tokens (k = 64) 10 us, the
// chain of P_qk, a page or two, and their barriers, and 4 to join.  Many: 32 sequences of up to
// 8000 tokens over 4096 (331 MB of pages and rings) 76-83 us with the queries' rotation and the
// join, 32 of 8000 (407 MB) 84, of 8-bit values (277 MB) 70: 4.0-4.9 TB/s, where the call without a
// window moves 5.9-6.1 with the same work a page.  What differs are short splits, each filling its
// query replicas, the ring's workgroups, which hold LDS for pages, and two more launches; their
// shares are not measured.
//
// kRotate: the blocks rotate their queries themselves (swan_long_api.hip has the rule).
template <typename T, int KP8, int GH, bool kRotate>
__global__ __launch_bounds__(128, KP8 <= 10 ? 2 : 1) void window_gqa_kernel(WindowLaunch a, SeqGroup g) {
  constexpr int R = qrep_replicas<GH>();
  __shared__ __attribute__((aligned(16))) GqaLds<GH, kD + 1> sh;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // 0: scores, 1: values
  const int lane = threadIdx.x & 63;
  const int HC = a.Hq / a.Hkv / GH, units = g.n * a.Hkv * HC;
  const int ui = blockIdx.x % units, x = blockIdx.x / units;
  const int b = g.seq[ui / (a.Hkv * HC)], h = ui / HC % a.Hkv;
  const int hq0 = (h * HC + ui % HC) * GH;
  if (x >= g.n_splits) {
    const int piece = (x - g.n_splits) / (GH / 2), j = (x - g.n_splits) % (GH / 2) * 2 + wave;
    if (64 * piece >= min(a.len[b], a.bb)) return;
    float* q = sh.qrep + wave * kD;
    if constexpr (kRotate) {
      static_assert(sizeof(sh.vt) >= 10 * kD * sizeof(float), "scratch");
      float both[2];
      rotate_here<2>(a, b, h, hq0 + j - wave, (float*)sh.vt, both);
      sh.qrep[threadIdx.x] = both[0];
      sh.qrep[kD + threadIdx.x] = both[1];
      __syncthreads();
    } else {
      const float* qh = a.qhat + ((int64_t)b * a.Hq + hq0 + j) * kD;
      q[lane] = qh[lane];
      q[lane + 64] = qh[lane + 64];
      wave_lds_fence();
    }
    ring_wave<_Float16>(a, b, h, hq0 + j, piece, q, (float*)sh.vt + wave * 64, lane);
    return;
  }
  const int split = x, ns = a.nsplit[b];
  if (split >= ns) return;  // uniform over the block
  const WindowPages list(a.len[b], a.bb, a.lo[b], a.sink[b]);
  const int x0 = split_begin(split, ns, list.count, true);
  const int x1 = split_begin(split + 1, ns, list.count, true);
  // the page size and loaded groups of this wave's role
  const int64_t pbytes = page_bytes_of(Fmt<T>::kValBytes, a.kact[wave][b]);
  const int n8 = kpad_of(a.kact[wave][b]) / 8;
  const char* base = (const char*)(wave == 0 ? a.k_pages : a.v_pages) + a.off[wave][b] +
                     (int64_t)h * a.npc * pbytes;
  PageRegs<T, KP8> ra, rb;
  auto load = [&](PageRegs<T, KP8>& r, int x) {  // (past the last: the resident spare arrays)
    const bool in = x < x1;
    load_page<T, KP8>(r, base + list.page(in ? x : x1 - 1) * pbytes, lane, in ? n8 : 0);
  };
  // large pages' registers stay free while the replicas are filled (as in attn_gqa_kernel)
  constexpr bool kEarly = sizeof(PageRegs<T, KP8>) <= 192;
  if constexpr (kEarly) load(ra, x0);
  {  // q_rep[dim][r][head]: thread t writes dim t, all replicas
    const int d = threadIdx.x;
    float q[GH];
    if constexpr (kRotate) {
      static_assert(sizeof(sh.vt) >= 5 * GH * kD * sizeof(float), "scratch");
      rotate_here<GH>(a, b, h, hq0, (float*)sh.vt, q);
    } else {
      const float* qh = a.qhat + ((int64_t)b * a.Hq + hq0) * kD;
#pragma unroll
      for (int j = 0; j < GH; ++j) q[j] = qh[j * kD + d];
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < GH; ++j) sh.qrep[(d * R + r) * GH + j] = q[j];
    if (d < R * GH) sh.qrep[kSpareRow * R * GH + d] = 0.f;
  }
  __syncthreads();
  if constexpr (!kEarly) load(ra, x0);
  auto seen = [&](int x) { return seen_slot(a, b, list, list.page(x), lane); };
  float* part = a.part + (((int64_t)b * a.Hq + hq0) * a.slots + split) * kPartFloats;
  const int64_t step = (int64_t)a.slots * kPartFloats;
  if (wave == 0) {
    float m[GH], l[GH];
    bool first = true;
#pragma unroll
    for (int j = 0; j < GH; ++j) m[j] = l[j] = 0.f;
    for (int x = x0; x < x1; x += 2) {
      load(rb, x + 1);
      gqa_scores<T, KP8, GH>(ra, seen(x), sh, (x - x0) & 1, lane, m, l, first);
      __syncthreads();
      load(ra, x + 2);
      if (x + 1 < x1) {
        gqa_scores<T, KP8, GH>(rb, seen(x + 1), sh, (x + 1 - x0) & 1, lane, m, l, first);
        __syncthreads();
      }
    }
#pragma unroll
    for (int j = 0; j < GH; ++j) {
      const float lt = wave_sum(l[j]);
      if (lane == 0) {
        part[j * step] = m[j];
        part[j * step + 1] = lt;
      }
    }
  } else {
    f4 acc[8];
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) acc[nt] = f4{0.f, 0.f, 0.f, 0.f};
    for (int x = x0; x < x1; x += 2) {
      load(rb, x + 1);
      gqa_scatter<T, KP8>(ra, seen(x), sh, lane);
      __syncthreads();
      gqa_mfma<GH, T>(sh, (x - x0) & 1, lane, acc);
      load(ra, x + 2);
      if (x + 1 < x1) {
        gqa_scatter<T, KP8>(rb, seen(x + 1), sh, lane);
        __syncthreads();
        gqa_mfma<GH, T>(sh, (x + 1 - x0) & 1, lane, acc);
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int j = 4 * (lane >> 4) + r;
      if (j < GH) {
#pragma unroll
        for (int nt = 0; nt < 8; ++nt) part[j * step + 4 + 16 * nt + (lane & 15)] = acc[nt][r];
      }
    }
  }
}

template <typename T, int KP8, int GH>
static hipError_t launch_gqa_k(const WindowLaunch& a, const SeqGroup& g) {
  const int units = g.n * a.Hkv * (a.Hq / a.Hkv / GH);
  const dim3 grid(units * (g.n_splits + pages_for(a.bb) * (GH / 2)));
  if constexpr (GH <= kRotateHeads) {
    if (a.rotate_here) {
      hipLaunchKernelGGL((window_gqa_kernel<T, KP8, GH, true>), grid, dim3(128), 0, a.stream, a, g);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((window_gqa_kernel<T, KP8, GH, false>), grid, dim3(128), 0, a.stream, a, g);
  return hipGetLastError();
}

template <typename T, int GH>
static hipError_t launch_gqa_g(const WindowLaunch& a, const SeqGroup& g, int kp8) {
  switch (kp8) {
#define SWAN_TIER(n) \
  case n:            \
    return launch_gqa_k<T, n, GH>(a, g);
    SWAN_TIER(2) SWAN_TIER(4) SWAN_TIER(6) SWAN_TIER(8) SWAN_TIER(10) SWAN_TIER(12) SWAN_TIER(16)
#undef SWAN_TIER
    default:
      return hipErrorInvalidValue;
  }
}

template <typename T>
static hipError_t launch_gqa_t(const WindowLaunch& a, const SeqGroup& g, int kp8) {
  switch (decode_heads_per_wave(a.dtype, a.Hq, a.Hkv)) {
    case 8:
      return launch_gqa_g<T, 8>(a, g, kp8);
    case 4:
      return launch_gqa_g<T, 4>(a, g, kp8);
    case 2:
      return launch_gqa_g<T, 2>(a, g, kp8);
    default:
      return hipErrorInvalidValue;
  }
}

hipError_t launch_window_gqa(const WindowLaunch& a, const SeqGroup& g, int kp8) {
  return a.dtype == SWAN_F16_E4M3 ? launch_gqa_t<E4M3V>(a, g, kp8)
                                  : launch_gqa_t<_Float16>(a, g, kp8);
}

}  // namespace swan
