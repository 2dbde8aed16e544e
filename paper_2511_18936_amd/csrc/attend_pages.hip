// Attention of many query rows over the pruned pages and the ring of a cache: a page's
// kept components are scattered into a dense tile of attend.h in LDS (its pruned zeros
// beside them), once for all query rows of the workgroup, then multiplied on MFMA.
//
// The rotated queries are float32.  On the binary16 formats each row is brought by a power
// of two to 2^13 .. 2^14 at its largest component and split into two binary16 parts, whose
// products with the keys are both taken: 22 bits, as the decode kernels' float32 queries
// against binary16 keys but for the last two.
#include <type_traits>

#include "attend.h"

namespace swan {

// Groups of 8 entries of a page of keys and one of values, numbered keys first, go to the 4
// waves round robin; a lane holds its token's 8 values and indices of each.
template <typename T, int NU>
struct PageStage {
  using E = typename Fmt<T>::Elem;
  static constexpr int CB = Fmt<T>::kChunkBytes;
  static constexpr int VCH = 8 * Fmt<T>::kValBytes / CB;
  using Chunk = typename std::conditional<CB == 16, u32x4, u32x2>::type;
  Chunk val[NU][VCH];
  u32x2 idx[NU];

  // kpage / vpage: NULL for a tile that is no page
  __device__ __forceinline__ void load(const char* kpage, const char* vpage, int nk, int nv,
                                       int wave, int lane) {
#pragma unroll
    for (int x = 0; x < NU; ++x) {
      const int u = wave + 4 * x;  // uniform
      const bool key = u < nk;
      const char* page = key ? kpage : vpage;
      if (u < nk + nv && page) {
        const int g = key ? u : u - nk, n8 = key ? nk : nv;
#pragma unroll
        for (int c = 0; c < VCH; ++c)
          val[x][c] = *(const Chunk*)(page + (g * VCH + c) * 64 * CB + lane * CB);
        idx[x] = *(const u32x2*)(page + n8 * VCH * 64 * CB + g * 512 + lane * 8);
      }
    }
  }

  // into the (zeroed) tiles; ktoken / vtoken: this lane has a token there
  __device__ __forceinline__ void scatter(char* kb, char* vb, int nk, int nv, int wave, int lane,
                                          bool ktoken, bool vtoken) const {
    using R = Rows<E>;
    constexpr int N = 16 / (int)sizeof(E);
    SWAN_LDS E* krow = (SWAN_LDS E*)((SWAN_LDS char*)kb + lane * R::kBytes);
    SWAN_LDS E* vrow = (SWAN_LDS E*)((SWAN_LDS char*)vb + lane * R::kBytes);
    const int turn = R::turn(lane) * N;
#pragma unroll
    for (int x = 0; x < NU; ++x) {
      const int u = wave + 4 * x;
      if (u < nk + nv) {
        SWAN_LDS E* to = u < nk ? krow : vrow;
        if (u < nk ? ktoken : vtoken) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            // (the mask keeps a damaged page's indices inside the row)
            const int d = ((e < 4 ? idx[x].x : idx[x].y) >> (8 * (e & 3))) & 0x7F;
            to[d ^ turn] = value(x, e);
          }
        }
      }
    }
  }

  __device__ __forceinline__ typename Fmt<T>::Elem value(int x, int e) const {
    if constexpr (sizeof(T) == 4) {
      return __uint_as_float(val[x][e >> 2][e & 3]);
    } else if constexpr (Fmt<T>::kValBytes == 1) {
      const uint32_t w = e < 4 ? val[x][0].x : val[x][0].y;
      const h2v two = (e & 2) ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true)
                              : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
      return (e & 1) ? two.y : two.x;
    } else {
      const uint32_t w = val[x][0][e >> 1];
      return __builtin_bit_cast(_Float16, (uint16_t)((e & 1) ? w >> 16 : w & 0xFFFFu));
    }
  }
};

// Grid as in attend_dense_kernel.  A group's keys are its pages, then tiles of its ring
// (in slot order: the sum has none).
template <typename T, int NU>
__global__ __launch_bounds__(256, sizeof(typename Fmt<T>::Elem) == 2 ? 2 : 1) void
attend_pages_kernel(AttendLaunch a) {
  using E = typename Fmt<T>::Elem;
  using Tl = Tile<E>;
  using R = Rows<E>;
  __shared__ __align__(1024) char kbuf[2][R::kTile];
  __shared__ __align__(1024) char vbuf[2][R::kTile];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = (int)a.by_g.d;
  const Unit un = unit_at(a, blockIdx.x);
  const int j = un.j, h = un.h;
  const int toks = a.toks[j], L = a.keys[j], cs = a.cseq[j];
  const uint32_t r = (uint32_t)un.tile * kTileRows + 32 * wave + (lane & 31);
  const int tok = (int)a.by_g.of(r), g = (int)(r - (uint32_t)tok * (uint32_t)G);
  const bool live = tok < toks;
  const bool busy = (int)a.by_g.of(un.tile * kTileRows + 32 * wave) < toks;  // some row is live
  int b = 0, i = 0;
  if (live) token_at(a, j, tok, b, i);
  const int64_t row = ((int64_t)b * a.Hq + h * G + g) * a.n + i;

  const int S = L > a.bb ? L - a.bb : 0, np = pages_for(S), nb = L < a.bb ? L : a.bb;
  const int nt = np + (nb + kTileKeys - 1) / kTileKeys;
  const int t0 = split_first(nt, un.split, un.nsplit);
  const int t1 = split_first(nt, un.split + 1, un.nsplit);
  const int nk = kpad_of(a.kact[0][j]) / 8, nv = kpad_of(a.kact[1][j]) / 8;
  const int64_t kbytes = page_bytes_of(Fmt<T>::kValBytes, 8 * nk);
  const int64_t vbytes = page_bytes_of(Fmt<T>::kValBytes, 8 * nv);
  const char* kpages = (const char*)a.k + a.off[0][j] + (int64_t)h * a.npc * kbytes;
  const char* vpages = (const char*)a.v + a.off[1][j] + (int64_t)h * a.npc * vbytes;
  const int64_t ring = ((int64_t)cs * a.Hkv + h) * a.bb * kD;

  const DmaFrom<E> from = dma_from<E>(wave, lane);
  PageStage<T, NU> st;
  // stage(k, v): the loads of tile k's keys and of tile v's values, where they are pages
  auto stage = [&](int k, int v) {
    st.load(k < t1 && k < np ? kpages + k * kbytes : nullptr,
            v < t1 && v < np ? vpages + v * vbytes : nullptr, nk, nv, wave, lane);
  };
  // clear(k, v): zeros where those tiles are pages, the ring's rows where they are not
  auto clear = [&](int k, int v) {
    const u32x4 zero = {0u, 0u, 0u, 0u};
    bool ring_tile = false;
    if (k < t1 && k < np) {
#pragma unroll
      for (int x = 0; x < R::kTile / 4096; ++x)
        ((u32x4*)kbuf[(k - t0) & 1])[tid + 256 * x] = zero;
    } else if (k < t1) {
      dma_tile(kbuf[(k - t0) & 1], (const E*)a.k_ring + ring + (int64_t)(k - np) * kTileKeys * kD,
               nb - (k - np) * kTileKeys, from, wave);
      ring_tile = true;
    }
    if (v < t1 && v < np) {
#pragma unroll
      for (int x = 0; x < R::kTile / 4096; ++x)
        ((u32x4*)vbuf[(v - t0) & 1])[tid + 256 * x] = zero;
    } else if (v < t1) {
      dma_tile(vbuf[(v - t0) & 1], (const E*)a.v_ring + ring + (int64_t)(v - np) * kTileKeys * kD,
               nb - (v - np) * kTileKeys, from, wave);
      ring_tile = true;
    }
    return ring_tile;
  };
  // scatter(k, v): what stage(k, v) loaded
  auto scatter = [&](int k, int v) {
    st.scatter(kbuf[(k - t0) & 1], vbuf[(v - t0) & 1], nk, nv, wave, lane,
               k < t1 && k * kPage + lane < S, v < t1 && v * kPage + lane < S);
  };
  stage(t0, t0);

  // the row's queries
  typename Tl::template Q<true> q;
  float c = 1.f;
  {
    const float* qr = (const float*)a.q + row * kD;
    if constexpr (sizeof(E) == 4) {
#pragma unroll
      for (int s = 0; s < 16; ++s)
        q.hi[s] = live ? *(const f4v*)(qr + 8 * s + 4 * (lane >> 5)) : f4v{0.f, 0.f, 0.f, 0.f};
    } else {
      float x[64], top = 0.f;
#pragma unroll
      for (int s = 0; s < 16; ++s) {
        const f4v v = live ? *(const f4v*)(qr + 16 * (s >> 1) + 8 * (lane >> 5) + 4 * (s & 1))
                           : f4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[4 * s + e] = v[e];
          top = fmaxf(top, fabsf(v[e]));
        }
      }
      top = max_halves(top);
      // 2^(13 - exponent); a row of zeros, infinities or NaNs as it is
      const int ex = (int)((__float_as_uint(top) >> 23) & 0xFF) - 127;
      const int up = top > 0.f && ex < 128 ? 13 - (ex < -100 ? -100 : ex) : 0;
      const float f = __builtin_ldexpf(1.f, up);
      c = __builtin_ldexpf(1.f, -up);
#pragma unroll
      for (int s = 0; s < 8; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = x[8 * s + e] * f;
          const _Float16 hi = (_Float16)y;
          q.hi[s][e] = hi;
          q.lo[s][e] = (_Float16)(y - (float)hi);
        }
    }
  }
  RowState rs;
  rs.clear();
  f16v Sc[2];
  bool ring_tile = clear(t0, t0);
  __syncthreads();
  scatter(t0, t0);
  stage(t0 + 1, t0 + 1);
  if (ring_tile) dma_wait();
  __syncthreads();
  for (int t = t0; t < t1; ++t) {
    const int par = (t - t0) & 1;
    ring_tile = clear(t + 1, t + 1);
    __syncthreads();
    scatter(t + 1, t + 1);
    stage(t + 2, t + 2);
    if (busy) {
      // (products first, where the other workgroup's wave has exponentials to do)
      __builtin_amdgcn_s_setprio(1);
      Tl::template scores<true>(kbuf[par], q, lane, Sc);
      __builtin_amdgcn_s_setprio(0);
      const int count = t < np ? S - t * kPage : nb - (t - np) * kTileKeys;
      if (count < kTileKeys) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (key_of(x, e, lane) >= count) Sc[x][e] = -INFINITY;
      }
      rs.raise(tile_max(Sc) * c);
      rs.l += Tl::template values<false>(vbuf[par], Sc, c, rs.safe_ref(), lane, rs.O, kbuf[0], q,
                                         Sc);
    }
    if (ring_tile) dma_wait();
    __syncthreads();
  }
  write_partial(a, rs, row, un.split, live, lane);
}

template <typename T>
static hipError_t launch_pages_t(const AttendLaunch& a) {
  // registers for 4 or 8 groups a wave in flight: up to 128 components of both roles, or 256
  int most = 0;
  for (int j = 0; j < a.groups; ++j) {
    const int n = kpad_of(a.kact[0][j]) / 8 + kpad_of(a.kact[1][j]) / 8;
    most = n > most ? n : most;
  }
  if (most <= 16)
    hipLaunchKernelGGL((attend_pages_kernel<T, 4>), dim3(a.units), dim3(256), 0, a.stream, a);
  else
    hipLaunchKernelGGL((attend_pages_kernel<T, 8>), dim3(a.units), dim3(256), 0, a.stream, a);
  return hipGetLastError();
}

hipError_t launch_attend_pages(const AttendLaunch& a) {
  if (a.dtype == SWAN_F32) return launch_pages_t<float>(a);
  if (a.dtype == SWAN_F16_E4M3) return launch_pages_t<E4M3V>(a);
  return launch_pages_t<_Float16>(a);
}

}  // namespace swan
