// Attention of many query rows over the pruned pages and the ring of a cache: a page's
// kept components are scattered into a dense tile of attend.h in LDS (its pruned zeros
// beside them), once for all query rows of the workgroup, then multiplied on MFMA.
//
// The rotated queries are float32.  On the binary16 formats each row is brought by a power
// of two to 2^13 .. 2^14 at its largest component and split into two binary16 parts, whose
// products with the keys are both taken: within 2^-23 of the decode kernels' float32 queries,
// a bit less than these.
#include <type_traits>

#include "attend.h"

namespace swan {

// A lane's token in groups of 8 entries of a page: values and indices
template <typename T, int N>
struct Groups {
  using E = typename Fmt<T>::Elem;
  static constexpr int CB = Fmt<T>::kChunkBytes;
  static constexpr int VCH = 8 * Fmt<T>::kValBytes / CB;
  using Chunk = typename std::conditional<CB == 16, u32x4, u32x2>::type;
  Chunk val[N][VCH];
  u32x2 idx[N];

  // group g of a page of n8 groups, as x
  __device__ __forceinline__ void load(int x, const char* page, int n8, int g, int lane) {
#pragma unroll
    for (int c = 0; c < VCH; ++c)
      val[x][c] = *(const Chunk*)(page + (g * VCH + c) * 64 * CB + lane * CB);
    idx[x] = *(const u32x2*)(page + n8 * VCH * 64 * CB + g * 512 + lane * 8);
  }

  // group x into the token's (zeroed) row, whose pieces are turned by `turn` elements
  __device__ __forceinline__ void scatter(int x, SWAN_LDS E* row, int turn) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // (the mask keeps a damaged page's indices inside the row)
      const int d = ((e < 4 ? idx[x].x : idx[x].y) >> (8 * (e & 3))) & 0x7F;
      row[d ^ turn] = value(x, e);
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

// The row of `lane`'s token in a tile, and how its pieces are turned
template <typename E>
__device__ __forceinline__ SWAN_LDS E* token_row(char* tile, int lane) {
  return (SWAN_LDS E*)((SWAN_LDS char*)tile + lane * Rows<E>::kBytes);
}
template <typename E>
__device__ __forceinline__ int token_turn(int lane) {
  return Rows<E>::turn(lane) * (16 / (int)sizeof(E));
}

// The groups of a page of keys and one of values, numbered keys first, go to the W waves
// round robin: up to NU each.
template <typename T, int NU, int W>
struct PageStage {
  using E = typename Fmt<T>::Elem;
  Groups<T, NU> groups;

  // kpage / vpage: NULL for a tile that is no page
  __device__ __forceinline__ void load(const char* kpage, const char* vpage, int nk, int nv,
                                       int wave, int lane) {
#pragma unroll
    for (int x = 0; x < NU; ++x) {
      const int u = wave + W * x;  // uniform
      const bool key = u < nk;
      const char* page = key ? kpage : vpage;
      if (u < nk + nv && page) groups.load(x, page, key ? nk : nv, key ? u : u - nk, lane);
    }
  }

  // into the (zeroed) tiles; token: this lane has one
  __device__ __forceinline__ void scatter(char* kb, char* vb, int nk, int nv, int wave, int lane,
                                          bool token) const {
    SWAN_LDS E* krow = token_row<E>(kb, lane);
    SWAN_LDS E* vrow = token_row<E>(vb, lane);
    const int turn = token_turn<E>(lane);
#pragma unroll
    for (int x = 0; x < NU; ++x) {
      const int u = wave + W * x;
      if (u < nk + nv && token) groups.scatter(x, u < nk ? krow : vrow, turn);
    }
  }
};

// This lane's half of its row's rotated queries, from float32 at qr (zeros unless `live`), and
// what their scores are multiplied by
template <typename E>
__device__ __forceinline__ float row_queries(const float* qr, bool live, int lane,
                                             typename Tile<E>::template Q<true>& q) {
  float c = 1.f;
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
    const float f = split_scale(max_halves(top), c);
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
  return c;
}

// A wave's 32 query rows, and their products with a tile
template <typename E, int W>
struct QueryRows {
  using Tl = Tile<E>;
  int64_t row;
  bool live, busy;  // this lane's row, some row of the wave is one
  float c;
  typename Tl::template Q<true> q;
  RowState<E> rs;

  __device__ __forceinline__ QueryRows(const AttendLaunch& a, const Unit& un, const Tokens& tokens,
                                      int wave, int lane) {
    const uint32_t r = (uint32_t)un.tile * (32 * W) + 32 * wave + (lane & 31);
    const int G = (int)a.by_g.d, toks = a.toks[un.j];
    const int tok = (int)a.by_g.of(r), g = (int)(r - (uint32_t)tok * (uint32_t)G);
    live = tok < toks;
    busy = (int)a.by_g.of(un.tile * (32 * W) + 32 * wave) < toks;
    int b, i;
    tokens.at(a, un.j, live ? tok : 0, b, i);
    row = ((int64_t)b * a.Hq + un.h * G + g) * a.n + i;
    c = row_queries<E>((const float*)a.q + row * kD, live, lane, q);
    rs.clear();
  }
  // one tile, of `count` keys (more: all); kOdd: with infinite values, as in Tile::values
  template <bool kOdd>
  __device__ __forceinline__ void tile(const char* kb, const char* vb, int count, int lane) {
    f16v S[2];
    // (products first, where the other workgroup's wave has exponentials to do)
    if constexpr (W == 4) __builtin_amdgcn_s_setprio(1);
    Tl::template scores<true>(kb, q, lane, S);
    if constexpr (W == 4) __builtin_amdgcn_s_setprio(0);
    if (count < kTileKeys) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (key_of(x, e, lane) >= count) S[x][e] = -INFINITY;
    }
    rs.raise(tile_max(S) * c);
    rs.l += Tl::template values<false, kOdd>(vb, S, c, rs.safe_ref(), lane, rs.O, kb, q, S);
  }
};

// Grid as in attend_dense_kernel.  A group's keys are its pages, then tiles of its ring
// (in slot order: the sum has none).
//
// W = 4: two workgroups of 128 rows share a CU, each with two tiles in LDS; a tile is
// cleared, filled after a barrier while the one before is multiplied, and a second barrier
// ends both.  W = 8, for many rows: one workgroup of 256, so a page is scattered once where
// two did it, and a third tile saves a barrier: t + 2 is cleared and t + 1 filled beside the
// products of t.  The second wave of each SIMD multiplies first and has priority, so that one
// scatters while the other multiplies (measured: without the priority 4 % more).  The ring's
// tiles pass through registers there, as the third is past what dma_tile reaches.
//
// Bound by a wave's chain per tile of products, scattering and exponentials.  Measured under
// the profiler, k = 64 of 128: 4 x 256 rows of 32 heads on 8 over 4 x 8192 keys 266 us (with
// workgroups of 128 rows 10 % more), where MFMA (two parts of q and of p: 64 instructions of
// 32 cycles for 32 rows and 64 keys) is busy in 48 % of the cycles and other vector
// instructions are issued in 32 %; 8 x 100 rows over 16384 shared keys, E4M3 values, 441 us,
// 44 % and 31 %.  Few rows: 32 tokens over 32768 keys 55 us, 1.9 TB/s of pages, MFMA 26 %; 4
// tokens of 32 heads over 4095 keys 20 us, where workgroups start and load for longer than
// they multiply.
template <typename T, int NU, int W>
__global__ __launch_bounds__(64 * W, sizeof(typename Fmt<T>::Elem) == 2 ? 2 : 1) void
attend_pages_kernel(AttendLaunch a) {
  using E = typename Fmt<T>::Elem;
  using R = Rows<E>;
  constexpr int N = W == 8 ? 3 : 2;
  // (one struct, so that the tiles begin at 0: dma_tile reaches the first 64 KiB)
  __shared__ struct alignas(1024) {
    char buf[2 * N][R::kTile];  // keys and values of N tiles
    int odd;                    // some row's sum is no number
  } sh;
  auto& buf = sh.buf;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Tokens tokens(a, lane);
  const Unit un = unit_at(a, blockIdx.x);
  const int j = un.j, h = un.h, L = a.keys[j], cs = a.cseq[j];
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

  const DmaFrom<E> from = dma_from<E>(wave & 3, lane);
  PageStage<T, NU, W> st;
  // stage: the loads of tile t, where it is a page
  auto stage = [&](int t) {
    const bool page = t < t1 && t < np;
    st.load(page ? kpages + t * kbytes : nullptr, page ? vpages + t * vbytes : nullptr, nk, nv, wave,
            lane);
  };
  // clear: zeros where tile t is a page, the ring's rows (true: to be waited for) where not
  auto clear = [&](int t, int at) {
    char* kb = buf[at];
    char* vb = buf[N + at];
    if (t >= t1) return false;
    if (t < np) {
      const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int x = 0; x < R::kTile / (1024 * W); ++x) {
        ((u32x4*)kb)[tid + 64 * W * x] = zero;
        ((u32x4*)vb)[tid + 64 * W * x] = zero;
      }
      return false;
    }
    const int first = (t - np) * kTileKeys;
    constexpr bool kAsync = sizeof(E) == 2 && W == 4;
    if (W == 4 || wave < 4)
      dma_tile<E, kAsync>(kb, (const E*)a.k_ring + ring + (int64_t)first * kD, nb - first, from,
                          wave & 3);
    if (W == 4 || wave >= 4)
      dma_tile<E, kAsync>(vb, (const E*)a.v_ring + ring + (int64_t)first * kD, nb - first, from,
                          wave & 3);
    return kAsync;
  };
  // scatter: what stage(t) loaded
  auto scatter = [&](int t, int at) {
    st.scatter(buf[at], buf[N + at], nk, nv, wave, lane, t < t1 && t * kPage + lane < S);
  };
  auto count = [&](int t) { return t < np ? S - t * kPage : nb - (t - np) * kTileKeys; };
  stage(t0);

  QueryRows<E, W> rows(a, un, tokens, wave, lane);
  if (tid == 0) sh.odd = 0;
  // all tiles, of which the first is staged
  auto attend = [&](auto odd) {
    constexpr bool kOdd = decltype(odd)::value;
    bool ring_tile = clear(t0, 0);
    if constexpr (W == 8) clear(t0 + 1, 1);
    __syncthreads();
    scatter(t0, 0);
    stage(t0 + 1);
    if (ring_tile) dma_wait();
    __syncthreads();
    if constexpr (W == 4) {
      for (int t = t0; t < t1; ++t) {
        const int par = (t - t0) & 1;
        ring_tile = clear(t + 1, par ^ 1);
        __syncthreads();
        scatter(t + 1, par ^ 1);
        stage(t + 2);
        if (rows.busy) rows.template tile<kOdd>(buf[par], buf[N + par], count(t), lane);
        if (ring_tile) dma_wait();
        __syncthreads();
      }
    } else {
      const bool late = wave >= 4;
      if (late) __builtin_amdgcn_s_setprio(1);
      int x0 = 0, x1 = 1, x2 = 2;
      auto prepare = [&](int t) {
        scatter(t + 1, x1);
        stage(t + 2);
        clear(t + 2, x2);
      };
      for (int t = t0; t < t1; ++t) {
        if (!late) prepare(t);
        if (rows.busy) rows.template tile<kOdd>(buf[x0], buf[N + x0], count(t), lane);
        if (late) prepare(t);
        __syncthreads();
        const int x = x0;
        x0 = x1;
        x1 = x2;
        x2 = x;
      }
    }
  };
  attend(std::false_type());
  if constexpr (sizeof(E) == 2) {
    // An infinite value's products with the parts of p may have made NaNs: once more, with
    // care.  (The barrier is also behind the tiles' last reads.)
    if (rows.live && rows.rs.odd()) sh.odd = 1;
    __syncthreads();
    if (sh.odd) {
      rows.rs.clear();
      stage(t0);
      attend(std::true_type());
    }
  }
  write_partial(a, rows.rs, rows.row, un.split, rows.live, lane);
}

template <typename T>
static hipError_t launch_pages_t(const AttendLaunch& a) {
  // registers for the groups that a wave has in flight: those of up to 128 components in both
  // roles, or of 256 (4 tokens of 32 heads over 4095 keys, k = 48: 35.7 us with room for 128
  // components, 39.3 for 256)
  int most = 0;
  for (int j = 0; j < a.groups; ++j) {
    const int n = kpad_of(a.kact[0][j]) / 8 + kpad_of(a.kact[1][j]) / 8;
    most = n > most ? n : most;
  }
  const dim3 grid(a.units), four(256), eight(512);
  if (a.tile_rows > kTileRows) {
    if constexpr (sizeof(typename Fmt<T>::Elem) == 2) {
      if (most <= 16)
        hipLaunchKernelGGL((attend_pages_kernel<T, 2, 8>), grid, eight, 0, a.stream, a);
      else
        hipLaunchKernelGGL((attend_pages_kernel<T, 4, 8>), grid, eight, 0, a.stream, a);
    }
  } else if (most <= 16) {
    hipLaunchKernelGGL((attend_pages_kernel<T, 4, 4>), grid, four, 0, a.stream, a);
  } else {
    hipLaunchKernelGGL((attend_pages_kernel<T, 8, 4>), grid, four, 0, a.stream, a);
  }
  return hipGetLastError();
}

hipError_t launch_attend_pages(const AttendLaunch& a) {
  if (a.dtype == SWAN_F32) return launch_pages_t<float>(a);
  if (a.dtype == SWAN_F16_E4M3) return launch_pages_t<E4M3V>(a);
  return launch_pages_t<_Float16>(a);
}

}  // namespace swan
