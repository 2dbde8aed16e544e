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

// The least / largest v of a wave
template <bool kMax>
__device__ __forceinline__ int wave_pick(int v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const int o = __shfl_xor(v, d, 64);
    v = kMax ? max(v, o) : min(v, o);
  }
  return __builtin_amdgcn_readfirstlane(v);
}

// With a sliding window: the tiles of a source that some row of a row tile sees.
struct Seen {
  int skip, sink_tiles, nt;  // page tiles before the window; of these with first keys; tiles
  // tok_a .. tok_b: the row tile's tokens.  L tokens are cached, in np pages (S of them) and
  // ring tiles.
  __device__ __forceinline__ void find(const AttendLaunch& a, const Tokens& tokens, int j, int tok_a,
                                  int tok_b, int L, int S, int np, int ring_tiles, int lane) {
    // lane l has list entry l: the first key of its first row in the tile, and its first keys
    const int next = __shfl_down(tokens.tok0, 1, 64);  // (by every lane: each is read from)
    const int end = lane + 1 >= a.first[j + 1] ? a.toks[j] : next;
    const bool mine = lane >= a.first[j] && lane < a.first[j + 1] && tokens.tok0 <= tok_b &&
                      end > tok_a;
    const int lo = wave_pick<false>(mine ? a.lo[lane] + max(0, tok_a - tokens.tok0) : INT32_MAX);
    const int sink = wave_pick<true>(mine ? (int)a.sink[lane] : 0);
    skip = lo >= S ? np : max(0, lo) / kTileKeys;
    sink_tiles = min((min(sink, S) + kTileKeys - 1) / kTileKeys, skip);
    nt = np - skip + sink_tiles + (lo < L || sink > S ? ring_tiles : 0);
  }
  // the page or ring tile that the t-th of these is
  __device__ __forceinline__ int tile(int t) const { return t < sink_tiles ? t : t - sink_tiles + skip; }
};

// The tokens of a tile: `count` keys (more: all), key `at` being token key0 + at, from at =
// turn on `wrap` less.
struct Span {
  int count, key0, turn, wrap;
  __device__ __forceinline__ int token(int at) const { return key0 + at - (at >= turn ? wrap : 0); }
  __device__ __forceinline__ int least() const { return wrap ? key0 + turn - wrap : key0; }
};

// A wave's 32 query rows, and their products with a tile
template <typename E, int W, bool kWin>
struct QueryRows {
  using Tl = Tile<E>;
  int64_t row;
  bool live, busy;  // this lane's row, some row of the wave is one
  float c;
  typename Tl::template Q<true> q;
  RowState<E> rs;
  int lo, sink;        // with a window: this lane's row sees no key from `sink` to `lo`
  int full, all_sink;  // the largest lo, the least sink of the wave's rows

  __device__ __forceinline__ QueryRows(const AttendLaunch& a, const Unit& un, const Tokens& tokens,
                                      int wave, int lane) {
    const uint32_t r = (uint32_t)un.tile * (32 * W) + 32 * wave + (lane & 31);
    const int G = (int)a.by_g.d, toks = a.toks[un.j];
    const int tok = (int)a.by_g.of(r), g = (int)(r - (uint32_t)tok * (uint32_t)G);
    live = tok < toks;
    busy = (int)a.by_g.of(un.tile * (32 * W) + 32 * wave) < toks;
    int e, b, i;
    tokens.at(a, un.j, live ? tok : 0, e, b, i);
    row = ((int64_t)b * a.Hq + un.h * G + g) * a.n + i;
    c = row_queries<E>((const float*)a.q + row * kD, live, lane, q);
    rs.clear();
    if constexpr (kWin) {
      lo = a.lo[e] + i;
      sink = a.sink[e];
      full = wave_pick<true>(live ? lo : INT32_MIN);
      all_sink = wave_pick<false>(live ? sink : INT32_MAX);
    }
  }
  // scores of a tile
  __device__ __forceinline__ void scores(const char* kb, const Span& sp, int lane, f16v (&S)[2]) {
    // (products first, where the other workgroup's wave has exponentials to do)
    if constexpr (W == 4) __builtin_amdgcn_s_setprio(1);
    Tl::template scores<true>(kb, q, lane, S);
    if constexpr (W == 4) __builtin_amdgcn_s_setprio(0);
    if (sp.count < kTileKeys) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (key_of(x, e, lane) >= sp.count) S[x][e] = -INFINITY;
    }
    if constexpr (kWin) {
      if (sp.least() < full && (sp.wrap || sp.key0 + kTileKeys > all_sink)) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (!sees(sp.token(key_of(x, e, lane)))) S[x][e] = -INFINITY;
      }
    }
    rs.raise(tile_max(S) * c);
  }
  __device__ __forceinline__ bool sees(int token) const { return token >= lo || token < sink; }
  // one tile; kOdd: with infinite values, as in Tile::values
  template <bool kOdd>
  __device__ __forceinline__ void tile(const char* kb, const char* vb, const Span& sp, int lane) {
    f16v S[2];
    scores(kb, sp, lane, S);
    rs.l += Tl::template values<false, kOdd>(vb, S, c, rs.safe_ref(), lane, rs.O, kb, q, S);
  }
  // one tile without the values that are no numbers of the tokens odd; those: value(key, dim)
  template <typename V>
  __device__ __forceinline__ void apart(const char* kb, const char* vb, const Span& sp,
                                        uint64_t odd, int lane, V value) {
    f16v S[2], P[2];
    scores(kb, sp, lane, S);
    const float ref = rs.safe_ref();
    rs.l += Tl::template values<false, false>(vb, S, c, ref, lane, rs.O, kb, q, P);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int e = 0; e < 16; ++e) P[x][e] = __builtin_amdgcn_exp2f(fmaf(S[x][e], c, -ref));
    add_nonfinite(
        odd, value, [&](int key) { return key < sp.count && sees(sp.token(key)); }, P, lane, rs.O);
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
//
// kWin: with a sliding window, over the tiles that some row of the row tile sees (Seen), masked
// where a wave's row does not see them whole.  4 x 256 rows of 32 heads on 8 over windows of 4096
// (k = 64) 158 us, 3.6 a tile, as without a window; 8 x 9 rows of 32 heads over windows of 1000
// (E4M3, k = 48) 42 us, where a tile's scatter and barriers take 3 us for however few rows.
template <typename T, int NU, int W, bool kWin>
__global__ __launch_bounds__(64 * W, sizeof(typename Fmt<T>::Elem) == 2 ? 2 : 1) void
attend_pages_kernel(AttendLaunch a) {
  using E = typename Fmt<T>::Elem;
  using R = Rows<E>;
  constexpr int N = W == 8 ? 3 : 2;
  // (one struct, so that the tiles begin at 0: dma_tile reaches the first 64 KiB)
  __shared__ struct alignas(1024) {
    char buf[2 * N][R::kTile];  // keys and values of N tiles
    int odd;                    // some row's sum is no number
    uint64_t odd_keys;          // keys of a tile with values that are no numbers
  } sh;
  auto& buf = sh.buf;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Tokens tokens(a, lane);
  const Unit un = unit_at(a, blockIdx.x);
  const int j = un.j, h = un.h, L = a.keys[j], cs = a.cseq[j];
  const int S = L > a.bb ? L - a.bb : 0, np = pages_for(S), nb = L < a.bb ? L : a.bb;
  const int ring_tiles = (nb + kTileKeys - 1) / kTileKeys;
  Seen seen;
  if constexpr (kWin) {
    const uint32_t r0 = (uint32_t)un.tile * (32 * W);
    seen.find(a, tokens, j, (int)a.by_g.of(r0),
              min(a.toks[j] - 1, (int)a.by_g.of(r0 + 32 * W - 1)), L, S, np, ring_tiles, lane);
  } else {
    seen.nt = np + ring_tiles;
  }
  const int nt = seen.nt;
  // the page or ring tile that the t-th one is
  auto tile_at = [&](int t) { return kWin ? seen.tile(t) : t; };
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
  auto stage = [&](int x) {
    const int t = tile_at(x);
    const bool page = x < t1 && t < np;
    st.load(page ? kpages + t * kbytes : nullptr, page ? vpages + t * vbytes : nullptr, nk, nv, wave,
            lane);
  };
  // clear: zeros where tile t is a page, the ring's rows (true: to be waited for) where not
  auto clear = [&](int x, int at) {
    char* kb = buf[at];
    char* vb = buf[N + at];
    if (x >= t1) return false;
    const int t = tile_at(x);
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
  auto scatter = [&](int x, int at) {
    st.scatter(buf[at], buf[N + at], nk, nv, wave, lane, x < t1 && tile_at(x) * kPage + lane < S);
  };
  QueryRows<E, W, kWin> rows(a, un, tokens, wave, lane);
  // the tokens of the t-th tile; a ring's slot s is token L - L % bb + s, from slot L % bb on
  // bb less (L <= bb: token s)
  const int turn = kWin && L > a.bb && a.bb > 0 ? L % a.bb : 0;
  auto span = [&](int x) {
    const int t = tile_at(x), slot0 = (t - np) * kTileKeys;
    const bool ring = t >= np, wrapped = ring && L > a.bb;
    return Span{ring ? nb - slot0 : S - t * kPage,
                !ring ? t * kPage : wrapped ? L - turn + slot0 : slot0,
                wrapped ? turn - slot0 : kTileKeys, wrapped ? a.bb : 0};
  };
  stage(t0);

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
        if (rows.busy) rows.template tile<kOdd>(buf[par], buf[N + par], span(t), lane);
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
        if (rows.busy) rows.template tile<kOdd>(buf[x0], buf[N + x0], span(t), lane);
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
  if constexpr (kWin) {
    // A value that is no number, of a token that only some rows see, makes NaNs of the other
    // rows (0 times it), and an infinite one may of any row (its products with the parts of
    // p): once more, one tile at a time, with such values out of the tile and added in the
    // rows that see their token.
    if (rows.live && rows.rs.odd()) sh.odd = 1;
    __syncthreads();
    if (sh.odd) {
      rows.rs.clear();
#pragma unroll 1
      for (int t = t0; t < t1; ++t) {
        if (tid == 0) sh.odd_keys = 0;
        stage(t);
        const bool ring_tile = clear(t, 0);
        __syncthreads();
        scatter(t, 0);
        if (ring_tile) dma_wait();
        __syncthreads();
        const u32x4* from = (const u32x4*)buf[N];
        for (int x = tid; x < R::kTile / 16; x += 64 * W) ((u32x4*)buf[N + 1])[x] = from[x];
        __syncthreads();
        const uint64_t mine = take_nonfinite<E, 64 * W>(buf[N], tid);
        if (mine) atomicOr((unsigned long long*)&sh.odd_keys, (unsigned long long)mine);
        __syncthreads();
        const SWAN_LDS char* raw = (const SWAN_LDS char*)(SWAN_LDS char*)buf[N + 1];
        if (rows.busy)
          rows.apart(buf[0], buf[N], span(t), sh.odd_keys, lane, [&](int key, int d) {
            return (float)*(const SWAN_LDS E*)(raw + R::at(key, d));
          });
        __syncthreads();
      }
    }
  } else if constexpr (sizeof(E) == 2) {
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

template <typename T, bool kWin>
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
        hipLaunchKernelGGL((attend_pages_kernel<T, 2, 8, kWin>), grid, eight, 0, a.stream, a);
      else
        hipLaunchKernelGGL((attend_pages_kernel<T, 4, 8, kWin>), grid, eight, 0, a.stream, a);
    }
  } else if (most <= 16) {
    hipLaunchKernelGGL((attend_pages_kernel<T, 4, 4, kWin>), grid, four, 0, a.stream, a);
  } else {
    hipLaunchKernelGGL((attend_pages_kernel<T, 8, 4, kWin>), grid, four, 0, a.stream, a);
  }
  return hipGetLastError();
}

template <bool kWin>
static hipError_t launch_pages_w(const AttendLaunch& a) {
  if (a.dtype == SWAN_F32) return launch_pages_t<float, kWin>(a);
  if (a.dtype == SWAN_F16_E4M3) return launch_pages_t<E4M3V, kWin>(a);
  return launch_pages_t<_Float16, kWin>(a);
}

hipError_t launch_attend_pages(const AttendLaunch& a) {
  return a.window > 0 ? launch_pages_w<true>(a) : launch_pages_w<false>(a);
}

}  // namespace swan
