// Attention of the rows of a prompt (causal), or of rows over another sequence's keys and
// values: dense tiles of attend.h, continued from a state where one is given.
#include "attend.h"

namespace swan {

// Values of a tile that are no numbers leave it (0 times them would be NaN in the rows that
// must not see their key): zeros in their place, and the keys of this thread's that had one.
template <typename T>
__device__ __forceinline__ uint64_t take_nonfinite(char* vb, int tid) {
  using R = Rows<T>;
  uint64_t keys = 0;
#pragma unroll 1
  for (int piece = tid; piece < R::kTile / 16; piece += 256) {
    u32x4 x = *(u32x4*)(vb + 16 * piece);
    bool odd = false;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (sizeof(T) == 4) {
        const bool a = (x[w] & 0x7F800000u) == 0x7F800000u;
        x[w] = a ? 0u : x[w];
        odd |= a;
      } else {
        const bool a = (x[w] & 0x7C00u) == 0x7C00u, b = (x[w] & 0x7C000000u) == 0x7C000000u;
        x[w] &= (a ? 0xFFFF0000u : ~0u) & (b ? 0xFFFFu : ~0u);
        odd |= a || b;
      }
    }
    if (odd) {
      *(u32x4*)(vb + 16 * piece) = x;
      keys |= 1ull << (piece / R::kPieces);
    }
  }
  return keys;
}

// O += p v for the values that take_nonfinite() took out of the tile, key by key, in the
// rows that see the key.  Rare: the loops are for size, not for speed.
template <typename T>
__device__ __forceinline__ void add_nonfinite(uint64_t keys, const T* vp, int key0, int limit,
                                              const f16v (&P)[2], int lane, f16v (&O)[4]) {
#pragma unroll 1
  while (keys) {
    const int key = __builtin_ctzll(keys);
    keys &= keys - 1;
    float mine = 0.f;  // p of key 8 (key / 8) + 4 (lane / 32) + key % 4
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (key_of(t, i, 0) == (key & ~4)) mine = P[t][i];
    const f4v both = both_halves(mine);
    const float p = key & 4 ? both.y : both.x;
    const T* row = vp + (int64_t)(key0 + key) * kD + 4 * (lane >> 5);
    if (key0 + key < limit) {
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float v = (float)row[32 * d + 8 * (i >> 2) + (i & 3)];
          if (!(v - v == 0.f)) O[d][i] += p * v;
        }
    }
  }
}

// Grid: a.units workgroups of 4 waves (unit_at), a group's last row tiles, of a causal prompt
// the longest, first.
//
// Two workgroups of 64 KiB of LDS share a CU.  Tiles go to LDS without passing registers, keys
// one tile ahead of values, and the scores of a tile are taken in steps between the
// exponentials of the one before.  Long prompts are bound by what a SIMD's two waves issue: of
// the cycles MFMA is busy in 46 %, other vector instructions are issued in 38 %, seldom both.
// Measured, binary16: 32 query heads on 8, 4096 causal rows 213-235 us by machine, 880-970
// TFLOP/s of products done, p's second part among them (a large matrix product reaches 1200); 8
// prompts of up to 1009 rows, 32 heads 69-77 us (short rows of tiles, 6 us to start and end
// each).  Few rows split the keys until the GPU is full and are bound by memory: single tokens
// of 16 heads over up to 1500 keys of 16 sequences 24 us, 4.3 TB/s, and 4 us to join; the
// waves without a row leave LDS to the others (28.6 us with the join; 34.7 if they multiply
// too).  Float32 (no double use of a CU: its tiles take 128 KiB): 2 x 333 rows, 8 heads on 2,
// 23 us and 6 to join, the latency of few workgroups.
//
// The last tile stands behind the loop, without scores to take ahead: as a condition inside
// the loop it made registers spill.
template <typename T>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void attend_dense_kernel(AttendLaunch a) {
  using Tl = Tile<T>;
  using R = Rows<T>;
  // (one struct, so that the tiles begin at 0: dma_tile reaches the first 64 KiB)
  __shared__ struct alignas(1024) {
    char k[2][R::kTile], v[2][R::kTile];
    uint64_t odd_keys;  // keys of a tile with values that are no numbers
  } sh;
  auto &kbuf = sh.k, &vbuf = sh.v;
  uint64_t& odd_keys = sh.odd_keys;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = (int)a.by_g.d;
  const Unit un = unit_at(a, blockIdx.x);
  const int h = un.h, toks = a.toks[un.j], keys = a.keys[un.j], b = a.cseq[un.j];
  const uint32_t rows = (uint32_t)toks * (uint32_t)G;  // below 2^31
  const uint32_t row0 = ((rows + kTileRows - 1) / kTileRows - 1 - un.tile) * kTileRows;

  // this lane's row
  const uint32_t r = row0 + 32 * wave + (lane & 31);
  const int tok = (int)a.by_g.of(r), g = (int)(r - (uint32_t)tok * (uint32_t)G);
  const bool live = tok < toks;
  const bool busy = (int)a.by_g.of(row0 + 32 * wave) < toks;  // some row of the wave is one
  const int64_t row = ((int64_t)b * a.Hq + h * G + g) * a.n + tok;
  // Causal: row i sees the keys up to i + shift.  limit: those this lane's row sees; all_see,
  // block_all: that every row of the wave, of the workgroup sees; seen: that some row does.
  const int shift = keys - toks;
  auto sees = [&](int tok) { return a.causal ? min(keys, max(0, tok + shift + 1)) : keys; };
  const int limit = live ? sees(tok) : 0;
  const int all_see = sees((int)a.by_g.of(row0 + 32 * wave));
  const int block_all = sees((int)a.by_g.of(row0));
  const int seen = sees(min(toks - 1, (int)a.by_g.of(row0 + kTileRows - 1)));
  const int nt = (seen + kTileKeys - 1) / kTileKeys;
  const int t0 = split_first(nt, un.split, un.nsplit);
  const int t1 = split_first(nt, un.split + 1, un.nsplit);

  const int64_t kv0 = ((int64_t)b * a.Hkv + h) * a.m * kD;
  const T* kp = (const T*)a.k + kv0;
  const T* vp = (const T*)a.v + kv0;
  const DmaFrom<T> from = dma_from<T>(wave, lane);
  // tile t is tile t - t0 of its buffers' turns; past the last, nothing
  auto load_k = [&](int t) {
    if (t < t1)
      dma_tile(kbuf[(t - t0) & 1], kp + (int64_t)t * kTileKeys * kD, keys - t * kTileKeys, from,
               wave);
  };
  auto load_v = [&](int t) {
    if (t < t1)
      dma_tile(vbuf[(t - t0) & 1], vp + (int64_t)t * kTileKeys * kD, keys - t * kTileKeys, from,
               wave);
  };
  load_k(t0);
  load_v(t0);
  load_k(t0 + 1);

  typename Tl::template Q<false> q;
  {
    const T* qr = (const T*)a.q + row * kD;
    constexpr int N = sizeof(q.hi) / 16, E = 16 / (int)sizeof(T);
    u32x4* to = (u32x4*)&q;
#pragma unroll
    for (int s = 0; s < N; ++s)
      to[s] = live ? *(const u32x4*)(qr + 2 * E * s + E * (lane >> 5)) : u32x4{0u, 0u, 0u, 0u};
  }
  RowState<T> rs;
  // A tile's scores are taken during the exponentials of the one before, so its keys are in
  // LDS one tile ahead of its values; a buffer is loaded again after the barrier behind its
  // last reads.
  //
  auto begin = [&]() {  // the state to continue from, or none
#pragma clang fp contract(off)
    rs.clear();
    if (!a.o0 || !live || a.part) return;
    const float lse = a.lse0[row] * kLog2e;
    if (lse == -INFINITY) return;
    rs.ref = lse - Lag<T>::kHead;
    const float w = __builtin_amdgcn_exp2f(lse - rs.ref);  // (2^Lag::kHead but for a rounded ref)
    rs.l = lane < 32 ? w : 0.f;
    const float* o = a.o0 + row * kD + 4 * (lane >> 5);
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f4v x = *(const f4v*)(o + 32 * d + 8 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) rs.O[d][4 * i + e] = x[e] * w;
      }
  };
  auto mask = [&](f16v (&S)[2], int key0) {
    if (key0 + kTileKeys > all_see) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (key0 + key_of(x, i, lane) >= limit) S[x][i] = -INFINITY;
    }
  };
  begin();
  f16v S[2], next[2];
  dma_wait();
  __syncthreads();
  if (busy && t0 < t1) Tl::template scores<false>(kbuf[0], q, lane, S);
  __syncthreads();
  for (int t = t0; t < t1 - 1; ++t) {
    const int par = (t - t0) & 1;
    load_k(t + 2);
    load_v(t + 1);
    if (busy) {
      mask(S, t * kTileKeys);
      float c = a.qmult;
      const float ref = take_scores(rs, S, c);
      rs.l += Tl::template values<true, false>(vbuf[par], S, c, ref, lane, rs.O, kbuf[par ^ 1], q,
                                               next);
      S[0] = next[0];
      S[1] = next[1];
    }
    dma_wait();
    __syncthreads();
  }
  if (busy && t0 < t1) {
    mask(S, (t1 - 1) * kTileKeys);
    float c = a.qmult;
    const float ref = take_scores(rs, S, c);
    rs.l += Tl::template values<false, false>(vbuf[(t1 - 1 - t0) & 1], S, c, ref, lane, rs.O,
                                              kbuf[0], q, next);
  }
  // Values that are no numbers, of keys that only some rows see, make NaNs of the other rows
  // (0 times them), and infinite ones of any key in binary16, where the parts of p may be 0 or
  // of both signs.  Where a row's result is no number the workgroup starts again, takes such
  // values out of the tiles and adds them in the rows that see their key: slowly, but it
  // costs the other calls one look at the result.
  if (sizeof(T) == 2 || block_all < seen) {
    if (__syncthreads_or(live && rs.odd())) {  // (also: the tiles' last reads are done)
      begin();
#pragma unroll 1
      for (int t = t0; t < t1; ++t) {
        const int key0 = t * kTileKeys;
        if (tid == 0) odd_keys = 0;
        dma_tile(kbuf[0], kp + (int64_t)key0 * kD, keys - key0, from, wave);
        dma_tile(vbuf[0], vp + (int64_t)key0 * kD, keys - key0, from, wave);
        dma_wait();
        __syncthreads();
        const uint64_t mine = take_nonfinite<T>(vbuf[0], tid);
        if (mine) atomicOr((unsigned long long*)&odd_keys, (unsigned long long)mine);
        __syncthreads();
        Tl::template scores<false>(kbuf[0], q, lane, S);
        mask(S, key0);
        float c = a.qmult;
        const float ref = take_scores(rs, S, c);
        rs.l += Tl::template values<false, false>(vbuf[0], S, c, ref, lane, rs.O, kbuf[0], q, next);
        if (const uint64_t odd = odd_keys) {
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              S[x][i] = __builtin_amdgcn_exp2f(fmaf(S[x][i], c, -ref));
          add_nonfinite(odd, vp, key0, limit, S, lane, rs.O);
        }
        __syncthreads();
      }
    }
  }
  if (a.part) {
    write_partial(a, rs, row, un.split, live, lane);
    return;
  }
  const float l = sum_halves(rs.l);
  if (!live) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* out = (T*)a.out + row * kD + 4 * (lane >> 5);
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      struct alignas(4 * sizeof(T)) {
        T v[4];
      } y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y.v[e] = (T)(rs.O[d][4 * i + e] * inv);
      *(decltype(y)*)(out + 32 * d + 8 * i) = y;
    }
}

hipError_t launch_attend_dense(const AttendLaunch& a) {
  if (a.dtype == SWAN_F32)
    hipLaunchKernelGGL(attend_dense_kernel<float>, dim3(a.units), dim3(256), 0, a.stream, a);
  else
    hipLaunchKernelGGL(attend_dense_kernel<_Float16>, dim3(a.units), dim3(256), 0, a.stream, a);
  return hipGetLastError();
}

}  // namespace swan
