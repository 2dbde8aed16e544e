// Sequences of one cache copied to places of another: pages token by token (a page is chunks
// of 64 slots; a chunk's slots move together), rings row by row.  Tokens first .. first +
// drop - 1 are left out, so token t of the copy is token t of the source before them and
// t + drop from there on; the ring's rows go to the slots of their new positions.
#include "swan_device.h"
#include "swan_layer_ops.h"

namespace swan {

constexpr int kCopyRing = 64;  // ring rows of a workgroup

// Grid (pages, then ring pieces; kv heads; list entries x roles): a workgroup has a page of
// the copy, wave w its chunks w, w + 4, ..
//
// Bound by memory.  8 sequences of 4001 tokens, 32 heads, k = 48 (529 MB read and written): 83 us,
// 6.4 TB/s, where each call has other caches; 76 us with the same ones again, which the 256 MB of
// the last cache hold in part.  32 of up to 8000 tokens, 8 heads, k = 64, cut to windows of 4096
// that begin anywhere in a page: 83 us, 6.4 TB/s, and 80.
// Non-temporal stores: copies of 300 MB 102 us, with ordinary stores 112, of 96 MB 37 and 40, of
// 26 MB 13.2 and 14.4, each call with other caches; below 10 MB no difference.  They leave the
// copy to be read from HBM: with the first decode over it 167 and 169 us, 73 and 69, 38 and 37, so
// up to some 200 MB a copy that is read at once would gain 1-5 % by ordinary ones.  With the same
// caches again: non-temporal loads 78 us for 77, but 88 for tokens moved within their pages, and
// both 83 and 94; loads four chunks ahead gain nothing.
template <int VB>
__global__ __launch_bounds__(256) void copy_kernel(CopyLaunch a) {
  constexpr int CB = VB == 1 ? 8 : 16, VCH = 8 * VB / CB;
  using Chunk = typename std::conditional<CB == 16, u32x4, u32x2>::type;
  const int e = blockIdx.z >> 1, role = blockIdx.z & 1, h = blockIdx.y;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int L = a.len[e], drop = a.drop[e], first = a.first[e];
  if ((int)blockIdx.x < a.max_pages) {
    const int S = (L > a.bb ? L - a.bb : 0) - drop, t = blockIdx.x * kPage + lane;
    if ((int)blockIdx.x * kPage >= S) return;
    const int groups = kpad_of(a.k[role][e]) / 8;
    const int64_t bytes = page_bytes_of(VB, a.k[role][e]);
    const int from = t < first ? t : t + drop;
    const char* src = (const char*)a.src[role] + a.off_src[role][e] +
                      ((int64_t)h * a.npc_src + from / kPage) * bytes;
    char* dst = (char*)a.dst[role] + a.off_dst[role][e] +
                ((int64_t)h * a.npc_dst + blockIdx.x) * bytes;
    if (t >= S) return;
    const int slot = from % kPage;
    for (int c = wave; c < groups * VCH; c += 4)
      __builtin_nontemporal_store(*(const Chunk*)(src + (c * kPage + slot) * CB),
                                  (Chunk*)(dst + (c * kPage + lane) * CB));
    src += groups * VCH * kPage * CB;
    dst += groups * VCH * kPage * CB;
    for (int c = wave; c < groups; c += 4)
      __builtin_nontemporal_store(*(const u32x2*)(src + (c * kPage + slot) * 8),
                                  (u32x2*)(dst + (c * kPage + lane) * 8));
    return;
  }
  constexpr int kRow = kD * (VB == 4 ? 4 : 2), kPieces = kRow / 16;  // of a ring row
  const int nb = min(L, a.bb), x0 = ((int)blockIdx.x - a.max_pages) * kCopyRing;
  const char* src = (const char*)a.src[2 + role] + ((int64_t)a.from[e] * a.Hkv + h) * a.bb * kRow;
  char* dst = (char*)a.dst[2 + role] + ((int64_t)a.to[e] * a.Hkv + h) * a.bb * kRow;
  const int end = min(nb, x0 + kCopyRing) * kPieces;
  for (int i = x0 * kPieces + threadIdx.x; i < end; i += 256) {
    const int pos = L - nb + i / kPieces, piece = i % kPieces;
    *(u32x4*)(dst + (int64_t)((pos - drop) % a.bb) * kRow + 16 * piece) =
        *(const u32x4*)(src + (int64_t)(pos % a.bb) * kRow + 16 * piece);
  }
}

hipError_t launch_copy(const CopyLaunch& a) {
  const dim3 grid(a.max_pages + (a.bb + kCopyRing - 1) / kCopyRing, a.Hkv, 2 * a.n);
  if (grid.x == 0) return hipSuccess;
  if (a.dtype == SWAN_F32)
    hipLaunchKernelGGL(copy_kernel<4>, grid, dim3(256), 0, a.stream, a);
  else if (a.dtype == SWAN_F16)
    hipLaunchKernelGGL(copy_kernel<2>, grid, dim3(256), 0, a.stream, a);
  else
    hipLaunchKernelGGL(copy_kernel<1>, grid, dim3(256), 0, a.stream, a);
  return hipGetLastError();
}

}  // namespace swan
