// Launchers of what a layer runs around its cache: the rows of its projections, and the
// attention of several rows per sequence (over cached tokens, over a prompt).
#pragma once

#include "swan_device.h"
#include "swan_internal.h"
#include "swan_layer.h"

namespace swan {

// [q | k | v] projections to heads (qkv_rows.hip)
struct QkvRowsLaunch {
  const void* x;        // rows of Hq q, Hkv k and Hkv v heads, 128 elements each
  int64_t seq, row;     // elements from a sequence (a row) to the next
  void* out[3];         // q, k, v: [B][heads][n][128]
  const void* w[2];     // norm weights of q and k (NULL: no norm)
  int wstep;            // elements from a head's weights to the next's (0: shared)
  int w32;              // the weights are float32 (else the rows' type)
  int B, Hq, Hkv, n, dtype;
  double eps, base;
  int32_t pos0[SWAN_MAX_BATCH];
  hipStream_t stream;
};
hipError_t launch_qkv_rows(const QkvRowsLaunch& a);

// ---------------------------------------------------------------------------
// attention of several rows per sequence (attend.h): rows of q over one of
//   pages  the pruned pages and the ring of a sequence of a cache (attend_pages.hip)
//   dense  keys and values [B][Hkv][m][128], causal or not (attend_dense.hip)
// Query rows go by group: a group's sequences attend to the same keys of a kv head, so
// all their tokens and all G query heads of it are rows of the same tiles; row
// tok * G + g of a (group, kv head) is head g of token tok, the tokens of the group's
// sequences one sequence after another.
// ---------------------------------------------------------------------------
constexpr int kTileRows = 128;   // query rows of a workgroup, 32 per wave
constexpr int kManyRows = 256;   // of one over pages for many rows
constexpr int kTileKeys = 64;    // keys of a tile (a page)
constexpr int kMaxSlots = 256;   // splits of the keys of a group, per source

// n / d for 32-bit n by a multiplication and shifts (Granlund and Montgomery, 1994)
struct Divisor {
  uint32_t mul, sh1, sh2, d;
  void set(uint32_t by) {
    d = by;
    uint32_t l = 0;
    while (l < 32 && (1ull << l) < by) ++l;
    mul = (uint32_t)(((1ull << 32) * ((1ull << l) - by)) / by + 1);
    sh1 = l < 1 ? l : 1;
    sh2 = l < 1 ? 0 : l - 1;
  }
  __device__ __forceinline__ uint32_t of(uint32_t n) const {
    const uint32_t t = __umulhi(mul, n);
    return (t + ((n - t) >> sh1)) >> sh2;
  }
};

struct AttendLaunch {
  const void* q;       // dense: rows of the storage type; pages: float32, rotated, x qmult
  const float* o0;     // dense: the state to continue from (or NULL), as o / lse below
  const float* lse0;
  void* out;           // dense, one split: [B][Hq][n][128] of the storage type
  float* part;         // partials [B Hq n][slots][kPartFloats]; NULL: write `out`
  const void* k;       // dense: keys; pages: the keys' pages
  const void* v;
  const void* k_ring;  // pages
  const void* v_ring;
  float qmult;         // dense: scale log2(e)
  int B, Hq, Hkv, n;   // n: rows of q per sequence (its token stride)
  int m, causal;       // dense: rows of k and v per sequence
  int bb, npc;         // pages: buffer tokens; page capacity of a (sequence, head)
  int slots, slot0;    // partials of a row, and the first of this source
  int dtype, groups;
  int tile_rows;       // pages: query rows of a workgroup, kTileRows or kManyRows
  Divisor by_g, by_hkv;  // of the query heads per kv head; of the kv heads
  int units;           // kv heads x row tiles x splits of all groups
  int32_t unit0[SWAN_MAX_BATCH + 1];  // first unit of a group
  int32_t tok0[SWAN_MAX_BATCH + 1];   // first token of a list entry, from its group's first
  int32_t keys[SWAN_MAX_BATCH];       // keys of a group
  int32_t toks[SWAN_MAX_BATCH];       // tokens of a group
  int64_t off[2][SWAN_MAX_BATCH];     // pages: byte offset of the group's key / value pages
  // (32-bit, as a scalar load takes them)
  int32_t nsplit[SWAN_MAX_BATCH];     // splits of a group's keys
  int32_t first[SWAN_MAX_BATCH + 1];  // first list entry of a group
  int32_t cseq[SWAN_MAX_BATCH];       // pages: cache sequence of a group; dense: its sequence
  int32_t kact[2][SWAN_MAX_BATCH];    // pages: k of the group's keys / values
  uint8_t seq[SWAN_MAX_BATCH];        // sequence of a list entry
  hipStream_t stream;
};
static_assert(sizeof(AttendLaunch) <= 4096, "passed to the kernels by value");
hipError_t launch_attend_pages(const AttendLaunch& a);
hipError_t launch_attend_dense(const AttendLaunch& a);

// y = x . M of float32 or storage-type rows [B][H][n][128], M = P of the head's kv head
// (H / Hkv heads share it) or its transpose, times mult; float32 rows out
struct RotateLaunch {
  const void* x;
  const float* P;
  float* y;
  float mult;
  int x_dtype;     // SWAN_F32 or SWAN_F16
  int transposed;
  int B, H, Hkv, n;
  int32_t rows[SWAN_MAX_BATCH];
  hipStream_t stream;
};
hipError_t launch_rotate_rows(const RotateLaunch& a);

// The partials of a row to one result: of up to two sources and a state, or (decode, with
// `own`) of one source and a decode step's own cache.
struct JoinLaunch {
  const float* part;   // [B H n][slots][kPartFloats]
  const float* o0;     // a state to continue from, or NULL
  const float* lse0;
  const float* P_vo;   // with `own`: rotates the result back, or NULL
  void* out;           // storage type, or NULL
  float* o;            // float32 state, or NULL (unless `out`)
  float* lse;
  int B, H, Hkv, n, slots, dtype;
  int own_slots;       // decode: the partials of swan_decode_attention, own_slots + 1 per row
  const float* own;
  int own_bb;
  SeqTab own_tab;
  int16_t used[2][SWAN_MAX_BATCH];  // partials of a sequence from slot base[s] on
  int base[2];
  int32_t rows[SWAN_MAX_BATCH];
  hipStream_t stream;
};
static_assert(sizeof(JoinLaunch) <= 4096, "passed to the kernels by value");
hipError_t launch_join(const JoinLaunch& a);

}  // namespace swan
