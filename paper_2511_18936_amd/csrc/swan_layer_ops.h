// Launchers of what a layer runs around its cache: the rows of its projections, and the
// attention of several rows per sequence (over cached tokens, over a prompt).
#pragma once

#include "swan_device.h"
#include "swan_internal.h"
#include "swan_layer.h"

namespace swan {

// other forms of RoPE (rotary.h): the frequencies of half pairs, then zeros
struct RotaryForm {
  double magnitude;
  int half, interleaved;
  double freq[kD / 2];
};

// [q | k | v] projections to heads (qkv_rows.hip); with a form also heads alone, whose rows
// are anywhere (head), and which may be written in place
struct QkvRowsLaunch {
  const void* x;        // rows of Hq q, Hkv k and Hkv v heads, 128 elements each
  int64_t seq, row;     // elements from a sequence (a row) to the next
  int64_t head;         // with a form: from a head of a row to the next (else 128)
  void* out[3];         // q, k, v: [B][heads][n][128]
  const void* w[2];     // norm weights of q and k (NULL: no norm)
  int wstep;            // elements from a head's weights to the next's (0: shared)
  int w32;              // the weights are float32 (else the rows' type)
  int B, Hq, Hkv, n, dtype;
  double eps, base;
  int32_t pos0[SWAN_MAX_BATCH];
  hipStream_t stream;
};
hipError_t launch_qkv_rows(const QkvRowsLaunch& a, const RotaryForm* form = nullptr);

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
  // With a sliding window a row sees the keys from its first one on (to its causal limit,
  // where there is one), and those below `sink`, both numbered from the source's first key.
  // dense: the first one is the limit - window; pages: lo + i for row i of a list entry.
  int window;                         // 0: none
  int32_t lo[SWAN_MAX_BATCH];
  uint16_t sink[SWAN_MAX_BATCH];      // of a list entry (dense: group)
  hipStream_t stream;
};
constexpr int kMaxSinks = 65535;
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

// The partials of a row to one result: of up to two sources and a state, or (decode) of up to
// two sources and, with `own`, a decode step's own cache.
struct JoinLaunch {
  const float* part;   // [B H n][slots][kPartFloats]
  const float* o0;     // a state to continue from, or NULL
  const float* lse0;
  const float* P_vo;   // decode: rotates the result back, or NULL
  void* out;           // storage type, or NULL
  float* o;            // float32 state, or NULL (unless `out`)
  float* lse;
  int B, H, Hkv, n, slots, dtype;
  int decode;          // rows are single tokens, rotated back with P_vo
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

// ---------------------------------------------------------------------------
// decode with a sliding window (window_decode.h): the partials of one token per sequence over
// the tokens of its cache from lo on, and those below sink.  Sequence b's parts are its
// nsplit[b] splits of the pages that hold such tokens, then one for each 64 slots of its ring.
// ---------------------------------------------------------------------------
struct WindowLaunch {
  const void* q;       // [B][Hq][128] of the storage type
  const float* P_qk;
  float* qhat;         // [B][Hq][128]: rotated, x qmult
  float* part;         // [B][Hq][slots][kPartFloats]
  const void* k_pages;
  const void* v_pages;
  const void* k_ring;
  const void* v_ring;
  float qmult;
  int B, Hq, Hkv, bb, npc, slots, dtype;
  int qhat_ready;      // qhat is there already (decode steps)
  int rotate_here;     // the attention's blocks rotate q themselves (grouped heads)
  int32_t len[SWAN_MAX_BATCH], lo[SWAN_MAX_BATCH], sink[SWAN_MAX_BATCH];
  int32_t nsplit[SWAN_MAX_BATCH];  // 0: no such page
  int32_t kact[2][SWAN_MAX_BATCH];
  int64_t off[2][SWAN_MAX_BATCH];
  hipStream_t stream;
};
constexpr int kRotateHeads = 4;  // the most heads a block for which rotate_here may be set
hipError_t launch_window(const WindowLaunch& a);
// the sequences of one launch, whose k_pad is 8 kp8 at most
hipError_t launch_window_gqa(const WindowLaunch& a, const SeqGroup& g, int kp8);

// The pages of a sequence that hold tokens from lo on or below sink: the first `sinks`, then
// those from `skip` on.
struct WindowPages {
  int S, sinks, skip, count;  // pruned tokens; ... ; the pages in all
  __host__ __device__ WindowPages(int L, int bb, int lo, int sink) {
    S = L > bb ? L - bb : 0;
    const int np = pages_for(S);
    skip = lo >= S ? np : (lo > 0 ? lo : 0) / kPage;
    sinks = pages_for(sink < S ? sink : S);
    if (sinks > skip) sinks = skip;
    count = sinks + np - skip;
  }
  __host__ __device__ int page(int x) const { return x < sinks ? x : x - sinks + skip; }
};

// ---------------------------------------------------------------------------
// sequences of a cache to places of another (copy_sequences.hip)
// ---------------------------------------------------------------------------
struct CopyLaunch {
  const void* src[4];  // key pages, value pages, key ring, value ring
  void* dst[4];
  int Hkv, bb, npc_src, npc_dst, dtype, n;
  int max_pages;                   // of a destination sequence
  int32_t from[SWAN_MAX_BATCH];    // list entry: source sequence
  int32_t to[SWAN_MAX_BATCH];      // destination sequence
  int32_t len[SWAN_MAX_BATCH];     // tokens of the source
  int32_t first[SWAN_MAX_BATCH];   // tokens first .. first + drop - 1 are left out
  int32_t drop[SWAN_MAX_BATCH];
  int32_t k[2][SWAN_MAX_BATCH];
  int64_t off_src[2][SWAN_MAX_BATCH];
  int64_t off_dst[2][SWAN_MAX_BATCH];
  hipStream_t stream;
};
static_assert(sizeof(CopyLaunch) <= 4096, "passed to the kernel by value");
hipError_t launch_copy(const CopyLaunch& a);

}  // namespace swan
