// Packed documents: what dh_docs_plan leaves in a micro-batch's table.
#pragma once
#include "common.h"

// The table: a head of DOCS_HEAD ints, then three ints a row (arrays lo, hi, pre of T): the row's document is rows lo .. hi-1 and its prefix ends before row
// `pre`.  Rows of no document have lo = hi = pre = their own index.  So row r sees keys lo[r] .. max(r + 1, pre[r]) - 1, and key j is seen by
// rows (j < pre[j] ? lo[j] : j) .. hi[j] - 1.  All four borders ascend with the row.
// Behind them the work of the tiled kernels, lists for blocks of 128 queries and for blocks of 128 keys: units of a block and a run of the 64-row tiles it
// meets, longest first.  A block with more tiles than the list's chunk length is cut into units of even length, whose partial results get a slot of workspace each;
// a second list names these blocks.  Lengths follow from the documents, on the device; room for them follows from T and the heads alone.  There is one
// list of the forward pass, and one of dQ and one of dK and dV for heads of 128 and of 64 each: more blocks of the shorter heads are resident at once, and where the backward pass is one
// launch its two kinds share the chip.
#define DOCS_MAX_T (1 << 28)
#define DOCS_MAX_DOCS (1 << 28)  // the plan's searches add two places among the starts in 32 bits
#define DOCS_MAX_RUN (1 << 30)  // tiles that a block may meet, over the heads of a group: counted in 32 bits, as is the sum of two such counts
#define DOCS_MAX_HEADS 1024
#define DOCS_HEAD 16
enum { DOCS_LIVE0, DOCS_LIVE1, DOCS_T, DOCS_NQ, DOCS_NKV, DOCS_COUNTS };  // head: the rows of documents are [live0, live1); from DOCS_COUNTS on, each list's units and cut blocks
enum { DOCS_Q, DOCS_DQ128, DOCS_DQ64, DOCS_K128, DOCS_K64, DOCS_LISTS };
#define DOCS_BLOCK 128
#define DOCS_TILE 64
// A chunk holds DOCS_CHUNK tiles at least: shorter ones cost more in beginnings, ends and merges than they share out, longer ones leave units of the chip idle.  us, D = 128:
// Q 2, 4, 8: forward of 17 documents in 4096 rows on 4:1 heads 23.6, 22.2, 22.8, backward of 1000 rows of 8 heads 28.4, 28.4, 30.9;
// K 2, 3, 6: backward of 500 rows on 8:2 23.9, 22.7, 24.4, of 100 rows there 17.2, 18.7, 20.0.
#define DOCS_CHUNK_Q 4
#define DOCS_CHUNK_K 3
// Where no block can have more than DOCS_WHOLE tiles none is cut, and no launch is needed to merge.  us: Q 4 and 10: forward of 300 rows of 4 heads 14.9 and 10.6; 10 and 13: training step
// of 700 39.5 and 46.7; K 4 and 8: backward of 440 rows of 4 heads 22.3 and 20.2; 8 and 12: of 100 rows on 8:2 18.6 and 22.9.
#define DOCS_WHOLE_Q 10
#define DOCS_WHOLE_K 8
// All heads' tiles together make at most DOCS_TARGET chunks: room for partial results follows from that, two a chunk (at D = 128 135 MB for a target of 1024 of O or dQ, or of 512 of dK
// and dV).  us: Q 512, 1024, 2048: forward of 16384 rows on 4:1 heads 327, 303, 302; K 256, 512, 1024: backward there 927, 921, 940, of 8192 rows on 32:8 668, 676, 693.
#define DOCS_TARGET_Q 1024
#define DOCS_TARGET_K 512
// Whether both halves of the backward pass go out as one launch: up to `most` 128-row blocks of all heads (figures where it is launched; at D = 64 up to four times as many, where
// lists by shares no longer pay).
#define DOCS_ONE_128 960
#define DOCS_ONE_64 1024
__host__ __device__ static inline bool docs_one_launch(int T, int nq, int nkv, int most) { return (long long)((T + DOCS_BLOCK - 1) / DOCS_BLOCK) * (nq + nkv) <= most; }
struct DocsCaps { int blocks, units, slots, splits; };
// Tiles that a chunk holds at least, by the two rules above.
__host__ __device__ static inline int docs_least(int T, int grp, int chunk, int whole) {
  const long long most = (((long long)T + DOCS_TILE - 1) / DOCS_TILE + 1) * grp;
  return most <= whole ? whole : chunk;
}
// With chunks of c > tiles of all blocks / (target / heads): sum of ceil(t / c) <= blocks + target / heads; blocks that are cut have t > c, and their units are
// fewer than 2 t / c.  A block has at most tiles(T) + 1 tiles of each head of its group.
static inline DocsCaps docs_caps(int T, int heads, int grp, int target, int chunk) {
  const long long blocks = ((long long)T + DOCS_BLOCK - 1) / DOCS_BLOCK, most = (((long long)T + DOCS_TILE - 1) / DOCS_TILE + 1) * grp, extra = target / heads + 1;
  const long long slots = most <= chunk ? 0 : blocks * ((most + chunk - 1) / chunk);
  DocsCaps c;
  c.blocks = (int)blocks;
  c.units = (int)(blocks + extra);
  c.slots = (int)(slots < 2 * extra ? slots : 2 * extra);
  c.splits = (int)(blocks < extra ? blocks : extra);
  if (c.slots == 0) c.splits = 0;
  return c;
}
struct DocsUnit { int block2, f0, f1, slot; };       // block * 2 + (1: its first unit); its run of tiles [f0, f1); slot of its partial result or -1
struct DocsSpan { int first, n, pad0, pad1; };       // of a key block: its query tiles (first, count); f0 and f1 count through the heads of the group
struct DocsSplit { int block, slot, n, pad; };       // a block that is cut: slots of its n units
struct DocsList {
  DocsUnit* units;
  DocsSpan* spans;    // lists of keys: of each unit
  DocsSplit* splits;
  DocsCaps cap;
  int counts;         // head[counts]: units; head[counts + 1]: splits
};
struct DocsTable {
  int32_t *head, *lo, *hi, *pre;
  DocsList list[DOCS_LISTS];
  size_t bytes, fwd_bytes;  // of the whole table, and of what the forward pass reads
};
static inline DocsTable docs_table(void* table, int T, int nq, int nkv) {
  DocsTable v;
  size_t at = 0;
  auto take = [&](size_t bytes) { char* r = (char*)table + at; at = dh_align_up(at + bytes, 16); return r; };
  v.head = (int32_t*)take(DOCS_HEAD * sizeof(int32_t));
  v.lo = (int32_t*)take((size_t)T * sizeof(int32_t));
  v.hi = (int32_t*)take((size_t)T * sizeof(int32_t));
  v.pre = (int32_t*)take((size_t)T * sizeof(int32_t));
  for (int i = 0; i < DOCS_LISTS; i++) {
    const bool keys = i >= DOCS_K128;
    DocsList& l = v.list[i];
    l.cap = keys ? docs_caps(T, nkv, nq / nkv, DOCS_TARGET_K, docs_least(T, nq / nkv, DOCS_CHUNK_K, DOCS_WHOLE_K)) : docs_caps(T, nq, 1, DOCS_TARGET_Q, docs_least(T, 1, DOCS_CHUNK_Q, DOCS_WHOLE_Q));
    l.units = (DocsUnit*)take((size_t)l.cap.units * sizeof(DocsUnit));
    l.spans = keys ? (DocsSpan*)take((size_t)l.cap.units * sizeof(DocsSpan)) : nullptr;
    l.splits = (DocsSplit*)take((size_t)l.cap.splits * sizeof(DocsSplit));
    l.counts = DOCS_COUNTS + 2 * i;
    if (i == DOCS_Q) v.fwd_bytes = at;
  }
  v.bytes = at;
  return v;
}
// What the kernels of one pass and head width read.
struct DocsView {
  int T;
  const int32_t *head, *lo, *hi, *pre;
  DocsList q, k;
};
static inline DocsView docs_view(const void* table, int T, int nq, int nkv, int d, bool bwd) {
  const DocsTable t = docs_table(const_cast<void*>(table), T, nq, nkv);
  return {T, t.head, t.lo, t.hi, t.pre, t.list[!bwd ? DOCS_Q : d == 64 ? DOCS_DQ64 : DOCS_DQ128], t.list[d == 64 ? DOCS_K64 : DOCS_K128]};
}
// Whether the table was made for these sizes: a kernel that finds others does nothing.
__device__ __forceinline__ bool docs_fits(const DocsView& v, int nq, int nkv) { return v.head[DOCS_T] == v.T && v.head[DOCS_NQ] == nq && v.head[DOCS_NKV] == nkv; }

struct DocsAttn {
  DocsView v;
  int nq, nkv, d;
  float scale, cap;
};
int dh_launch_attn_docs_fwd_f32(const DocsAttn& a, const float* qkv, float* o, float* lse, hipStream_t stream);
int dh_launch_attn_docs_bwd_f32(const DocsAttn& a, const float* qkv, const float* o, const float* dout, const float* lse, float* dqkv, float* delta, hipStream_t stream);
int dh_launch_attn_docs_fwd_bf16(const DocsAttn& a, const bf16_t* qkv, bf16_t* o, float* lse, void* ws, size_t ws_bytes, hipStream_t stream);
size_t dh_attn_docs_fwd_bf16_ws_bytes(int T, int nq, int nkv, int d);
int dh_launch_attn_docs_bwd_bf16(const DocsAttn& a, const bf16_t* qkv, const bf16_t* o, const bf16_t* dout, const float* lse, bf16_t* dqkv, float* delta, void* ws, size_t ws_bytes,
                                 hipStream_t stream);
size_t dh_attn_docs_bwd_bf16_ws_bytes(int T, int nq, int nkv, int d);

// A scaled score under the cap, and the cap's slope there.
__device__ __forceinline__ float docs_capped(float x, float cap, float& slope) {
  if (cap <= 0.f) { slope = 1.f; return x; }
  const float t = tanhf(x / cap);
  slope = 1.f - t * t;
  return cap * t;
}
