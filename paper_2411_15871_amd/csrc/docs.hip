// Attention over packed documents: the micro-batch's table, and the entry points.
#include <cstdint>
#include "docs.h"

// ------------------------------------------------------------------------------------ the table
// How many of the n ascending starts lie at or before row r: the wave looks at 64 of them at a time and keeps the 64th of the range that holds the border (one
// load up to 64 documents, two up to 4096).
__device__ __forceinline__ int starts_upto(const int32_t* start, int n, int r) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;  // the answer lies in [lo, hi]
  while (hi - lo > 64) {
    const int step = (hi - lo + 63) / 64, at = lo + lane * step;
    const int k = __popcll(__ballot(at < hi && start[min(at, n - 1)] <= r));  // the probes at or before r
    const int to = lo + min(64, max(k, 1)) * step;
    lo = k == 0 ? lo : lo + (k - 1) * step + 1;
    hi = k == 0 ? lo : min(hi, to);
  }
  return lo + __popcll(__ballot(lo + lane < hi && start[min(lo + lane, n - 1)] <= r));
}

// The work lists, a block each: thread b looks at block b (b + 256 ...) of 128 rows.  keys: a list of key blocks.
#define DOCS_STARTS 4096
struct DocsPlanArgs {
  int T, n_docs, nq, nkv;
  const int32_t *start, *prefix;
  int32_t* pos;
  DocsTable t;
};
// The rows of documents, [live0, live1): whatever the starts are, no row outside is given to a document, and 0 <= live0 <= live1 <= T.
template <class Start>
__device__ __forceinline__ void docs_live(const DocsPlanArgs& a, const Start* start, int& live0, int& live1) {
  live0 = a.n_docs > 0 ? min(max(start[0], 0), a.T) : 0;
  live1 = a.n_docs > 0 ? min(max(start[a.n_docs], live0), a.T) : 0;
}
// The document of row r: its rows [s, e) and the end of its prefix; false: none.  start: a.start, or its copy in LDS.
template <class Start>
__device__ __forceinline__ bool docs_find(const DocsPlanArgs& a, const Start* start, int live0, int live1, int r, int& s, int& e, int& c) {
  int lo = 0, hi = a.n_docs + 1;  // how many starts lie at or before r
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= r) lo = mid + 1;
    else hi = mid;
  }
  if (lo < 1 || lo > a.n_docs) return false;
  s = max(start[lo - 1], live0);
  e = min(start[lo], live1);
  if (s > r || r >= e) return false;
  c = a.prefix ? s + min(max(a.prefix[lo - 1], 0), e - s) : s;
  return true;
}
// The tiles that block b meets: first and count (0: none of its rows is of a document).
template <class Start>
__device__ __forceinline__ int docs_tiles(const DocsPlanArgs& a, const Start* start, int live0, int live1, bool keys, int b, int& first) {
  const int r0 = max(b * DOCS_BLOCK, live0), r1 = min(b * DOCS_BLOCK + DOCS_BLOCK, live1) - 1;
  int s0, e0, c0, s1, e1, c1;
  if (r0 > r1 || !docs_find(a, start, live0, live1, r0, s0, e0, c0) || !docs_find(a, start, live0, live1, r1, s1, e1, c1)) return 0;
  const int from = keys ? (r0 < c0 ? s0 : r0) : s0, to = keys ? e1 : max(r1 + 1, c1);
  first = from / DOCS_TILE;
  return max(0, (to + DOCS_TILE - 1) / DOCS_TILE - first);
}
// The chunk length, between `shortest` and `longest`, whose launch is expected to be through first: 64 lengths in even ratios, a lane each.  In tiles of a block that shares its
// unit of the chip with another (queries; 2.1 us at D = 128) or has it to itself (keys; 2.3 us): up to one round of resident blocks the longest unit counts, a fifth faster
// alone; beyond, everything over all units (a unit's beginning and end count 1.5 tiles beside another's work) and a quarter of the longest one for the end.  A partial
// result is written and read back (beyond 512 of them from memory), and the merge takes a while longer if there is any.  tiles[b]: of the first DOCS_BLOCKS blocks; longer
// rows are cut at `shortest`.  (Always `shortest` and this, us: one document of 4096 rows on 4:1 heads, forward 49 and 39, backward 131 and 91; 32:8 x 8192 forward 248 and 230.)
#define DOCS_BLOCKS 1024
__device__ __forceinline__ int docs_chunk(const DocsPlanArgs& a, int list, int blocks, int shortest, int longest, float all, const int* tiles) {
  __shared__ int units[4][64], cuts[4][64], tops[4][64];
  if (blocks > DOCS_BLOCKS || shortest >= longest || all <= 144.f) return shortest;  // (so few tiles: any cut fits)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, heads = list >= DOCS_K128 ? a.nkv : a.nq;
  const int ch = max(shortest, (int)ceilf((float)longest * exp2f(-(float)lane / 63.f * log2f((float)longest / (float)shortest)) - 1e-3f));
  const float inv = 1.f / (float)ch;
  int n = 0, cut = 0, top = 0;
  for (int b = wave; b < blocks; b += 4) {
    const int t = tiles[b], k = (int)ceilf((float)t * inv - 1e-4f);
    n += k;
    cut += k > 1 ? k : 0;
    top = max(top, min(t, ch));
  }
  units[wave][lane] = n;
  cuts[wave][lane] = cut;
  tops[wave][lane] = top;
  __syncthreads();
  const float N = (float)(units[0][lane] + units[1][lane] + units[2][lane] + units[3][lane]) * heads, C = (float)(cuts[0][lane] + cuts[1][lane] + cuts[2][lane] + cuts[3][lane]) * heads;
  const float L = (float)max(max(tops[0][lane], tops[1][lane]), max(tops[2][lane], tops[3][lane]));
  // Blocks resident at once; where the backward pass is one launch, each kind's share of them.  (dQ by the forward pass's list and by its own, us: 2000 rows on 16:4 66 and 55,
  // 16:8 x 4096 capped 154 and 143, at D = 64 4001 rows of 8 heads 49.2 and 47.7.  Shares of dQ, D = 128, 80, 112, 200: 1500 rows on 8:2 44, 38, 40; D = 64, 272, 400: 2000 on 16:4 41,
  // 39.  Of dK and dV, 112, 144, 176: 2000 rows 57, 55, 57, 1000 of 8 heads 28, 28, 36; D = 64, 180, 240, 300: 4001 rows 58, 48, 48, 2000 44, 39, 40.)
  const bool one = docs_one_launch(a.T, a.nq, a.nkv, list == DOCS_DQ64 || list == DOCS_K64 ? DOCS_ONE_64 : DOCS_ONE_128), pairs = list == DOCS_Q || list == DOCS_DQ64 || (list == DOCS_DQ128 && !one);
  const float slots = list == DOCS_Q ? 512.f : list == DOCS_DQ128 ? (one ? 112.f : 512.f) : list == DOCS_DQ64 ? (one ? 400.f : 512.f) : list == DOCS_K64 ? (one ? 240.f : 400.f) : one ? 144.f : 256.f;
  const float together = fmaxf(L, (all + 1.5f * N) / slots + 0.25f * L);
  const float time = (N > slots ? together : !pairs ? L : L * (0.8f + 0.2f / 256.f * fmaxf(N - 256.f, 0.f))) + (C > 0.f ? 1.5f + 0.004f * C + 0.008f * fmaxf(C - 512.f, 0.f) : 0.f);
  float best = time;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) best = fminf(best, __shfl_xor(best, d, 64));
  const unsigned long long who = __ballot(time == best);
  return __builtin_amdgcn_readlane(ch, who ? __builtin_ctzll(who) : 63);
}

__device__ __forceinline__ void docs_head(const DocsPlanArgs& a, int list, int live0, int live1, int units, int splits) {
  a.t.head[a.t.list[list].counts] = units;
  a.t.head[a.t.list[list].counts + 1] = splits;
  if (list != 0) return;
  a.t.head[DOCS_LIVE0] = live0;
  a.t.head[DOCS_LIVE1] = live1;
  a.t.head[DOCS_T] = a.T;
  a.t.head[DOCS_NQ] = a.nq;
  a.t.head[DOCS_NKV] = a.nkv;
}
template <class Start>
__device__ __forceinline__ void docs_lists(const DocsPlanArgs& a, const Start* start, int list) {
  __shared__ unsigned long long wave_all[4], wave_cut[4];
  __shared__ int wave_top[4], hist[64], from[64], tiles[DOCS_BLOCKS], all_units;
  const bool keys = list >= DOCS_K128;
  const int tid = threadIdx.x, grp = keys ? a.nq / a.nkv : 1, heads = keys ? a.nkv : a.nq;
  const DocsCaps cap = a.t.list[list].cap;
  DocsUnit* units = a.t.list[list].units;
  DocsSpan* spans = a.t.list[list].spans;
  DocsSplit* splits = a.t.list[list].splits;
  int live0, live1;
  docs_live(a, start, live0, live1);
  if (tid < 64) hist[tid] = 0;
  unsigned long long mine = 0;
  int top = 1, first0 = 0, tiles0 = 0, first;
  for (int b = tid; b < cap.blocks; b += 256) {
    const int t = docs_tiles(a, start, live0, live1, keys, b, first) * grp;
    if (b == tid) { tiles0 = t; first0 = first; }
    if (b < DOCS_BLOCKS) tiles[b] = t;
    mine += t;
    top = max(top, t);
  }
  if (cap.slots == 0 && cap.blocks <= 64) {  // nothing is cut and everything is resident at once: one unit a block, in their order
    const uint64_t have = __ballot(tiles0 > 0);
    if (tid < 64) {
      const int at = __popcll(have & ((1ull << tid) - 1));
      if (tiles0 > 0) {
        units[at] = {tid * 2 + 1, keys ? 0 : first0, (keys ? 0 : first0) + tiles0, -1};
        if (keys) spans[at] = {first0, tiles0 / grp, 0, 0};
      }
      if (tid == 0) docs_head(a, list, live0, live1, __popcll(have), 0);
    }
    return;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {  // (a lane's addition to one place of LDS after the other took 3 us)
    mine += __shfl_xor(mine, d, 64);
    top = max(top, __shfl_xor(top, d, 64));
  }
  if ((tid & 63) == 0) { wave_all[tid >> 6] = mine; wave_top[tid >> 6] = top; }
  __syncthreads();
  const unsigned long long all = wave_all[0] + wave_all[1] + wave_all[2] + wave_all[3];
  const int longest = max(max(wave_top[0], wave_top[1]), max(wave_top[2], wave_top[3]));
  // all heads' tiles over the target, rounded up (float64 holds them exactly; a quotient off by a rounding still leaves the bounds of docs_caps: the next whole number is taken)
  const int target = keys ? DOCS_TARGET_K : DOCS_TARGET_Q, least = keys ? docs_least(a.T, grp, DOCS_CHUNK_K, DOCS_WHOLE_K) : docs_least(a.T, 1, DOCS_CHUNK_Q, DOCS_WHOLE_Q);
  const double want = floor((double)all * heads / target) + 1.0;
  const int shortest = (int)fmin(fmax(want, (double)least), (double)longest);
  const int ch = docs_chunk(a, list, cap.blocks, shortest, longest, (float)all * heads, tiles);
  const float steps = 63.f / (float)ch;
  // Units longest first, counted by length in 64 steps, then placed.  A block of t tiles makes n = ceil(t / ch) units, t % n of them a tile longer than the others.
  auto bucket = [&](int len) { return min(max(63 - (int)((float)len * steps), 0), 63); };
  for (int b = tid; b < cap.blocks; b += 256) {
    const int t = b == tid ? tiles0 : docs_tiles(a, start, live0, live1, keys, b, first) * grp;
    if (t == 0) continue;
    const int n = (t + ch - 1) / ch, len = t / n, more = t - len * n;
    if (more > 0) atomicAdd(&hist[bucket(len + 1)], more);
    atomicAdd(&hist[bucket(len)], n - more);
  }
  __syncthreads();
  if (tid < 64) {
    int upto = hist[tid];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d, 64);
      if (tid >= d) upto += o;
    }
    from[tid] = upto - hist[tid];
    if (tid == 63) all_units = min(upto, cap.units);
  }
  unsigned long long cut = 0;  // slots and, in the upper half, blocks that are cut, before these 256 blocks'
  for (int b0 = 0; b0 < cap.blocks; b0 += 256) {
    const int b = b0 + tid;
    first = first0;
    const int t = b >= cap.blocks ? 0 : b0 == 0 ? tiles0 : docs_tiles(a, start, live0, live1, keys, b, first) * grp;
    const int n = (t + ch - 1) / ch;
    const unsigned long long own = n > 1 ? (1ull << 32) + n : 0;
    unsigned long long upto = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned long long o = __shfl_up(upto, d, 64);
      if ((tid & 63) >= d) upto += o;
    }
    __syncthreads();  // `from` is there; the round before is through with wave_cut
    if ((tid & 63) == 63) wave_cut[tid >> 6] = upto;
    __syncthreads();
    for (int w = 0; w < (tid >> 6); w++) upto += wave_cut[w];
    const unsigned long long before = cut + upto - own;
    cut += wave_cut[0] + wave_cut[1] + wave_cut[2] + wave_cut[3];
    if (t == 0) continue;
    const int slot = n > 1 ? (int)(uint32_t)before : -1, k = (int)(before >> 32);
    if (n > 1 && k < cap.splits) splits[k] = {b, slot, n, 0};
    const int len = t / n, more = t - len * n;
    const int at0 = more > 0 ? atomicAdd(&from[bucket(len + 1)], more) : 0, at1 = atomicAdd(&from[bucket(len)], n - more) - more;
    const DocsSpan span = {first, t / grp, 0, 0};
    for (int u = 0, f = keys ? 0 : first; u < n; u++) {
      const int at = (u < more ? at0 : at1) + u, end = f + len + (u < more ? 1 : 0);
      if (at < cap.units) {
        units[at] = {b * 2 + (u == 0 ? 1 : 0), f, end, slot < 0 ? -1 : slot + u};
        if (keys) spans[at] = span;
      }
      f = end;
    }
  }
  if (tid == 0) docs_head(a, list, live0, live1, all_units, min((int)(cut >> 32), cap.splits));
}

// The first blocks make the work lists; in the others a wave takes 64 rows: the document of its first row, then, 64 starts at a time, how many more begin at or
// before each lane's row.
__global__ __launch_bounds__(256) void docs_plan_kernel(const DocsPlanArgs a) {
  if (blockIdx.x < DOCS_LISTS) {  // a chain of searches, in LDS where the starts fit (17 documents, 4096 rows: 13 us from memory)
    __shared__ int copy[DOCS_STARTS];
    const int list = blockIdx.x;
    if (a.n_docs >= DOCS_STARTS) {
      docs_lists(a, a.start, list);
    } else {
      for (int i = threadIdx.x; i < (a.n_docs > 0 ? a.n_docs + 1 : 0); i += 256) copy[i] = a.start[i];
      __syncthreads();
      docs_lists(a, (const __attribute__((address_space(3))) int*)copy, list);
    }
    return;
  }
  const int T = a.T, n_docs = a.n_docs;
  const int32_t* start = a.start;
  const int lane = threadIdx.x & 63, r0 = ((blockIdx.x - DOCS_LISTS) * 4 + (threadIdx.x >> 6)) * 64, r = r0 + lane;
  if (r0 >= T) return;
  int n = 0, live0, live1;  // n: starts at or before the lane's row
  docs_live(a, start, live0, live1);
  if (n_docs > 0) {
    int base = starts_upto(start, n_docs + 1, r0);
    n = base;
    for (bool more = true; more;) {
      const int s = base + lane <= n_docs ? start[base + lane] : INT32_MAX;
      const int s0 = __builtin_amdgcn_readlane(s, 0), s63 = __builtin_amdgcn_readlane(s, 63);
      if (s0 == s63 && s0 < r0 + 64) {  // empty documents at one place, at least 63: all that lie there (starts padded to 4096 behind the last document: 77 us one by one, 9 this way)
        const int next = max(starts_upto(start, n_docs + 1, s0), base + 64);
        n += s0 <= r ? next - base : 0;
        base = next;
      } else {
#pragma unroll 8
        for (int i = 0; i < 64; i++) n += __builtin_amdgcn_readlane(s, i) <= r ? 1 : 0;
        base += 64;
      }
      more = base <= n_docs && s63 < r0 + 64;
    }
  }
  if (r >= T) return;
  int lo = r, hi = r, pre = r;
  if (n >= 1 && n <= n_docs) {
    const int s = max(start[n - 1], live0), e = min(start[n], live1);
    if (s <= r && r < e) {
      lo = s;
      hi = e;
      pre = a.prefix ? s + min(max(a.prefix[n - 1], 0), e - s) : s;
    }
  }
  a.t.lo[r] = lo;
  a.t.hi[r] = hi;
  a.t.pre[r] = pre;
  if (a.pos) a.pos[r] = r - lo;
}

static int check_docs(const char* who, const dh_docs* docs, bool fwd) {  // fwd: the call reads the forward pass's part of the table alone
  if (!docs) DH_FAIL(DH_ERR_INVALID_ARG, "%s: null pointer", who);
  if (docs->T < 0 || docs->n_docs < 0 || docs->nq <= 0 || docs->nkv <= 0 || docs->nq % docs->nkv)
    DH_FAIL(DH_ERR_SHAPE, "%s: T=%d n_docs=%d nq=%d nkv=%d", who, docs->T, docs->n_docs, docs->nq, docs->nkv);
  if (docs->T > DOCS_MAX_T || docs->nq > DOCS_MAX_HEADS) DH_FAIL(DH_ERR_SHAPE, "%s: T=%d nq=%d (at most %d and %d)", who, docs->T, docs->nq, DOCS_MAX_T, DOCS_MAX_HEADS);
  if (docs->n_docs > DOCS_MAX_DOCS) DH_FAIL(DH_ERR_SHAPE, "%s: %d documents (at most %d)", who, docs->n_docs, DOCS_MAX_DOCS);
  if (((long long)docs->T / DOCS_TILE + 2) * (docs->nq / docs->nkv) > DOCS_MAX_RUN)
    DH_FAIL(DH_ERR_SHAPE, "%s: T=%d with %d query heads a group (T/64 times these at most 2^30)", who, docs->T, docs->nq / docs->nkv);
  if (docs->T > 0 && (!docs->table || (docs->n_docs > 0 && !docs->doc_start))) DH_FAIL(DH_ERR_INVALID_ARG, "%s: null pointer", who);
  if ((uintptr_t)docs->table & 15) DH_FAIL(DH_ERR_INVALID_ARG, "%s: table must be 16-byte aligned", who);
  if (docs->T > 0) {
    const DocsTable t = docs_table(nullptr, docs->T, docs->nq, docs->nkv);
    const size_t need = fwd ? t.fwd_bytes : t.bytes;
    if (docs->table_bytes < need) DH_FAIL(DH_ERR_WORKSPACE_TOO_SMALL, "%s: table of %zu < %zu bytes", who, docs->table_bytes, need);
  }
  return DH_OK;
}

extern "C" size_t dh_docs_table_bytes(int T, int nq, int nkv) {
  if (T <= 0 || nq <= 0 || nkv <= 0) return 0;
  return docs_table(nullptr, T, nq, nkv).bytes;
}

extern "C" int dh_docs_plan(const dh_docs* docs, void* stream) {
  if (int rc = check_docs("docs_plan", docs, false)) return rc;
  if (docs->T == 0) return DH_OK;
  const DocsPlanArgs a = {docs->T, docs->n_docs, docs->nq, docs->nkv, docs->doc_start, docs->prefix, docs->pos, docs_table(docs->table, docs->T, docs->nq, docs->nkv)};
  docs_plan_kernel<<<DOCS_LISTS + (unsigned)(((size_t)docs->T + 255) / 256), 256, 0, (hipStream_t)stream>>>(a);
  DH_LAUNCH_CHECK();
  return DH_OK;
}

// ------------------------------------------------------------------------------------ entry points
static int check_attn_docs(const char* who, bool fwd, int dtype, const dh_docs* docs, int d, float cap) {
  if (int rc = check_docs(who, docs, fwd)) return rc;
  if (dtype != DH_F32 && dtype != DH_BF16) DH_FAIL(DH_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (dtype == DH_F32 && (d <= 0 || d % 8 || d > 256)) DH_FAIL(DH_ERR_SHAPE, "%s: head_dim %d must be a multiple of 8, at most 256", who, d);
  if (dtype == DH_BF16 && d != 64 && d != 128) DH_FAIL(DH_ERR_SHAPE, "%s: head_dim %d must be 64 or 128", who, d);
  if (cap != 0.f && !(cap >= 1e-3f && cap <= 1e3f)) DH_FAIL(DH_ERR_INVALID_ARG, "%s: cap %g must be 0 (none) or 0.001 to 1000", who, (double)cap);  // (bf16: off by 2^-22 cap)
  return DH_OK;
}
static bool unaligned16(const void* p) { return ((uintptr_t)p & 15) != 0; }
static DocsAttn attn_of(const dh_docs* docs, int d, float cap, bool bwd) { return {docs_view(docs->table, docs->T, docs->nq, docs->nkv, d, bwd), docs->nq, docs->nkv, d, (float)(1.0 / sqrt((double)d)), cap}; }

static bool sized(int dtype, int T, int nq, int nkv, int d) {
  return dtype == DH_BF16 && T > 0 && T <= DOCS_MAX_T && nkv > 0 && nq > 0 && nq <= DOCS_MAX_HEADS && nq % nkv == 0 && (d == 64 || d == 128);
}
extern "C" size_t dh_attn_docs_fwd_workspace_bytes(int dtype, int T, int nq, int nkv, int d) { return sized(dtype, T, nq, nkv, d) ? dh_attn_docs_fwd_bf16_ws_bytes(T, nq, nkv, d) : 0; }
extern "C" size_t dh_attn_docs_bwd_workspace_bytes(int dtype, int T, int nq, int nkv, int d) { return sized(dtype, T, nq, nkv, d) ? dh_attn_docs_bwd_bf16_ws_bytes(T, nq, nkv, d) : 0; }

extern "C" int dh_attn_docs_fwd(int dtype, const dh_docs* docs, int d, float cap, const void* qkv, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_attn_docs("attn_docs_fwd", true, dtype, docs, d, cap)) return rc;
  if (docs->T == 0 || docs->n_docs == 0) return DH_OK;
  if (!qkv || !o || !lse) DH_FAIL(DH_ERR_INVALID_ARG, "attn_docs_fwd: null pointer");
  if (unaligned16(qkv) || unaligned16(o)) DH_FAIL(DH_ERR_INVALID_ARG, "attn_docs_fwd: qkv and o must be 16-byte aligned");
  const size_t need = dh_attn_docs_fwd_workspace_bytes(dtype, docs->T, docs->nq, docs->nkv, d);
  if (need > 0 && (!ws || ws_bytes < need)) DH_FAIL(DH_ERR_WORKSPACE_TOO_SMALL, "attn_docs_fwd: workspace %zu < %zu bytes", ws_bytes, need);
  if (unaligned16(ws)) DH_FAIL(DH_ERR_INVALID_ARG, "attn_docs_fwd: ws must be 16-byte aligned");
  const DocsAttn a = attn_of(docs, d, cap, false);
  if (dtype == DH_BF16) return dh_launch_attn_docs_fwd_bf16(a, (const bf16_t*)qkv, (bf16_t*)o, lse, ws, ws_bytes, (hipStream_t)stream);
  return dh_launch_attn_docs_fwd_f32(a, (const float*)qkv, (float*)o, lse, (hipStream_t)stream);
}

extern "C" int dh_attn_docs_bwd(int dtype, const dh_docs* docs, int d, float cap, const void* qkv, const void* o, const void* dout, const float* lse, void* dqkv, float* delta,
                                void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_attn_docs("attn_docs_bwd", false, dtype, docs, d, cap)) return rc;
  if (docs->T == 0 || docs->n_docs == 0) return DH_OK;
  if (!qkv || !o || !dout || !lse || !dqkv || !delta) DH_FAIL(DH_ERR_INVALID_ARG, "attn_docs_bwd: null pointer");
  if (unaligned16(qkv) || unaligned16(o) || unaligned16(dout) || unaligned16(dqkv)) DH_FAIL(DH_ERR_INVALID_ARG, "attn_docs_bwd: qkv, o, dout and dqkv must be 16-byte aligned");
  const size_t need = dh_attn_docs_bwd_workspace_bytes(dtype, docs->T, docs->nq, docs->nkv, d);
  if (need > 0 && (!ws || ws_bytes < need)) DH_FAIL(DH_ERR_WORKSPACE_TOO_SMALL, "attn_docs_bwd: workspace %zu < %zu bytes", ws_bytes, need);
  if (unaligned16(ws)) DH_FAIL(DH_ERR_INVALID_ARG, "attn_docs_bwd: ws must be 16-byte aligned");
  const DocsAttn a = attn_of(docs, d, cap, true);
  if (dtype == DH_F32) return dh_launch_attn_docs_bwd_f32(a, (const float*)qkv, (const float*)o, (const float*)dout, lse, (float*)dqkv, delta, (hipStream_t)stream);
  return dh_launch_attn_docs_bwd_bf16(a, (const bf16_t*)qkv, (const bf16_t*)o, (const bf16_t*)dout, lse, (bf16_t*)dqkv, delta, ws, ws_bytes, (hipStream_t)stream);
}
