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

// A wave per 64 rows: the document of its first row, then, 64 starts at a time, how many more begin at or before each lane's row.
__global__ __launch_bounds__(256) void docs_rows_kernel(int T, int n_docs, const int32_t* __restrict__ start, const int32_t* __restrict__ prefix, int32_t* __restrict__ head,
                                                        int32_t* __restrict__ lo, int32_t* __restrict__ hi, int32_t* __restrict__ pre, int32_t* __restrict__ pos) {
  const int lane = threadIdx.x & 63, r0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * 64, r = r0 + lane;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const int a = min(max(n_docs > 0 ? start[0] : 0, 0), T);
    head[DOCS_LIVE0] = a;
    head[DOCS_LIVE1] = min(max(n_docs > 0 ? start[n_docs] : 0, a), T);
  }
  if (r0 >= T) return;
  int n = 0;  // starts at or before the lane's row
  if (n_docs > 0) {
    int base = starts_upto(start, n_docs + 1, r0);
    n = base;
    for (bool more = true; more;) {
      const int s = base + lane <= n_docs ? start[base + lane] : INT32_MAX;
#pragma unroll
      for (int i = 0; i < 64; i++) n += __builtin_amdgcn_readlane(s, i) <= r ? 1 : 0;
      base += 64;
      more = base <= n_docs && __builtin_amdgcn_readlane(s, 63) < r0 + 64;
    }
  }
  if (r >= T) return;
  int a = r, z = r, c = r;
  if (n >= 1 && n <= n_docs) {
    const int s = max(start[n - 1], 0), e = min(start[n], T);
    if (s <= r && r < e) {
      a = s;
      z = e;
      c = prefix ? s + min(max(prefix[n - 1], 0), e - s) : s;
    }
  }
  lo[r] = a;
  hi[r] = z;
  pre[r] = c;
  if (pos) pos[r] = r - a;
}

static int check_docs(const char* who, const dh_docs* docs) {
  if (!docs) DH_FAIL(DH_ERR_INVALID_ARG, "%s: null pointer", who);
  if (docs->T < 0 || docs->n_docs < 0 || docs->nq <= 0 || docs->nkv <= 0 || docs->nq % docs->nkv)
    DH_FAIL(DH_ERR_SHAPE, "%s: T=%d n_docs=%d nq=%d nkv=%d", who, docs->T, docs->n_docs, docs->nq, docs->nkv);
  if (docs->T > 0 && (!docs->table || (docs->n_docs > 0 && !docs->doc_start))) DH_FAIL(DH_ERR_INVALID_ARG, "%s: null pointer", who);
  if ((uintptr_t)docs->table & 15) DH_FAIL(DH_ERR_INVALID_ARG, "%s: table must be 16-byte aligned", who);
  return DH_OK;
}

extern "C" size_t dh_docs_table_bytes(int T, int nq, int nkv) {
  if (T <= 0 || nq <= 0 || nkv <= 0) return 0;
  return (DOCS_HEAD + 3 * (size_t)T) * sizeof(int32_t);
}

extern "C" int dh_docs_plan(const dh_docs* docs, void* stream) {
  if (int rc = check_docs("docs_plan", docs)) return rc;
  if (docs->T == 0) return DH_OK;
  const DocsView v = docs_view(docs);
  docs_rows_kernel<<<(unsigned)(((size_t)docs->T + 255) / 256), 256, 0, (hipStream_t)stream>>>(docs->T, docs->n_docs, docs->doc_start, docs->prefix, (int32_t*)v.head,
                                                                                           (int32_t*)v.lo, (int32_t*)v.hi, (int32_t*)v.pre, docs->pos);
  DH_LAUNCH_CHECK();
  return DH_OK;
}

// ------------------------------------------------------------------------------------ attention, a wave a row
struct DocsAttn {
  DocsView v;
  int nq, nkv, d;
  float scale, cap;
};
// grid (rows / 4, nq)
template <typename T>
__global__ __launch_bounds__(256) void attn_docs_fwd_rows_kernel(const DocsAttn a, const T* __restrict__ qkv, T* __restrict__ o, float* __restrict__ lse) {
  const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6), h = blockIdx.y, hk = h / (a.nq / a.nkv), d = a.d;
  if (r >= a.v.T) return;
  const int lo = a.v.lo[r], hi = max(r + 1, a.v.pre[r]);
  if (a.v.hi[r] <= lo) return;
  const size_t ld = (size_t)(a.nq + 2 * a.nkv) * d;
  const T* k = qkv + (size_t)(a.nq + hk) * d;
  float acc[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  docs_row_fwd(qkv + (size_t)r * ld + (size_t)h * d, k, k + (size_t)a.nkv * d, ld, lo, hi, d, a.scale, a.cap, acc, m, l);
  T* out = o + ((size_t)r * a.nq + h) * d;
#pragma unroll
  for (int c = 0; c < 4; c++)
    if (lane + 64 * c < d) out[lane + 64 * c] = from_f32<T>(acc[c] / l);
  if (lane == 0) lse[(size_t)h * a.v.T + r] = m + logf(l);
}
// dQ and delta; grid (rows / 4, nq)
template <typename T>
__global__ __launch_bounds__(256) void attn_docs_dq_rows_kernel(const DocsAttn a, const T* __restrict__ qkv, const T* __restrict__ o, const T* __restrict__ dout,
                                                                const float* __restrict__ lse, T* __restrict__ dqkv, float* __restrict__ delta) {
  const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6), h = blockIdx.y, hk = h / (a.nq / a.nkv), d = a.d;
  if (r >= a.v.T) return;
  const int lo = a.v.lo[r], hi = max(r + 1, a.v.pre[r]);
  if (a.v.hi[r] <= lo) return;
  const size_t ld = (size_t)(a.nq + 2 * a.nkv) * d, row = ((size_t)r * a.nq + h) * d, st = (size_t)h * a.v.T + r;
  const T* k = qkv + (size_t)(a.nq + hk) * d;
  float acc[4] = {0.f, 0.f, 0.f, 0.f}, dl = 0.f;
  for (int c = lane; c < d; c += 64) dl = fmaf(to_f32(dout[row + c]), to_f32(o[row + c]), dl);
  dl = wave_sum(dl);
  if (lane == 0) delta[st] = dl;
  docs_row_dq(qkv + (size_t)r * ld + (size_t)h * d, dout + row, k, k + (size_t)a.nkv * d, ld, lo, hi, d, a.scale, a.cap, lse[st], dl, acc);
  T* out = dqkv + (size_t)r * ld + (size_t)h * d;
#pragma unroll
  for (int c = 0; c < 4; c++)
    if (lane + 64 * c < d) out[lane + 64 * c] = from_f32<T>(acc[c] * a.scale);
}
// dK, dV; grid (rows / 4, nkv)
template <typename T>
__global__ __launch_bounds__(256) void attn_docs_dkv_rows_kernel(const DocsAttn a, const T* __restrict__ qkv, const T* __restrict__ dout, const float* __restrict__ lse,
                                                                 const float* __restrict__ delta, T* __restrict__ dqkv) {
  const int lane = threadIdx.x & 63, j = blockIdx.x * 4 + (threadIdx.x >> 6), hk = blockIdx.y, grp = a.nq / a.nkv, d = a.d;
  if (j >= a.v.T) return;
  const int first = j < a.v.pre[j] ? a.v.lo[j] : j, end = a.v.hi[j];
  if (end <= a.v.lo[j]) return;
  const size_t ld = (size_t)(a.nq + 2 * a.nkv) * d;
  const T* k = qkv + (size_t)j * ld + (size_t)(a.nq + hk) * d;
  float dk[4] = {0.f, 0.f, 0.f, 0.f}, dv[4] = {0.f, 0.f, 0.f, 0.f};
  for (int h = hk * grp; h < (hk + 1) * grp; h++)
    docs_row_dkv(k, k + (size_t)a.nkv * d, qkv + (size_t)h * d, ld, dout + (size_t)h * d, (size_t)a.nq * d, lse + (size_t)h * a.v.T, delta + (size_t)h * a.v.T, first, end, d, a.scale,
                 a.cap, dk, dv);
  T* out = dqkv + (size_t)j * ld + (size_t)(a.nq + hk) * d;
#pragma unroll
  for (int c = 0; c < 4; c++)
    if (lane + 64 * c < d) {
      out[lane + 64 * c] = from_f32<T>(dk[c] * a.scale);
      out[(size_t)a.nkv * d + lane + 64 * c] = from_f32<T>(dv[c]);
    }
}

// ------------------------------------------------------------------------------------ entry points
static int check_attn_docs(const char* who, int dtype, const dh_docs* docs, int d, float cap) {
  if (int rc = check_docs(who, docs)) return rc;
  if (dtype != DH_F32 && dtype != DH_BF16) DH_FAIL(DH_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (dtype == DH_F32 && (d <= 0 || d % 8 || d > 256)) DH_FAIL(DH_ERR_SHAPE, "%s: head_dim %d must be a multiple of 8, at most 256", who, d);
  if (dtype == DH_BF16 && d != 64 && d != 128) DH_FAIL(DH_ERR_SHAPE, "%s: head_dim %d must be 64 or 128", who, d);
  if (!(cap >= 0.f) || cap > 1e30f) DH_FAIL(DH_ERR_INVALID_ARG, "%s: cap %g must be 0 (none) or positive and finite", who, (double)cap);
  return DH_OK;
}
static bool unaligned16(const void* p) { return ((uintptr_t)p & 15) != 0; }
static DocsAttn attn_of(const dh_docs* docs, int d, float cap) { return {docs_view(docs), docs->nq, docs->nkv, d, (float)(1.0 / sqrt((double)d)), cap}; }

extern "C" size_t dh_attn_docs_fwd_workspace_bytes(int, int, int, int, int) { return 0; }
extern "C" size_t dh_attn_docs_bwd_workspace_bytes(int, int, int, int, int) { return 0; }

extern "C" int dh_attn_docs_fwd(int dtype, const dh_docs* docs, int d, float cap, const void* qkv, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_attn_docs("attn_docs_fwd", dtype, docs, d, cap)) return rc;
  if (docs->T == 0 || docs->n_docs == 0) return DH_OK;
  if (!qkv || !o || !lse) DH_FAIL(DH_ERR_INVALID_ARG, "attn_docs_fwd: null pointer");
  if (unaligned16(qkv) || unaligned16(o)) DH_FAIL(DH_ERR_INVALID_ARG, "attn_docs_fwd: qkv and o must be 16-byte aligned");
  (void)ws; (void)ws_bytes;
  const DocsAttn a = attn_of(docs, d, cap);
  const dim3 grid((unsigned)((docs->T + 3LL) / 4), docs->nq);
  if (dtype == DH_F32) attn_docs_fwd_rows_kernel<float><<<grid, 256, 0, (hipStream_t)stream>>>(a, (const float*)qkv, (float*)o, lse);
  else attn_docs_fwd_rows_kernel<bf16_t><<<grid, 256, 0, (hipStream_t)stream>>>(a, (const bf16_t*)qkv, (bf16_t*)o, lse);
  DH_LAUNCH_CHECK();
  return DH_OK;
}

template <typename T>
static int bwd_rows(const DocsAttn& a, const T* qkv, const T* o, const T* dout, const float* lse, T* dqkv, float* delta, hipStream_t stream) {
  const unsigned rows = (unsigned)((a.v.T + 3LL) / 4);
  attn_docs_dq_rows_kernel<T><<<dim3(rows, a.nq), 256, 0, stream>>>(a, qkv, o, dout, lse, dqkv, delta);
  DH_LAUNCH_CHECK();
  attn_docs_dkv_rows_kernel<T><<<dim3(rows, a.nkv), 256, 0, stream>>>(a, qkv, dout, lse, delta, dqkv);
  DH_LAUNCH_CHECK();
  return DH_OK;
}

extern "C" int dh_attn_docs_bwd(int dtype, const dh_docs* docs, int d, float cap, const void* qkv, const void* o, const void* dout, const float* lse, void* dqkv, float* delta,
                                void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_attn_docs("attn_docs_bwd", dtype, docs, d, cap)) return rc;
  if (docs->T == 0 || docs->n_docs == 0) return DH_OK;
  if (!qkv || !o || !dout || !lse || !dqkv || !delta) DH_FAIL(DH_ERR_INVALID_ARG, "attn_docs_bwd: null pointer");
  if (unaligned16(qkv) || unaligned16(o) || unaligned16(dout) || unaligned16(dqkv)) DH_FAIL(DH_ERR_INVALID_ARG, "attn_docs_bwd: qkv, o, dout and dqkv must be 16-byte aligned");
  (void)ws; (void)ws_bytes;
  const DocsAttn a = attn_of(docs, d, cap);
  if (dtype == DH_F32) return bwd_rows<float>(a, (const float*)qkv, (const float*)o, (const float*)dout, lse, (float*)dqkv, delta, (hipStream_t)stream);
  return bwd_rows<bf16_t>(a, (const bf16_t*)qkv, (const bf16_t*)o, (const bf16_t*)dout, lse, (bf16_t*)dqkv, delta, (hipStream_t)stream);
}
