// The norm of many gradient tensors together, and the gradients clipped to a largest norm: what comes between the last backward pass of a global batch and the
// optimizer.  Bound by memory: the norm reads every element once, the clipped copy reads and writes it once.
#include <algorithm>
#include <cstdint>
#include <memory>
#include <new>
#include "common.h"

// A launch takes up to GR_TENSORS tensors as arguments (a launch's arguments hold 4 KiB), further ones go out in further launches.  A block works on one chunk
// of one tensor; chunk sizes follow from the total, so that partial sums stay few.
#define GR_TENSORS 96
#define GR_THREADS 256
#define GR_VECS 8  // 16-byte vectors a thread has in flight; each is touched once, past the caches (1.7 GB, norm and copy: 924 -> 882 us)
struct GradArgs {
  const void* data[GR_TENSORS];
  void* out[GR_TENSORS];
  unsigned long long n[GR_TENSORS];
  unsigned first[GR_TENSORS + 1];  // first block of each tensor
  unsigned long long bf16[(GR_TENSORS + 63) / 64];
  int tensors;
  unsigned chunk;                  // 16-byte vectors of a chunk
};

// The tensor that the block works on and its chunk there.
__device__ __forceinline__ int grad_tensor(const GradArgs& a, unsigned block, unsigned& chunk) {
  int lo = 0, hi = a.tensors - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.first[mid] <= block) lo = mid;
    else hi = mid - 1;
  }
  chunk = block - a.first[lo];
  return lo;
}
// Elements before the first 16-byte boundary of p, at most n.
template <typename T>
__host__ __device__ static inline unsigned long long grad_head(const void* p, unsigned long long n) {
  const unsigned long long h = (16 - ((uintptr_t)p & 15)) % 16 / sizeof(T);
  return h < n ? h : n;
}
template <typename T> static unsigned long long grad_vecs(const void* p, unsigned long long n) { return (n - grad_head<T>(p, n)) / (16 / sizeof(T)); }

template <typename T> struct Vec16 { static constexpr int N = 16 / sizeof(T); T v[N]; };
template <typename T>
__device__ __forceinline__ Vec16<T> load16(const T* p) {
  return __builtin_bit_cast(Vec16<T>, __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p)));
}

// Sum of squares of one chunk in float64: squares of float32 are exact there, none of them overflows or vanishes.
template <typename T>
__device__ __forceinline__ double chunk_squares(const T* data, unsigned long long n, unsigned chunk, unsigned per) {
  constexpr int V = Vec16<T>::N;
  const unsigned long long head = grad_head<T>(data, n), vecs = (n - head) / V, v0 = (unsigned long long)chunk * per, v1 = min(vecs, v0 + per);
  const T* body = data + head;
  double s = 0.0;
  unsigned long long i = v0 + threadIdx.x;
  for (; i + (GR_VECS - 1) * GR_THREADS < v1; i += GR_VECS * GR_THREADS) {
    Vec16<T> x[GR_VECS];
#pragma unroll
    for (int u = 0; u < GR_VECS; u++) x[u] = load16(body + (i + u * GR_THREADS) * V);
#pragma unroll
    for (int u = 0; u < GR_VECS; u++)
#pragma unroll
      for (int k = 0; k < V; k++) { const double d = (double)to_f32(x[u].v[k]); s = fma(d, d, s); }
  }
  for (; i < v1; i += GR_THREADS) {
    const Vec16<T> x = load16(body + i * V);
#pragma unroll
    for (int k = 0; k < V; k++) { const double d = (double)to_f32(x.v[k]); s = fma(d, d, s); }
  }
  if (chunk == 0) {  // the elements outside the whole vectors: fewer than 2 V
    const unsigned long long tail = head + vecs * V, rest = n - vecs * V;
    if (threadIdx.x < rest) {
      const double d = (double)to_f32(data[threadIdx.x < head ? threadIdx.x : tail + (threadIdx.x - head)]);
      s = fma(d, d, s);
    }
  }
  return s;
}
// Sum over a block's threads in a fixed order; the first thread gets the result.
__device__ __forceinline__ double block_sum_f64(double s, double* part, int waves) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int w = 1; w < waves; w++) s += part[w];
  return s;
}
__global__ __launch_bounds__(GR_THREADS) void grad_squares_kernel(const GradArgs a, double* __restrict__ partial) {
  __shared__ double part[GR_THREADS / 64];
  unsigned chunk;
  const int t = grad_tensor(a, blockIdx.x, chunk);
  double s = (a.bf16[t >> 6] >> (t & 63)) & 1 ? chunk_squares((const bf16_t*)a.data[t], a.n[t], chunk, a.chunk) : chunk_squares((const float*)a.data[t], a.n[t], chunk, a.chunk);
  s = block_sum_f64(s, part, GR_THREADS / 64);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}
__global__ __launch_bounds__(1024) void grad_norm_kernel(const double* __restrict__ partial, int n, float* __restrict__ norm) {
  __shared__ double part[16];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 1024) s += partial[i];
  s = block_sum_f64(s, part, 16);
  if (threadIdx.x == 0) norm[0] = (float)sqrt(s);
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const T* data, T* out, unsigned long long n, unsigned chunk, unsigned per, float c) {
  constexpr int V = Vec16<T>::N;
  const unsigned long long head = grad_head<T>(data, n), vecs = (n - head) / V, v0 = (unsigned long long)chunk * per, v1 = min(vecs, v0 + per);
  const T* body = data + head;
  T* to = out + head;
  const bool aligned = ((uintptr_t)to & 15) == 0;  // out may lie otherwise to its 16-byte boundaries than data
  auto store = [&](unsigned long long i, Vec16<T> x) {
#pragma unroll
    for (int k = 0; k < V; k++) x.v[k] = from_f32<T>(to_f32(x.v[k]) * c);
    if (aligned) __builtin_nontemporal_store(__builtin_bit_cast(f32x4, x), reinterpret_cast<f32x4*>(to + i * V));
    else {
#pragma unroll
      for (int k = 0; k < V; k++) to[i * V + k] = x.v[k];
    }
  };
  unsigned long long i = v0 + threadIdx.x;
  for (; i + (GR_VECS - 1) * GR_THREADS < v1; i += GR_VECS * GR_THREADS) {
    Vec16<T> x[GR_VECS];
#pragma unroll
    for (int u = 0; u < GR_VECS; u++) x[u] = load16(body + (i + u * GR_THREADS) * V);
#pragma unroll
    for (int u = 0; u < GR_VECS; u++) store(i + u * GR_THREADS, x[u]);
  }
  for (; i < v1; i += GR_THREADS) store(i, load16(body + i * V));
  if (chunk == 0) {
    const unsigned long long tail = head + vecs * V, rest = n - vecs * V;
    if (threadIdx.x < rest) {
      const unsigned long long e = threadIdx.x < head ? threadIdx.x : tail + (threadIdx.x - head);
      out[e] = from_f32<T>(to_f32(data[e]) * c);
    }
  }
}
__global__ __launch_bounds__(GR_THREADS) void grad_scale_kernel(const GradArgs a, const float* __restrict__ norm, float max_norm) {
  const float n = norm[0];
  float c = max_norm / (n + 1e-6f);
  if (!(c < 1.f) || !(n < INFINITY)) c = 1.f;  // a norm that is no number fails the first comparison
  unsigned chunk;
  const int t = grad_tensor(a, blockIdx.x, chunk);
  const void* data = a.data[t];
  void* out = a.out[t];
  if (c == 1.f && data == out) return;
  if ((a.bf16[t >> 6] >> (t & 63)) & 1) chunk_scale((const bf16_t*)data, (bf16_t*)out, a.n[t], chunk, a.chunk, c);
  else chunk_scale((const float*)data, (float*)out, a.n[t], chunk, a.chunk, c);
}

// ------------------------------------------------------------------------------------ host side
static int check_tensors(const char* who, int n, const dh_tensor* t) {
  if (n < 0) DH_FAIL(DH_ERR_SHAPE, "%s: %d tensors", who, n);
  if (n > 0 && !t) DH_FAIL(DH_ERR_INVALID_ARG, "%s: null pointer", who);
  for (int i = 0; i < n; i++) {
    if (t[i].dtype != DH_F32 && t[i].dtype != DH_BF16) DH_FAIL(DH_ERR_INVALID_ARG, "%s: tensor %d: unknown dtype %d", who, i, t[i].dtype);
    const size_t e = dh_elem_size(t[i].dtype);
    if (t[i].n > 0 && !t[i].data) DH_FAIL(DH_ERR_INVALID_ARG, "%s: tensor %d: null pointer", who, i);
    if (t[i].n > ((size_t)1 << 46)) DH_FAIL(DH_ERR_SHAPE, "%s: tensor %d: %zu elements", who, i, t[i].n);
    if ((uintptr_t)t[i].data % e || (uintptr_t)t[i].out % e) DH_FAIL(DH_ERR_INVALID_ARG, "%s: tensor %d is not aligned to its elements", who, i);
  }
  return DH_OK;
}
// Results that meet another tensor, or their own data other than as a whole: blocks would race, and an element be scaled twice or not at all.
static int check_apart(const char* who, int n, const dh_tensor* t) {
  struct Range { uintptr_t from, to; bool written; };
  if (n == 0) return DH_OK;
  std::unique_ptr<Range[]> ranges(new (std::nothrow) Range[2 * (size_t)n]);
  if (!ranges) DH_FAIL(DH_ERR_UNSUPPORTED, "%s: no host memory for %d tensors", who, n);
  size_t k = 0;
  for (int i = 0; i < n; i++) {
    if (t[i].n == 0) continue;
    const uintptr_t bytes = t[i].n * dh_elem_size(t[i].dtype), data = (uintptr_t)t[i].data, out = t[i].out ? (uintptr_t)t[i].out : data;
    ranges[k++] = {out, out + bytes, true};
    if (out != data) ranges[k++] = {data, data + bytes, false};
  }
  std::sort(ranges.get(), ranges.get() + k, [](const Range& a, const Range& b) { return a.from < b.from; });
  uintptr_t any = 0, written = 0;  // ends of all ranges before this one, and of those that are written
  for (size_t i = 0; i < k; i++) {
    const Range& r = ranges[i];
    if (r.from < (r.written ? any : written)) DH_FAIL(DH_ERR_INVALID_ARG, "%s: a result overlaps another tensor, or its own in part", who);
    any = std::max(any, r.to);
    if (r.written) written = std::max(written, r.to);
  }
  return DH_OK;
}
// Vectors of a chunk: 4096 (64 KiB), more where that would make over 16384 chunks (1.7 GB of gradients, norm and copy: 4096 larger ones 914 us, these 893).
static unsigned chunk_vecs(int n, const dh_tensor* t) {
  unsigned long long all = 0;
  for (int i = 0; i < n; i++) all += (unsigned long long)t[i].n * dh_elem_size(t[i].dtype) / 16 + 1;
  const unsigned long long per = std::max(4096ull, (all + 16383) / 16384);
  return (unsigned)std::min((per + GR_VECS * GR_THREADS - 1) / (GR_VECS * GR_THREADS) * (GR_VECS * GR_THREADS), 1ull << 31);
}
static unsigned long long chunks_of_tensor(const dh_tensor& t, unsigned per) {
  const unsigned long long vecs = t.dtype == DH_BF16 ? grad_vecs<bf16_t>(t.data, t.n) : grad_vecs<float>(t.data, t.n);
  return std::max(1ull, (vecs + per - 1) / per);
}
// launch(args, blocks before these, blocks) for each launch's tensors; empty tensors are left out.
template <class Launch>
static int each_launch(int n, const dh_tensor* t, Launch launch) {
  const unsigned per = chunk_vecs(n, t);
  unsigned before = 0;
  for (int i = 0; i < n;) {
    GradArgs a = {};
    a.chunk = per;
    for (; i < n && a.tensors < GR_TENSORS; i++) {
      if (t[i].n == 0) continue;
      const int k = a.tensors++;
      a.data[k] = t[i].data;
      a.out[k] = t[i].out ? t[i].out : const_cast<void*>(t[i].data);
      a.n[k] = t[i].n;
      if (t[i].dtype == DH_BF16) a.bf16[k >> 6] |= 1ull << (k & 63);
      a.first[k + 1] = a.first[k] + (unsigned)chunks_of_tensor(t[i], per);
    }
    if (a.tensors == 0) break;
    const unsigned blocks = a.first[a.tensors];
    if (int rc = launch(a, before, blocks)) return rc;
    before += blocks;
  }
  return DH_OK;
}

extern "C" size_t dh_grad_norm_ws_bytes(int n_tensors, const dh_tensor* tensors) {
  if (n_tensors <= 0 || !tensors) return 0;
  const unsigned per = chunk_vecs(n_tensors, tensors);
  unsigned long long blocks = 0;
  for (int i = 0; i < n_tensors; i++) blocks += tensors[i].n ? chunks_of_tensor(tensors[i], per) : 0;
  return blocks * sizeof(double);
}

extern "C" int dh_grad_norm(int n_tensors, const dh_tensor* tensors, float* norm, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_tensors("grad_norm", n_tensors, tensors)) return rc;
  if (!norm) DH_FAIL(DH_ERR_INVALID_ARG, "grad_norm: null pointer");
  const size_t need = dh_grad_norm_ws_bytes(n_tensors, tensors);
  if (need > 0 && (!ws || ws_bytes < need)) DH_FAIL(DH_ERR_WORKSPACE_TOO_SMALL, "grad_norm: workspace %zu < %zu bytes", ws_bytes, need);
  if ((uintptr_t)ws & 7) DH_FAIL(DH_ERR_INVALID_ARG, "grad_norm: ws must be 8-byte aligned");
  hipStream_t s = (hipStream_t)stream;
  double* partial = (double*)ws;
  const int rc = each_launch(n_tensors, tensors, [&](const GradArgs& a, unsigned before, unsigned blocks) -> int {
    grad_squares_kernel<<<blocks, GR_THREADS, 0, s>>>(a, partial + before);
    DH_LAUNCH_CHECK();
    return DH_OK;
  });
  if (rc) return rc;
  grad_norm_kernel<<<1, 1024, 0, s>>>(partial, (int)(need / sizeof(double)), norm);
  DH_LAUNCH_CHECK();
  return DH_OK;
}

extern "C" int dh_grad_clip(int n_tensors, const dh_tensor* tensors, const float* norm, float max_norm, void* stream) {
  if (int rc = check_tensors("grad_clip", n_tensors, tensors)) return rc;
  if (!(max_norm > 0.f)) DH_FAIL(DH_ERR_INVALID_ARG, "grad_clip: max_norm %g must be positive", (double)max_norm);
  if (!norm) DH_FAIL(DH_ERR_INVALID_ARG, "grad_clip: null pointer");
  if (int rc = check_apart("grad_clip", n_tensors, tensors)) return rc;
  return each_launch(n_tensors, tensors, [&](const GradArgs& a, unsigned, unsigned blocks) -> int {
    grad_scale_kernel<<<blocks, GR_THREADS, 0, (hipStream_t)stream>>>(a, norm, max_norm);
    DH_LAUNCH_CHECK();
    return DH_OK;
  });
}
