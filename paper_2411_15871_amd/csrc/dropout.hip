// Dropout of what joins the residual stream, its mask made from a counter wherever it is needed.
//
// Bound by memory: each input is read and each result written once, beside ten rounds of integer products for the bits of 8 elements: 16384 x 8192 in bf16, both passes with the bias
// gradient, 279 us, 4.8 TB/s.  Few rows are bound by their launches.
#include <algorithm>
#include "common.h"

// The 8 x 16 random bits of a vector: Philox4x32-10 (J. Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", SC 2011): ten rounds of two 32 x 32 bit products.
struct Words { uint32_t w[4]; };
__device__ __forceinline__ Words philox(uint64_t vector, uint32_t step, uint32_t site, uint32_t k0, uint32_t k1) {
  uint32_t x0 = (uint32_t)vector, x1 = (uint32_t)(vector >> 32), x2 = step, x3 = site;
#pragma unroll
  for (int r = 0; r < 10; r++) {
    const uint64_t a = (uint64_t)0xD2511F53u * x0, b = (uint64_t)0xCD9E8D57u * x2;
    x0 = (uint32_t)(b >> 32) ^ x1 ^ k0;
    x1 = (uint32_t)b;
    x2 = (uint32_t)(a >> 32) ^ x3 ^ k1;
    x3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{x0, x1, x2, x3}};
}
__device__ __forceinline__ uint32_t bits16(const Words& r, int e) { return (e & 1) ? r.w[e >> 1] >> 16 : r.w[e >> 1] & 0xffffu; }

struct DropArgs {
  size_t vecs;       // 8 elements each
  int vrow;          // vectors of a row
  uint32_t below;    // an element is dropped where its bits are below
  float factor;      // 1 / the share that is kept
  uint32_t site;
  const uint64_t* rng;
};
#define DROP_THREADS 256
// a == nullptr: zeros
template <typename T, bool BIAS>
__global__ __launch_bounds__(DROP_THREADS) void dropout_add_fwd_kernel(const DropArgs d, const T* a, const T* b, const T* __restrict__ bias, T* out) {
  const uint64_t key = d.rng[0];
  const uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32), step = (uint32_t)d.rng[1];
  for (size_t i = (size_t)blockIdx.x * DROP_THREADS + threadIdx.x; i < d.vecs; i += (size_t)gridDim.x * DROP_THREADS) {
    Vec8<T> x, y, z;
    x.load(b + i * 8);
    if (a) y.load(a + i * 8);
    if (BIAS) z.load(bias + i % d.vrow * 8);
    const Words r = philox(i, step, d.site, k0, k1);
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float s = BIAS ? x.v[e] + z.v[e] : x.v[e];
      x.v[e] = bits16(r, e) >= d.below ? s * d.factor : 0.f;
      if (a) x.v[e] += y.v[e];
    }
    x.store(out + i * 8);
  }
}
template <typename T>
__global__ __launch_bounds__(DROP_THREADS) void dropout_bwd_kernel(const DropArgs d, const T* dout, T* dx) {
  const uint64_t key = d.rng[0];
  const uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32), step = (uint32_t)d.rng[1];
  for (size_t i = (size_t)blockIdx.x * DROP_THREADS + threadIdx.x; i < d.vecs; i += (size_t)gridDim.x * DROP_THREADS) {
    Vec8<T> x;
    x.load(dout + i * 8);
    const Words r = philox(i, step, d.site, k0, k1);
#pragma unroll
    for (int e = 0; e < 8; e++) x.v[e] = bits16(r, e) >= d.below ? x.v[e] * d.factor : 0.f;
    x.store(dx + i * 8);
  }
}
// With the bias gradient: a thread keeps one vector's columns and adds up its rows, a block (column group, row group) leaves a row of partial sums.
// grid (ceil(vrow / DB_COLS), row groups)
#define DB_COLS 64   // vectors of a row that a block takes side by side
#define DB_LANES 4   // rows side by side
template <typename T>
__global__ __launch_bounds__(DB_COLS * DB_LANES) void dropout_bwd_bias_kernel(const DropArgs d, int rows, int per, const T* dout, T* dx, float* __restrict__ partial) {
  __shared__ float red[DB_LANES - 1][8][DB_COLS];
  const uint64_t key = d.rng[0];
  const uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32), step = (uint32_t)d.rng[1];
  const int c = threadIdx.x % DB_COLS, lane = threadIdx.x / DB_COLS, col = blockIdx.x * DB_COLS + c;
  const uint32_t r1 = min((uint32_t)rows, (blockIdx.y + 1) * (uint32_t)per);
  float s[8] = {};
  if (col < d.vrow)
    for (uint32_t r = blockIdx.y * (uint32_t)per + lane; r < r1; r += DB_LANES) {
      const size_t i = (size_t)r * d.vrow + col;
      Vec8<T> x;
      x.load(dout + i * 8);
      const Words w = philox(i, step, d.site, k0, k1);
#pragma unroll
      for (int e = 0; e < 8; e++) {
        x.v[e] = bits16(w, e) >= d.below ? x.v[e] * d.factor : 0.f;
        s[e] += x.v[e];
      }
      x.store(dx + i * 8);
    }
  if (lane > 0)
#pragma unroll
    for (int e = 0; e < 8; e++) red[lane - 1][e][c] = s[e];
  __syncthreads();
  if (lane == 0 && col < d.vrow) {
#pragma unroll
    for (int e = 0; e < 8; e++)
      for (int l = 1; l < DB_LANES; l++) s[e] += red[l - 1][e][c];
    float* to = partial + ((size_t)blockIdx.y * d.vrow + col) * 8;
    *reinterpret_cast<f32x4*>(to) = f32x4{s[0], s[1], s[2], s[3]};
    *reinterpret_cast<f32x4*>(to + 4) = f32x4{s[4], s[5], s[6], s[7]};
  }
}
// Few rows: all of them by one block for 32 columns, so that nothing is left to add behind it.  4 vectors x 256 rows side by side, which meet in the wave and then in LDS, in order.  us, two launches and this
// one, bf16: 1 x 4096 4.1 and 3.5, 520 x 4096 6.8 and 4.8, 2048 x 4096 13.9 and 12.1, 2048 x 512 9.4 and 8.4; beyond these (drop_direct) its blocks are too few.
#define DD_COLS 4
template <typename T>
__global__ __launch_bounds__(1024) void dropout_bwd_direct_kernel(const DropArgs d, int rows, const T* dout, T* dx, int accumulate, float* __restrict__ dbias) {
  __shared__ float red[16][DD_COLS][8];
  const uint64_t key = d.rng[0];
  const uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32), step = (uint32_t)d.rng[1];
  const int c = threadIdx.x % DD_COLS, col = blockIdx.x * DD_COLS + c, wave = threadIdx.x >> 6;
  float s[8] = {};
  if (col < d.vrow)
    for (int r = threadIdx.x / DD_COLS; r < rows; r += 1024 / DD_COLS) {
      const size_t i = (size_t)r * d.vrow + col;
      Vec8<T> x;
      x.load(dout + i * 8);
      const Words w = philox(i, step, d.site, k0, k1);
#pragma unroll
      for (int e = 0; e < 8; e++) {
        x.v[e] = bits16(w, e) >= d.below ? x.v[e] * d.factor : 0.f;
        s[e] += x.v[e];
      }
      x.store(dx + i * 8);
    }
#pragma unroll
  for (int e = 0; e < 8; e++)
#pragma unroll
    for (int o = DD_COLS; o < 64; o <<= 1) s[e] += __shfl_xor(s[e], o, 64);
  if ((threadIdx.x & 63) < DD_COLS)
#pragma unroll
    for (int e = 0; e < 8; e++) red[wave][c][e] = s[e];
  __syncthreads();
  if (threadIdx.x < DD_COLS * 8 && blockIdx.x * DD_COLS + threadIdx.x / 8 < (unsigned)d.vrow) {
    float t = 0.f;
    for (int w = 0; w < 16; w++) t += red[w][threadIdx.x / 8][threadIdx.x % 8];
    float* to = dbias + (size_t)blockIdx.x * DD_COLS * 8 + threadIdx.x;
    *to = accumulate ? *to + t : t;
  }
}
// dbias from n partial rows, in their order by threads and then in the threads' order.  A block has 32 columns, 8 threads each.  Blocks stand along x and y, up to DROP_X along x: a launch counts its
// threads along an axis in 32 bits, which 2^29 columns with 8 threads each would pass.
#define DROP_X 65536
__global__ __launch_bounds__(256) void dropout_bias_finish_kernel(const float* __restrict__ partial, int n, int H, int accumulate, float* __restrict__ dbias) {
  __shared__ float red[8][33];
  const uint32_t c = threadIdx.x & 31, col = (blockIdx.y * gridDim.x + blockIdx.x) * 32 + c;
  const int l = threadIdx.x >> 5;
  float s = 0.f;
  if (col < (uint32_t)H)
    for (int r = l; r < n; r += 8) s += partial[(size_t)r * H + col];
  red[l][c] = s;
  __syncthreads();
  if (l == 0 && col < (uint32_t)H) {
    for (int x = 1; x < 8; x++) s += red[x][c];
    dbias[col] = accumulate ? dbias[col] + s : s;
  }
}

// ------------------------------------------------------------------------------------ host side
static bool drop_unaligned(const void* p, size_t a = 16) { return ((uintptr_t)p & (a - 1)) != 0; }
static int check_drop(const char* who, int dtype, int T, int H, float p, const uint64_t* rng) {
  if (dtype != DH_F32 && dtype != DH_BF16) DH_FAIL(DH_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (T < 0 || H <= 0 || H % 8) DH_FAIL(DH_ERR_SHAPE, "%s: T=%d H=%d (H must be a positive multiple of 8)", who, T, H);
  if (!(p >= 0.f && p <= 1.f)) DH_FAIL(DH_ERR_INVALID_ARG, "%s: p %g must be 0 to 1", who, (double)p);
  if (T > 0 && !rng) DH_FAIL(DH_ERR_INVALID_ARG, "%s: null pointer", who);
  if (drop_unaligned(rng, 8)) DH_FAIL(DH_ERR_INVALID_ARG, "%s: rng must be 8-byte aligned", who);
  return DH_OK;
}
static DropArgs drop_args(int T, int H, float p, const uint64_t* rng, uint32_t site) {
  const uint32_t below = (uint32_t)((double)p * 65536.0 + 0.5);
  return {(size_t)T * (H / 8), H / 8, below, below >= 65536 ? 0.f : (float)(65536.0 / (65536 - below)), site, rng};
}
static unsigned drop_blocks(size_t vecs) { return (unsigned)std::min((vecs + DROP_THREADS - 1) / DROP_THREADS, (size_t)4096); }
static bool drop_direct(int T, int H) { return T > 0 && T <= 2048 && (long long)T * H <= 8 << 20; }
static int drop_groups(int T, int H) {
  const int cols = (H / 8 + DB_COLS - 1) / DB_COLS;
  return (int)std::max(1ll, std::min((T + 15ll) / 16, (2048ll + cols - 1) / cols));
}
static int drop_per(int T, int H) { return (int)(((long long)T + drop_groups(T, H) - 1) / drop_groups(T, H)); }

extern "C" int dh_dropout_add_fwd(int dtype, int T, int H, const void* a, const void* b, const void* bias, float p, const uint64_t* rng, uint32_t site, void* out, void* stream) {
  if (int rc = check_drop("dropout_add_fwd", dtype, T, H, p, rng)) return rc;
  if (T == 0) return DH_OK;
  if (!b || !out) DH_FAIL(DH_ERR_INVALID_ARG, "dropout_add_fwd: null pointer");
  if (drop_unaligned(a) || drop_unaligned(b) || drop_unaligned(bias) || drop_unaligned(out)) DH_FAIL(DH_ERR_INVALID_ARG, "dropout_add_fwd: a, b, bias and out must be 16-byte aligned");
  const DropArgs d = drop_args(T, H, p, rng, site);
  const unsigned n = drop_blocks(d.vecs);
  hipStream_t s = (hipStream_t)stream;
  if (dtype == DH_BF16) {
    if (bias) dropout_add_fwd_kernel<bf16_t, true><<<n, DROP_THREADS, 0, s>>>(d, (const bf16_t*)a, (const bf16_t*)b, (const bf16_t*)bias, (bf16_t*)out);
    else dropout_add_fwd_kernel<bf16_t, false><<<n, DROP_THREADS, 0, s>>>(d, (const bf16_t*)a, (const bf16_t*)b, nullptr, (bf16_t*)out);
  } else {
    if (bias) dropout_add_fwd_kernel<float, true><<<n, DROP_THREADS, 0, s>>>(d, (const float*)a, (const float*)b, (const float*)bias, (float*)out);
    else dropout_add_fwd_kernel<float, false><<<n, DROP_THREADS, 0, s>>>(d, (const float*)a, (const float*)b, nullptr, (float*)out);
  }
  DH_LAUNCH_CHECK();
  return DH_OK;
}
extern "C" size_t dh_dropout_add_bwd_ws_bytes(int T, int H) { return T <= 0 || H <= 0 || H % 8 || drop_direct(T, H) ? 0 : (size_t)drop_groups(T, H) * H * sizeof(float); }
extern "C" int dh_dropout_add_bwd(int dtype, int T, int H, const void* dout, float p, const uint64_t* rng, uint32_t site, void* dx, float* dbias, int accumulate, void* ws, size_t ws_bytes,
                                  void* stream) {
  if (int rc = check_drop("dropout_add_bwd", dtype, T, H, p, rng)) return rc;
  if (T > 0 && (!dout || !dx)) DH_FAIL(DH_ERR_INVALID_ARG, "dropout_add_bwd: null pointer");
  if (drop_unaligned(dout) || drop_unaligned(dx) || drop_unaligned(dbias, 4) || drop_unaligned(ws)) DH_FAIL(DH_ERR_INVALID_ARG, "dropout_add_bwd: dout, dx and ws must be 16-byte aligned");
  const size_t need = dbias ? dh_dropout_add_bwd_ws_bytes(T, H) : 0;
  if (need > 0 && (!ws || ws_bytes < need)) DH_FAIL(DH_ERR_WORKSPACE_TOO_SMALL, "dropout_add_bwd: workspace %zu < %zu bytes", ws_bytes, need);
  if (T == 0 && !dbias) return DH_OK;
  const DropArgs d = drop_args(T, H, p, rng, site);
  hipStream_t s = (hipStream_t)stream;
  if (!dbias) {
    if (dtype == DH_BF16) dropout_bwd_kernel<bf16_t><<<drop_blocks(d.vecs), DROP_THREADS, 0, s>>>(d, (const bf16_t*)dout, (bf16_t*)dx);
    else dropout_bwd_kernel<float><<<drop_blocks(d.vecs), DROP_THREADS, 0, s>>>(d, (const float*)dout, (float*)dx);
    DH_LAUNCH_CHECK();
    return DH_OK;
  }
  if (drop_direct(T, H)) {
    const unsigned n = (H / 8 + DD_COLS - 1) / DD_COLS;
    if (dtype == DH_BF16) dropout_bwd_direct_kernel<bf16_t><<<n, 1024, 0, s>>>(d, T, (const bf16_t*)dout, (bf16_t*)dx, accumulate, dbias);
    else dropout_bwd_direct_kernel<float><<<n, 1024, 0, s>>>(d, T, (const float*)dout, (float*)dx, accumulate, dbias);
    DH_LAUNCH_CHECK();
    return DH_OK;
  }
  const int groups = T > 0 ? drop_groups(T, H) : 0, per = T > 0 ? drop_per(T, H) : 0;
  if (T > 0) {
    const dim3 grid((H / 8 + DB_COLS - 1) / DB_COLS, groups);
    if (dtype == DH_BF16) dropout_bwd_bias_kernel<bf16_t><<<grid, DB_COLS * DB_LANES, 0, s>>>(d, T, per, (const bf16_t*)dout, (bf16_t*)dx, (float*)ws);
    else dropout_bwd_bias_kernel<float><<<grid, DB_COLS * DB_LANES, 0, s>>>(d, T, per, (const float*)dout, (float*)dx, (float*)ws);
    DH_LAUNCH_CHECK();
  }
  const unsigned columns = (unsigned)((H + 31ll) / 32), along = std::min(columns, (unsigned)DROP_X);
  dropout_bias_finish_kernel<<<dim3(along, (columns + along - 1) / along), 256, 0, s>>>((const float*)ws, groups, H, accumulate, dbias);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
