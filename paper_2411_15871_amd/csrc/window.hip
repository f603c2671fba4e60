// Causal attention with a sliding window and sinks: entry points, and the form for single tokens.
#include <algorithm>
#include "window.h"

// ------------------------------------------------------------------------------------ single tokens
// Bound by memory: each visible row of the cache is read once.  LANES lanes read a row of a head, 8 elements each, so that a wave has 64 / LANES rows in flight a load; each such
// group keeps a reference maximum, sum and accumulators of its own for up to GH query heads, and all groups meet in LDS, in order.  64 sequences on 32:8 heads of 128, window 4096, bf16: all windows
// full 200 us, 5.4 TB/s; of mixed lengths, an eighth of them unused and an eighth at their first token, 147 to 162 us for 660 to 720 MB of visible rows, 4.3 to 4.5 TB/s: the longest end last (264 with
// sums across lanes through LDS, a maximum that follows every row and no rows fetched ahead).
struct WindowStep {
  WindowGeom g;  // seq: rows of the cache
  int chunk;     // keys of a block
  int splits;    // blocks that share a sequence's keys
};
#define WS_THREADS 256
#define WS_MAX_ROWS (1 << 30)  // counts of keys are 32-bit numbers, which a turn of the ring and the loads ahead may double
#define WS_ROWS 4    // rows a lane has in flight
#define WS_TAU 8.0f  // log2 of the headroom that weights may take over the reference maximum before it moves
// Sum over 8 or 16 neighbouring lanes, in all of them, by lane permutations inside the vector ALU.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
  x = dpp_add<0xb1>(x);   // lane ^ 1
  x = dpp_add<0x4e>(x);   // lane ^ 2
  x = dpp_add<0x141>(x);  // 8 lanes mirrored: the other four
  if constexpr (LANES == 16) x = dpp_add<0x140>(x);  // 16 lanes mirrored
  return x;
}
// grid (splits * head groups, nkv, batch)
template <typename T, int LANES, int GH>
__global__ __launch_bounds__(WS_THREADS) void window_step_kernel(const WindowStep a, const int32_t* __restrict__ pos, const T* __restrict__ qkv, T* __restrict__ kv, T* __restrict__ o,
                                                                 float* __restrict__ part) {
  constexpr int GROUPS = WS_THREADS / LANES;
  extern __shared__ float sm[];  // [GROUPS][GH][2 + LANES * 8]
  const WindowGeom& g = a.g;
  const int b = blockIdx.z, hk = blockIdx.y, split = blockIdx.x % a.splits, h0 = blockIdx.x / a.splits * GH, grp = g.nq / g.nkv, d = g.d, p = pos[b];
  const int group = threadIdx.x / LANES, l = threadIdx.x % LANES, heads = min(GH, grp - h0), c0 = l * 8;
  if (p < 0) return;
  const int lo = max(0, p - g.window + 1), ns = min(g.sinks, lo), n = ns + p + 1 - lo, turn = g.seq - g.sinks;
  const int from = split * a.chunk, to = min(n, from + a.chunk);
  const size_t ld = (size_t)2 * g.nkv * d;
  const T* token = qkv + (size_t)b * (g.nq + 2 * g.nkv) * d;
  T* cache = kv + (size_t)b * g.seq * ld + (size_t)hk * d;
  const T* now = token + (size_t)(g.nq + hk) * d;
  const bool on = c0 < d, ring = p >= g.seq;
  // Row of the c-th key that the token sees: sinks, then positions from lo on.  Behind the first turn lo lies behind the sinks, and the window wraps once at most.
  const int first = ring ? g.sinks + (lo - g.sinks) % turn : lo;
  auto row = [&](int c) {
    const int r = first + c - ns;
    return c < ns ? c : r < g.seq ? r : r - turn;
  };
  if (from < n && to == n && h0 == 0 && group == 0 && on) {  // the token's own key and value
    T* at = cache + row(n - 1) * ld + c0;
    Vec8<T> x, y;
    x.load(now + c0);
    y.load(now + (size_t)g.nkv * d + c0);
    x.store(at);
    y.store(at + (size_t)g.nkv * d);
  }
  float q[GH][8], acc[GH][8], m[GH], sum[GH];  // scores in log2
#pragma unroll
  for (int h = 0; h < GH; h++) {
    m[h] = -3.0e38f;
    sum[h] = 0.f;
    Vec8<T> x;
    if (on && h < heads) x.load(token + (size_t)(hk * grp + h0 + h) * d + c0);
#pragma unroll
    for (int e = 0; e < 8; e++) { q[h][e] = on && h < heads ? x.v[e] * (g.scale * 1.4426950408889634f) : 0.f; acc[h][e] = 0.f; }
  }
  Raw8<T> rk[WS_ROWS], rv[WS_ROWS];
  auto fetch = [&](int c) {
#pragma unroll
    for (int u = 0; u < WS_ROWS; u++) {
      const int cu = min(c + u * GROUPS, to - 1);
      const T* at = (cu == n - 1 ? now : cache + row(cu) * ld) + (on ? c0 : 0);  // lanes behind the head read its first columns, which count for nothing
      rk[u].load(at);
      rv[u].load(at + (size_t)g.nkv * d);
    }
  };
  if (from + group < to) fetch(from + group);
  for (int c = from + group; c < to; c += GROUPS * WS_ROWS) {
    float s[GH][WS_ROWS];
#pragma unroll
    for (int u = 0; u < WS_ROWS; u++)
#pragma unroll
      for (int h = 0; h < GH; h++) {
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) x = fmaf(q[h][e], rk[u].get(e), x);
        s[h][u] = on ? x : 0.f;
      }
    float v[WS_ROWS][8];
#pragma unroll
    for (int u = 0; u < WS_ROWS; u++)
#pragma unroll
      for (int e = 0; e < 8; e++) v[u][e] = rv[u].get(e);
    if (c + GROUPS * WS_ROWS < to) fetch(c + GROUPS * WS_ROWS);
    bool move = false;
    float top[GH];
#pragma unroll
    for (int h = 0; h < GH; h++) {
#pragma unroll
      for (int u = 0; u < WS_ROWS; u++) {
        const float x = lanes_sum<LANES>(s[h][u]);
        s[h][u] = c + u * GROUPS < to ? x : -INFINITY;
        top[h] = u == 0 ? x : __builtin_elementwise_maximum(top[h], s[h][u]);
      }
      move |= !(top[h] <= m[h] + WS_TAU);
    }
    if (__any(move)) {
#pragma unroll
      for (int h = 0; h < GH; h++) {
        const float mn = __builtin_elementwise_maximum(m[h], top[h]), alpha = __builtin_amdgcn_exp2f(m[h] - mn);
        sum[h] *= alpha;
#pragma unroll
        for (int e = 0; e < 8; e++) acc[h][e] *= alpha;
        m[h] = mn;
      }
    }
#pragma unroll
    for (int u = 0; u < WS_ROWS; u++) {
      const bool in = c + u * GROUPS < to;  // rows behind the block's last are copies of it, which may hold an infinity
#pragma unroll
      for (int h = 0; h < GH; h++) {
        const float w = __builtin_amdgcn_exp2f(s[h][u] - m[h]);
        sum[h] += in ? w : 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) acc[h][e] = fmaf(w, in ? v[u][e] : 0.f, acc[h][e]);
      }
    }
  }
  constexpr int PER = 2 + LANES * 8;
#pragma unroll
  for (int h = 0; h < GH; h++) {
    float* to_s = sm + (group * GH + h) * PER;
    if (l == 0) { to_s[0] = m[h]; to_s[1] = sum[h]; }
#pragma unroll
    for (int e = 0; e < 8; e++) to_s[2 + c0 + e] = acc[h][e];
  }
  __syncthreads();
  for (int x = threadIdx.x; x < heads * d; x += WS_THREADS) {
    const int h = x / d, c = x % d, hq = hk * grp + h0 + h;
    float M = -3.0e38f, L = 0.f, A = 0.f;
    for (int w = 0; w < GROUPS; w++) M = __builtin_elementwise_maximum(M, sm[(w * GH + h) * PER]);
    for (int w = 0; w < GROUPS; w++) {
      const float* of = sm + (w * GH + h) * PER;
      if (of[1] == 0.f) continue;  // no key, or none of any weight
      const float f = __builtin_amdgcn_exp2f(of[0] - M);
      L = fmaf(f, of[1], L);
      A = fmaf(f, of[2 + c], A);
    }
    if (a.splits == 1) {
      o[((size_t)b * g.nq + hq) * d + c] = from_f32<T>(A / L);  // no weight at all: 0 / 0
    } else {
      float* to_p = part + (((size_t)b * g.nq + hq) * a.splits + split) * (d + 2);
      if (c == 0) { to_p[0] = M; to_p[1] = L; }
      to_p[2 + c] = A;
    }
  }
}
// grid (nq, batch), d threads
template <typename T>
__global__ void window_step_merge_kernel(const WindowStep a, const int32_t* __restrict__ pos, const float* __restrict__ part, T* __restrict__ o) {
  extern __shared__ float sm[];  // reference maximum of each block's share, then their sums
  const int b = blockIdx.y, h = blockIdx.x, d = a.g.d, c = threadIdx.x, n = a.splits;
  if (pos[b] < 0) return;
  const float* of = part + ((size_t)b * a.g.nq + h) * n * (d + 2);
  for (int s = c; s < n; s += d) {
    sm[s] = of[(size_t)s * (d + 2)];
    sm[n + s] = of[(size_t)s * (d + 2) + 1];
  }
  __syncthreads();
  float M = -3.0e38f, L = 0.f, A = 0.f;
  for (int s = 0; s < n; s++) M = __builtin_elementwise_maximum(M, sm[s]);
#pragma unroll 8
  for (int s = 0; s < n; s++) {
    const float l = sm[n + s], x = of[(size_t)s * (d + 2) + 2 + c], f = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(sm[s] - M);
    L = fmaf(f, l, L);
    A = l == 0.f ? A : fmaf(f, x, A);
  }
  o[((size_t)b * a.g.nq + h) * d + c] = from_f32<T>(A / L);
}

// ------------------------------------------------------------------------------------ host side
static WindowGeom window_geom(int batch, int seq, int window, int sinks, int nq, int nkv, int d) { return {batch, seq, window, sinks, nq, nkv, d, (float)(1.0 / sqrt((double)d))}; }
static int check_window(const char* who, int dtype, int batch, int seq, int window, int sinks, int nq, int nkv, int d) {
  if (int rc = mix_check(who, dtype, batch, seq, nq, nkv, d)) return rc;
  if (window < 1 || sinks < 0) DH_FAIL(DH_ERR_SHAPE, "%s: window=%d sinks=%d (at least 1 and 0)", who, window, sinks);
  return DH_OK;
}
static bool window_sized(int dtype, int batch, int seq, int window, int sinks, int nq, int nkv, int d) { return mix_sized(dtype, batch, seq, nq, nkv, d) && window >= 1 && sinks >= 0; }
extern "C" size_t dh_attn_window_fwd_workspace_bytes(int dtype, int batch, int seq, int window, int sinks, int nq, int nkv, int d) {
  return dtype == DH_BF16 && window_sized(dtype, batch, seq, window, sinks, nq, nkv, d) ? dh_window_fwd_bf16_ws_bytes(window_geom(batch, seq, window, sinks, nq, nkv, d)) : 0;
}
extern "C" size_t dh_attn_window_bwd_workspace_bytes(int dtype, int batch, int seq, int window, int sinks, int nq, int nkv, int d) {
  return dtype == DH_BF16 && window_sized(dtype, batch, seq, window, sinks, nq, nkv, d) ? dh_window_bwd_bf16_ws_bytes(window_geom(batch, seq, window, sinks, nq, nkv, d)) : 0;
}

extern "C" int dh_attn_window_fwd(int dtype, int batch, int seq, int window, int sinks, int nq, int nkv, int d, const void* qkv, void* o, float* lse, void* ws, size_t ws_bytes,
                                  void* stream) {
  if (int rc = check_window("attn_window_fwd", dtype, batch, seq, window, sinks, nq, nkv, d)) return rc;
  if (batch == 0 || seq == 0) return DH_OK;
  if (!qkv || !o || !lse) DH_FAIL(DH_ERR_INVALID_ARG, "attn_window_fwd: null pointer");
  if (mix_unaligned(qkv) || mix_unaligned(o)) DH_FAIL(DH_ERR_INVALID_ARG, "attn_window_fwd: qkv and o must be 16-byte aligned");
  const size_t need = dh_attn_window_fwd_workspace_bytes(dtype, batch, seq, window, sinks, nq, nkv, d);
  if (need > 0 && (!ws || ws_bytes < need)) DH_FAIL(DH_ERR_WORKSPACE_TOO_SMALL, "attn_window_fwd: workspace %zu < %zu bytes", ws_bytes, need);
  if (mix_unaligned(ws)) DH_FAIL(DH_ERR_INVALID_ARG, "attn_window_fwd: ws must be 16-byte aligned");
  const WindowGeom g = window_geom(batch, seq, window, sinks, nq, nkv, d);
  return dtype == DH_BF16 ? dh_launch_window_fwd_bf16(g, (const bf16_t*)qkv, (bf16_t*)o, lse, ws, (hipStream_t)stream)
                          : dh_launch_window_fwd_f32(g, (const float*)qkv, (float*)o, lse, (hipStream_t)stream);
}
extern "C" int dh_attn_window_bwd(int dtype, int batch, int seq, int window, int sinks, int nq, int nkv, int d, const void* qkv, const void* o, const void* dout, const float* lse,
                                  void* dqkv, float* delta, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_window("attn_window_bwd", dtype, batch, seq, window, sinks, nq, nkv, d)) return rc;
  if (batch == 0 || seq == 0) return DH_OK;
  if (!qkv || !o || !dout || !lse || !dqkv || !delta) DH_FAIL(DH_ERR_INVALID_ARG, "attn_window_bwd: null pointer");
  if (mix_unaligned(qkv) || mix_unaligned(o) || mix_unaligned(dout) || mix_unaligned(dqkv)) DH_FAIL(DH_ERR_INVALID_ARG, "attn_window_bwd: qkv, o, dout and dqkv must be 16-byte aligned");
  const size_t need = dh_attn_window_bwd_workspace_bytes(dtype, batch, seq, window, sinks, nq, nkv, d);
  if (need > 0 && (!ws || ws_bytes < need)) DH_FAIL(DH_ERR_WORKSPACE_TOO_SMALL, "attn_window_bwd: workspace %zu < %zu bytes", ws_bytes, need);
  if (mix_unaligned(ws)) DH_FAIL(DH_ERR_INVALID_ARG, "attn_window_bwd: ws must be 16-byte aligned");
  const WindowGeom g = window_geom(batch, seq, window, sinks, nq, nkv, d);
  if (dtype == DH_BF16)
    return dh_launch_window_bwd_bf16(g, (const bf16_t*)qkv, (const bf16_t*)o, (const bf16_t*)dout, lse, (bf16_t*)dqkv, delta, ws, (hipStream_t)stream);
  return dh_launch_window_bwd_f32(g, (const float*)qkv, (const float*)o, (const float*)dout, lse, (float*)dqkv, delta, (hipStream_t)stream);
}

// Query heads that a block takes at once: up to 8; a group of more goes over several blocks, 8 each and the rest in the last (9 are 8 and 1), each of which reads the cache again.
static int step_heads(int grp) { return grp > 4 ? 8 : grp > 2 ? 4 : grp; }
// Blocks that share a sequence's keys: none holds fewer than 128, and there are no more than give each unit of the chip one.  us, 256, 512 and 1024 blocks, bf16, heads of 128: one sequence on 32:8, window
// 4096, 15.9, 17.8 and 17.7; 4 23.9, 25.1 and 32.1; 32 107, 117 and 132; 64 200, 201 and 226; 16 with window 1024 23.1, 24.2 and 29.7; 48 on 16:2 39, 44 and 44.
#define WS_BLOCKS 256
static WindowStep window_step_of(int batch, int cache_rows, int window, int sinks, int nq, int nkv, int d) {
  WindowStep a = {window_geom(batch, cache_rows, window, sinks, nq, nkv, d), 0, 1};
  const long long most = std::min((long long)window + sinks, (long long)cache_rows), grp = nq / nkv, blocks = (long long)batch * nkv * ((grp + step_heads(grp) - 1) / step_heads(grp));
  a.splits = (int)std::max(1ll, std::min({(most + 127) / 128, (WS_BLOCKS + blocks - 1) / blocks, 256ll}));
  a.chunk = (int)((most + a.splits - 1) / a.splits);
  return a;
}
extern "C" size_t dh_attn_window_step_workspace_bytes(int dtype, int batch, int cache_rows, int window, int sinks, int nq, int nkv, int d) {
  if (!mix_sized(dtype, batch, 1, nq, nkv, d) || cache_rows < 1 || cache_rows > WS_MAX_ROWS || window < 1 || sinks < 0) return 0;
  const WindowStep a = window_step_of(batch, cache_rows, window, sinks, nq, nkv, d);
  return a.splits == 1 ? 0 : (size_t)batch * nq * a.splits * (d + 2) * sizeof(float);
}
template <typename T, int LANES, int GH>
static int window_step_launch(const WindowStep& a, const int32_t* pos, const T* qkv, T* kv, T* o, float* part, hipStream_t s) {
  const int grp = a.g.nq / a.g.nkv;
  const size_t lds = (size_t)(WS_THREADS / LANES) * GH * (2 + LANES * 8) * sizeof(float);
  if (lds > 65536) {
    static bool ready[DH_MAX_DEVICES] = {};
    bool& set = ready[dh_device_index()];
    if (!set) {
      DH_HIP(hipFuncSetAttribute((const void*)window_step_kernel<T, LANES, GH>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
      set = true;
    }
  }
  window_step_kernel<T, LANES, GH><<<dim3((unsigned)a.splits * ((grp + GH - 1) / GH), a.g.nkv, a.g.batch), WS_THREADS, lds, s>>>(a, pos, qkv, kv, o, part);
  DH_LAUNCH_CHECK();
  if (a.splits > 1) {
    window_step_merge_kernel<T><<<dim3(a.g.nq, a.g.batch), a.g.d, 2 * a.splits * sizeof(float), s>>>(a, pos, part, o);
    DH_LAUNCH_CHECK();
  }
  return DH_OK;
}
template <typename T, int LANES>
static int window_step_heads(const WindowStep& a, const int32_t* pos, const T* qkv, T* kv, T* o, float* part, hipStream_t s) {
  switch (step_heads(a.g.nq / a.g.nkv)) {
    case 1: return window_step_launch<T, LANES, 1>(a, pos, qkv, kv, o, part, s);
    case 2: return window_step_launch<T, LANES, 2>(a, pos, qkv, kv, o, part, s);
    case 4: return window_step_launch<T, LANES, 4>(a, pos, qkv, kv, o, part, s);
    default: return window_step_launch<T, LANES, 8>(a, pos, qkv, kv, o, part, s);
  }
}
template <typename T>
static int window_step(const WindowStep& a, const int32_t* pos, const void* qkv, void* kv, void* o, void* ws, hipStream_t s) {
  const int d = a.g.d;
  if (d > 64) return window_step_heads<T, 16>(a, pos, (const T*)qkv, (T*)kv, (T*)o, (float*)ws, s);
  return window_step_heads<T, 8>(a, pos, (const T*)qkv, (T*)kv, (T*)o, (float*)ws, s);
}
extern "C" int dh_attn_window_step(int dtype, int batch, int cache_rows, int window, int sinks, int nq, int nkv, int d, const int32_t* pos, const void* qkv, void* kv, void* o, void* ws,
                                   size_t ws_bytes, void* stream) {
  if (int rc = check_window("attn_window_step", dtype, batch, 1, window, sinks, nq, nkv, d)) return rc;
  if (cache_rows < 1 || (long long)window + sinks > cache_rows)
    DH_FAIL(DH_ERR_SHAPE, "attn_window_step: %d rows of cache hold no window of %d behind %d sinks", cache_rows, window, sinks);
  if (cache_rows > WS_MAX_ROWS) DH_FAIL(DH_ERR_SHAPE, "attn_window_step: %d rows of cache (at most %d)", cache_rows, WS_MAX_ROWS);
  if (batch == 0) return DH_OK;
  if (!pos || !qkv || !kv || !o) DH_FAIL(DH_ERR_INVALID_ARG, "attn_window_step: null pointer");
  if (mix_unaligned(qkv) || mix_unaligned(kv) || mix_unaligned(o) || mix_unaligned(pos, 4)) DH_FAIL(DH_ERR_INVALID_ARG, "attn_window_step: qkv, kv and o must be 16-byte aligned, pos 4-byte");
  const size_t need = dh_attn_window_step_workspace_bytes(dtype, batch, cache_rows, window, sinks, nq, nkv, d);
  if (need > 0 && (!ws || ws_bytes < need)) DH_FAIL(DH_ERR_WORKSPACE_TOO_SMALL, "attn_window_step: workspace %zu < %zu bytes", ws_bytes, need);
  if (mix_unaligned(ws)) DH_FAIL(DH_ERR_INVALID_ARG, "attn_window_step: ws must be 16-byte aligned");
  const WindowStep a = window_step_of(batch, cache_rows, window, sinks, nq, nkv, d);
  return dtype == DH_BF16 ? window_step<bf16_t>(a, pos, qkv, kv, o, ws, (hipStream_t)stream) : window_step<float>(a, pos, qkv, kv, o, ws, (hipStream_t)stream);
}
