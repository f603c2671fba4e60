// Linear attention with a decay for each head: S_t = lambda S_(t-1) + k_t v_t^T, o_t = scale S_t^T q_t.
#include <algorithm>
#include "linattn.h"

// The recurrence as it stands, a token at a time: a block has a state, a thread one column (or row) of it in registers.
// grid (nkv, batch), 128 threads
#define LR_THREADS 128
template <typename T>
__global__ __launch_bounds__(LR_THREADS) void lin_rec_fwd_kernel(const LinGeom g, const T* __restrict__ qkv, const float* __restrict__ state_in, T* __restrict__ o,
                                                                 float* __restrict__ state_out) {
  __shared__ float ks[LR_THREADS], qs[LR_THREADS];
  const int hk = blockIdx.x, b = blockIdx.y, y = threadIdx.x, d = g.d, grp = g.nq / g.nkv;
  const size_t ld = (size_t)(g.nq + 2 * g.nkv) * d, st = ((size_t)b * g.nkv + hk) * d * d;
  const float lam = expf(g.log_decay[hk]);
  const bool on = y < d;
  float S[LR_THREADS];
#pragma unroll
  for (int x = 0; x < LR_THREADS; x++) S[x] = on && x < d && state_in ? state_in[st + (size_t)x * d + y] : 0.f;
  for (int t = 0; t < g.seq; t++) {
    const T* row = qkv + ((size_t)b * g.seq + t) * ld;
    __syncthreads();
    ks[y] = on ? to_f32(row[(size_t)(g.nq + hk) * d + y]) : 0.f;
    const float v = on ? to_f32(row[(size_t)(g.nq + g.nkv + hk) * d + y]) : 0.f;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < LR_THREADS; x++) S[x] = x < d ? fmaf(ks[x], v, lam * S[x]) : 0.f;
    for (int h = hk * grp; h < (hk + 1) * grp; h++) {
      __syncthreads();
      qs[y] = on ? to_f32(row[(size_t)h * d + y]) : 0.f;
      __syncthreads();
      float s = 0.f;
#pragma unroll
      for (int x = 0; x < LR_THREADS; x++) s = x < d ? fmaf(qs[x], S[x], s) : s;
      if (on) o[(((size_t)b * g.seq + t) * g.nq + h) * d + y] = from_f32<T>(s * g.scale);
    }
  }
  if (state_out && on)
#pragma unroll
    for (int x = 0; x < LR_THREADS; x++)
      if (x < d) state_out[st + (size_t)x * d + y] = S[x];
}
// grid (nkv, batch, 3): dq (forward in time), dk and dstate_in, dv (backward in time).  A thread holds M[.] = S[y][.] (dq), R[y][.] (dk) or R[.][y] (dv).
template <typename T>
__global__ __launch_bounds__(LR_THREADS) void lin_rec_bwd_kernel(const LinGeom g, const T* __restrict__ qkv, const float* __restrict__ state_in, const T* __restrict__ dout,
                                                                 const float* __restrict__ dstate_out, T* __restrict__ dqkv, float* __restrict__ dstate_in) {
  __shared__ float ws[LR_THREADS];
  const int hk = blockIdx.x, b = blockIdx.y, kind = blockIdx.z, y = threadIdx.x, d = g.d, grp = g.nq / g.nkv;
  const size_t ld = (size_t)(g.nq + 2 * g.nkv) * d, st = ((size_t)b * g.nkv + hk) * d * d;
  const float lam = expf(g.log_decay[hk]);
  const bool on = y < d;
  const float* from = kind == 0 ? state_in : dstate_out;
  float M[LR_THREADS];
#pragma unroll
  for (int x = 0; x < LR_THREADS; x++) M[x] = on && x < d && from ? from[st + (kind == 2 ? (size_t)x * d + y : (size_t)y * d + x)] : 0.f;
  auto share = [&](const T* p) {
    __syncthreads();
    ws[y] = on ? to_f32(p[y]) : 0.f;
    __syncthreads();
  };
  auto update = [&](float f, float own) {  // M = f M + own * (shared vector)
#pragma unroll
    for (int x = 0; x < LR_THREADS; x++) M[x] = x < d ? fmaf(own, ws[x], f * M[x]) : 0.f;
  };
  auto dot = [&]() {
    float s = 0.f;
#pragma unroll
    for (int x = 0; x < LR_THREADS; x++) s = x < d ? fmaf(ws[x], M[x], s) : s;
    return s;
  };
  for (int n = 0; n < g.seq; n++) {
    const int t = kind == 0 ? n : g.seq - 1 - n;
    const size_t tok = (size_t)b * g.seq + t;
    const T *row = qkv + tok * ld, *k = row + (size_t)(g.nq + hk) * d, *v = k + (size_t)g.nkv * d, *dor = dout + tok * g.nq * d;
    T* out = dqkv + tok * ld;
    if (kind == 0) {
      share(v);
      update(lam, on ? to_f32(k[y]) : 0.f);
      for (int h = hk * grp; h < (hk + 1) * grp; h++) {
        share(dor + (size_t)h * d);
        const float s = dot();
        if (on) out[(size_t)h * d + y] = from_f32<T>(s * g.scale);
      }
      continue;
    }
    for (int h = hk * grp; h < (hk + 1) * grp; h++) {
      const T *q = row + (size_t)h * d, *e = dor + (size_t)h * d;
      share(kind == 1 ? e : q);
      update(h == hk * grp && n > 0 ? lam : 1.f, on ? g.scale * to_f32((kind == 1 ? q : e)[y]) : 0.f);
    }
    share(kind == 1 ? v : k);
    const float s = dot();
    if (on) out[(size_t)(g.nq + (kind == 1 ? 0 : g.nkv) + hk) * d + y] = from_f32<T>(s);
  }
  if (kind == 1 && dstate_in && on)
#pragma unroll
    for (int x = 0; x < LR_THREADS; x++)
      if (x < d) dstate_in[st + (size_t)y * d + x] = g.seq > 0 ? lam * M[x] : M[x];
}

// ------------------------------------------------------------------------------------ single tokens
// Bound by memory: each element of a state is read and written once, 16 bytes a lane.  A block has a state (nkv, batch): d / 4 lanes side by side cover its rows, the row
// groups take every GROUPS-th row each, and their shares of o meet in LDS, in order.
#define LS_THREADS 256
template <typename T>
__global__ __launch_bounds__(LS_THREADS) void lin_step_kernel(const LinGeom g, const int32_t* __restrict__ pos, const T* __restrict__ qkv, const float* state_in, float* state_out,
                                                              T* __restrict__ o) {
  extern __shared__ float sm[];  // [groups][d]
  const int hk = blockIdx.x, b = blockIdx.y, d = g.d, grp = g.nq / g.nkv, per = d / 4, groups = LS_THREADS / per, r = threadIdx.x / per, c = threadIdx.x % per * 4;
  const int p = pos ? pos[b] : 1;
  if (p < 0) return;
  const float lam = expf(g.log_decay[hk]);
  const T* token = qkv + (size_t)b * (g.nq + 2 * g.nkv) * d;
  const T *k = token + (size_t)(g.nq + hk) * d, *v = k + (size_t)g.nkv * d;
  const size_t st = ((size_t)b * g.nkv + hk) * d * d;
  const bool on = r < groups;
  f32x4 v4 = {0.f, 0.f, 0.f, 0.f};
  if (on)
#pragma unroll
    for (int e = 0; e < 4; e++) v4[e] = to_f32(v[c + e]);
  for (int h = hk * grp; h < (hk + 1) * grp; h++) {
    const T* q = token + (size_t)h * d;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (on) {
      for (int x = r; x < d; x += groups) {
        f32x4* out = reinterpret_cast<f32x4*>(state_out + st + (size_t)x * d + c);
        f32x4 S;
        if (h == hk * grp) {
          S = p == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : *reinterpret_cast<const f32x4*>(state_in + st + (size_t)x * d + c);
          const float kx = to_f32(k[x]);
#pragma unroll
          for (int e = 0; e < 4; e++) S[e] = fmaf(kx, v4[e], lam * S[e]);
          *out = S;
        } else {
          S = *out;  // what this thread has stored
        }
        const float qx = to_f32(q[x]);
#pragma unroll
        for (int e = 0; e < 4; e++) acc[e] = fmaf(qx, S[e], acc[e]);
      }
      *reinterpret_cast<f32x4*>(sm + r * d + c) = acc;
    }
    __syncthreads();
    if ((int)threadIdx.x < d) {
      float s = 0.f;
      for (int w = 0; w < groups; w++) s += sm[w * d + threadIdx.x];
      o[((size_t)b * g.nq + h) * d + threadIdx.x] = from_f32<T>(s * g.scale);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------ host side
extern "C" size_t dh_linattn_fwd_workspace_bytes(int dtype, int batch, int seq, int nq, int nkv, int d) {
  return dtype == DH_BF16 && mix_sized(dtype, batch, seq, nq, nkv, d) ? dh_linattn_bf16_ws_bytes({batch, seq, nq, nkv, d, 1.f, nullptr}, false) : 0;
}
extern "C" size_t dh_linattn_bwd_workspace_bytes(int dtype, int batch, int seq, int nq, int nkv, int d) {
  return dtype == DH_BF16 && mix_sized(dtype, batch, seq, nq, nkv, d) ? dh_linattn_bf16_ws_bytes({batch, seq, nq, nkv, d, 1.f, nullptr}, true) : 0;
}

static bool lin_overlap(const void* a, const void* b, size_t bytes) { return a && b && (const char*)a < (const char*)b + bytes && (const char*)b < (const char*)a + bytes; }
extern "C" int dh_linattn_fwd(int dtype, int batch, int seq, int nq, int nkv, int d, float scale, const float* log_decay, const void* qkv, const float* state_in, void* o, float* state_out,
                              void* ws, size_t ws_bytes, void* stream) {
  if (int rc = mix_check("linattn_fwd", dtype, batch, seq, nq, nkv, d)) return rc;
  if (batch == 0) return DH_OK;
  if (!log_decay || (seq > 0 && (!qkv || !o))) DH_FAIL(DH_ERR_INVALID_ARG, "linattn_fwd: null pointer");
  if (mix_unaligned(qkv) || mix_unaligned(o) || mix_unaligned(state_in) || mix_unaligned(state_out) || mix_unaligned(log_decay, 4))
    DH_FAIL(DH_ERR_INVALID_ARG, "linattn_fwd: qkv, o and the states must be 16-byte aligned");
  if (lin_overlap(state_in, state_out, (size_t)batch * nkv * d * d * sizeof(float))) DH_FAIL(DH_ERR_INVALID_ARG, "linattn_fwd: state_out overlaps state_in");
  const size_t need = dh_linattn_fwd_workspace_bytes(dtype, batch, seq, nq, nkv, d);
  if (need > 0 && (!ws || ws_bytes < need)) DH_FAIL(DH_ERR_WORKSPACE_TOO_SMALL, "linattn_fwd: workspace %zu < %zu bytes", ws_bytes, need);
  if (mix_unaligned(ws)) DH_FAIL(DH_ERR_INVALID_ARG, "linattn_fwd: ws must be 16-byte aligned");
  const LinGeom g = {batch, seq, nq, nkv, d, scale, log_decay};
  hipStream_t s = (hipStream_t)stream;
  if (dtype == DH_BF16 && seq > 0) return dh_launch_linattn_fwd_bf16(g, (const bf16_t*)qkv, state_in, (bf16_t*)o, state_out, ws, s);
  lin_rec_fwd_kernel<float><<<dim3(nkv, batch), LR_THREADS, 0, s>>>(g, (const float*)qkv, state_in, (float*)o, state_out);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
extern "C" int dh_linattn_bwd(int dtype, int batch, int seq, int nq, int nkv, int d, float scale, const float* log_decay, const void* qkv, const float* state_in, const void* dout,
                              const float* dstate_out, void* dqkv, float* dstate_in, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = mix_check("linattn_bwd", dtype, batch, seq, nq, nkv, d)) return rc;
  if (batch == 0) return DH_OK;
  if (!log_decay || (seq > 0 && (!qkv || !dout || !dqkv))) DH_FAIL(DH_ERR_INVALID_ARG, "linattn_bwd: null pointer");
  if (mix_unaligned(qkv) || mix_unaligned(dout) || mix_unaligned(dqkv) || mix_unaligned(state_in) || mix_unaligned(dstate_out) || mix_unaligned(dstate_in) || mix_unaligned(log_decay, 4))
    DH_FAIL(DH_ERR_INVALID_ARG, "linattn_bwd: qkv, dout, dqkv and the states must be 16-byte aligned");
  if (lin_overlap(dstate_out, dstate_in, (size_t)batch * nkv * d * d * sizeof(float))) DH_FAIL(DH_ERR_INVALID_ARG, "linattn_bwd: dstate_in overlaps dstate_out");
  const size_t need = dh_linattn_bwd_workspace_bytes(dtype, batch, seq, nq, nkv, d);
  if (need > 0 && (!ws || ws_bytes < need)) DH_FAIL(DH_ERR_WORKSPACE_TOO_SMALL, "linattn_bwd: workspace %zu < %zu bytes", ws_bytes, need);
  if (mix_unaligned(ws)) DH_FAIL(DH_ERR_INVALID_ARG, "linattn_bwd: ws must be 16-byte aligned");
  const LinGeom g = {batch, seq, nq, nkv, d, scale, log_decay};
  hipStream_t s = (hipStream_t)stream;
  if (dtype == DH_BF16 && seq > 0) return dh_launch_linattn_bwd_bf16(g, (const bf16_t*)qkv, state_in, (const bf16_t*)dout, dstate_out, (bf16_t*)dqkv, dstate_in, ws, s);
  lin_rec_bwd_kernel<float><<<dim3(nkv, batch, 3), LR_THREADS, 0, s>>>(g, (const float*)qkv, state_in, (const float*)dout, dstate_out, (float*)dqkv, dstate_in);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
extern "C" int dh_linattn_step(int dtype, int batch, int nq, int nkv, int d, float scale, const float* log_decay, const int32_t* pos, const void* qkv, const float* state_in,
                               float* state_out, void* o, void* stream) {
  if (int rc = mix_check("linattn_step", dtype, batch, 1, nq, nkv, d)) return rc;
  if (batch == 0) return DH_OK;
  if (!log_decay || !qkv || !state_in || !state_out || !o) DH_FAIL(DH_ERR_INVALID_ARG, "linattn_step: null pointer");
  if (mix_unaligned(qkv) || mix_unaligned(o) || mix_unaligned(state_in) || mix_unaligned(state_out) || mix_unaligned(log_decay, 4) || mix_unaligned(pos, 4))
    DH_FAIL(DH_ERR_INVALID_ARG, "linattn_step: qkv, o and the states must be 16-byte aligned");
  if (state_in != state_out && lin_overlap(state_in, state_out, (size_t)batch * nkv * d * d * sizeof(float)))
    DH_FAIL(DH_ERR_INVALID_ARG, "linattn_step: state_out overlaps state_in other than as a whole");
  const LinGeom g = {batch, 1, nq, nkv, d, scale, log_decay};
  hipStream_t s = (hipStream_t)stream;
  const size_t lds = (size_t)(LS_THREADS / (d / 4)) * d * sizeof(float);
  if (dtype == DH_BF16) lin_step_kernel<bf16_t><<<dim3(nkv, batch), LS_THREADS, lds, s>>>(g, pos, (const bf16_t*)qkv, state_in, state_out, (bf16_t*)o);
  else lin_step_kernel<float><<<dim3(nkv, batch), LS_THREADS, lds, s>>>(g, pos, (const float*)qkv, state_in, state_out, (float*)o);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
