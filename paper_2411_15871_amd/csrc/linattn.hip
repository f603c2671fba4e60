// Linear attention with a decay for each head: S_t = lambda S_(t-1) + k_t v_t^T, o_t = scale S_t^T q_t.
#include <algorithm>
#include "linattn.h"

// ------------------------------------------------------------------------------------ states along the pieces of a row
// grid (ceil(d * d / 1024), nkv * passes, batch), four elements a thread, LIN_BATCH pieces of them in flight (4 and 16, two passes of 16 pieces of 16 states of 128: 14.6 and 12.0 us)
#define LIN_BATCH 16
__global__ __launch_bounds__(256) void lin_carry_kernel(const LinGeom g, int pieces, int tokens, const LinCarry c0, const LinCarry c1) {
  const int b = blockIdx.z, hk = blockIdx.y % g.nkv, e = (blockIdx.x * 256 + threadIdx.x) * 4, dd = g.d * g.d;
  if (e >= dd) return;
  const LinCarry& c = (int)blockIdx.y >= g.nkv ? c1 : c0;
  const size_t head = (size_t)b * g.nkv + hk;
  const float l2 = g.log_decay[hk] * 1.4426950408889634f, f = lin_pow(l2, tokens), f_last = lin_pow(l2, g.seq - (pieces - 1) * tokens);
  const bool alone = lin_alone(l2);
  f32x4 run = {0.f, 0.f, 0.f, 0.f};
  if (c.first) run = *reinterpret_cast<const f32x4*>(c.first + head * dd + e);
  float* at = c.sums + head * pieces * dd + e;
  for (int i0 = 0; i0 < pieces; i0 += LIN_BATCH) {
    f32x4 sum[LIN_BATCH];
#pragma unroll
    for (int u = 0; u < LIN_BATCH; u++) {
      const int i = min(i0 + u, pieces - 1), s = c.rev ? pieces - 1 - i : i;
      sum[u] = *reinterpret_cast<const f32x4*>(at + (size_t)s * dd);
    }
#pragma unroll
    for (int u = 0; u < LIN_BATCH; u++) {
      if (i0 + u >= pieces) break;
      const int s = c.rev ? pieces - 1 - i0 - u : i0 + u;
      *reinterpret_cast<f32x4*>(at + (size_t)s * dd) = run;
      run = alone ? sum[u] : run * (s == pieces - 1 ? f_last : f) + sum[u];
    }
  }
  if (c.last) *reinterpret_cast<f32x4*>(c.last + head * dd + e) = run;
}
int dh_launch_lin_carry(const LinGeom& g, int pieces, int tokens, const LinCarry& c0, const LinCarry* c1, hipStream_t s) {
  lin_carry_kernel<<<dim3((g.d * g.d + 1023) / 1024, g.nkv * (c1 ? 2 : 1), g.batch), 256, 0, s>>>(g, pieces, tokens, c0, c1 ? *c1 : LinCarry{});
  DH_LAUNCH_CHECK();
  return DH_OK;
}

// ------------------------------------------------------------------------------------ single tokens
// Bound by memory: each element of a state is read and written once, 16 bytes a lane, LS_ROWS of them in flight, for up to GH query heads of its group (further ones read what the thread has stored).  A
// block has `cols` columns of a state: cols / 4 lanes side by side cover its rows, the row groups take every groups-th row each, and their shares of o meet in LDS, in order.
// Where blocks are few a state's columns are shared out over several (LS_BLOCKS).  bf16, heads of 128, us, whole states a block and shared: one sequence on 32:8 7.3 and 5.3, 16 9.4 and 7.6; 128 on
// 32:32 106, 5.1 TB/s, either way (88 where the same states come again and the chip still holds some of their 268 MB).  (With a head of the group after the other over the state 16.7 for one sequence, 37 instead of 19 for 64 on 32:8.)
#define LS_THREADS 256
#define LS_ROWS 4
#define LS_BLOCKS 1024
template <typename T, int GH>
__global__ __launch_bounds__(LS_THREADS) void lin_step_kernel(const LinGeom g, int cols, const int32_t* __restrict__ pos, const T* __restrict__ qkv, const float* state_in, float* state_out,
                                                              T* __restrict__ o) {
  extern __shared__ float sm[];  // k[d], q[GH][d], shares of o [groups][GH][cols]
  const int hk = blockIdx.y, b = blockIdx.z, d = g.d, grp = g.nq / g.nkv, per = cols / 4, groups = LS_THREADS / per, r = threadIdx.x / per, cl = threadIdx.x % per * 4, c = blockIdx.x * cols + cl;
  const int p = pos ? pos[b] : 1;
  if (p < 0) return;
  float *ks = sm, *qs = ks + d, *red = qs + GH * d;
  const float log_decay = g.log_decay[hk], lam = expf(log_decay);
  const bool begins = p == 0 || lin_alone(log_decay * 1.4426950408889634f);  // what state_in holds does not count
  const T* token = qkv + (size_t)b * (g.nq + 2 * g.nkv) * d;
  const T *k = token + (size_t)(g.nq + hk) * d, *v = k + (size_t)g.nkv * d;
  const size_t st = ((size_t)b * g.nkv + hk) * d * d + c;
  const bool on = r < groups;
  f32x4 v4 = {0.f, 0.f, 0.f, 0.f};
  if (on)
#pragma unroll
    for (int e = 0; e < 4; e++) v4[e] = to_f32(v[c + e]);
  for (int e = threadIdx.x; e < d; e += LS_THREADS) ks[e] = to_f32(k[e]);
  for (int h0 = 0; h0 < grp; h0 += GH) {
    const T* q = token + (size_t)(hk * grp + h0) * d;
    const int heads = min(GH, grp - h0);
    for (int e = threadIdx.x; e < GH * d; e += LS_THREADS) qs[e] = e < heads * d ? to_f32(q[e]) : 0.f;
    __syncthreads();
    f32x4 acc[GH];
#pragma unroll
    for (int h = 0; h < GH; h++) acc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (on) {
      const float* from = h0 == 0 ? state_in : state_out;
      for (int x0 = r; x0 < d; x0 += groups * LS_ROWS) {
        f32x4 S[LS_ROWS];
#pragma unroll
        for (int u = 0; u < LS_ROWS; u++) {
          const int x = x0 + u * groups;
          S[u] = x < d && (h0 > 0 || !begins) ? *reinterpret_cast<const f32x4*>(from + st + (size_t)x * d) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int u = 0; u < LS_ROWS; u++) {
          const int x = x0 + u * groups;
          if (x >= d) break;
          if (h0 == 0) {
#pragma unroll
            for (int e = 0; e < 4; e++) S[u][e] = fmaf(ks[x], v4[e], lam * S[u][e]);
            *reinterpret_cast<f32x4*>(state_out + st + (size_t)x * d) = S[u];
          }
#pragma unroll
          for (int h = 0; h < GH; h++) {
            const float qx = qs[h * d + x];
#pragma unroll
            for (int e = 0; e < 4; e++) acc[h][e] = fmaf(qx, S[u][e], acc[h][e]);
          }
        }
      }
#pragma unroll
      for (int h = 0; h < GH; h++) *reinterpret_cast<f32x4*>(red + (r * GH + h) * cols + cl) = acc[h];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < heads * cols; e += LS_THREADS) {
      float s = 0.f;
      for (int w = 0; w < groups; w++) s += red[w * GH * cols + e];
      o[((size_t)b * g.nq + hk * grp + h0 + e / cols) * d + blockIdx.x * cols + e % cols] = from_f32<T>(s * g.scale);
    }
  }
}

// ------------------------------------------------------------------------------------ host side
static size_t lin_ws_bytes(int dtype, const LinGeom& g, bool bwd) {
  if (!mix_sized(dtype, g.batch, g.seq, g.nq, g.nkv, g.d)) return 0;
  return dtype == DH_BF16 ? dh_linattn_bf16_ws_bytes(g, bwd) : dh_linattn_f32_ws_bytes(g, bwd);
}
extern "C" size_t dh_linattn_fwd_workspace_bytes(int dtype, int batch, int seq, int nq, int nkv, int d) {
  return lin_ws_bytes(dtype, {batch, seq, nq, nkv, d, 1.f, nullptr}, false);
}
extern "C" size_t dh_linattn_bwd_workspace_bytes(int dtype, int batch, int seq, int nq, int nkv, int d) {
  return lin_ws_bytes(dtype, {batch, seq, nq, nkv, d, 1.f, nullptr}, true);
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
  if (seq == 0) return state_out ? dh_launch_lin_carry(g, 0, 0, {nullptr, state_in, state_out, 0}, nullptr, s) : DH_OK;
  if (dtype == DH_BF16) return dh_launch_linattn_fwd_bf16(g, (const bf16_t*)qkv, state_in, (bf16_t*)o, state_out, ws, s);
  return dh_launch_linattn_fwd_f32(g, (const float*)qkv, state_in, (float*)o, state_out, ws, s);
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
  if (seq == 0) return dstate_in ? dh_launch_lin_carry(g, 0, 0, {nullptr, dstate_out, dstate_in, 0}, nullptr, s) : DH_OK;
  if (dtype == DH_BF16) return dh_launch_linattn_bwd_bf16(g, (const bf16_t*)qkv, state_in, (const bf16_t*)dout, dstate_out, (bf16_t*)dqkv, dstate_in, ws, s);
  return dh_launch_linattn_bwd_f32(g, (const float*)qkv, state_in, (const float*)dout, dstate_out, (float*)dqkv, dstate_in, ws, s);
}
template <typename T, int GH>
static void lin_step_launch(const LinGeom& g, const int32_t* pos, const T* qkv, const float* state_in, float* state_out, T* o, hipStream_t s) {
  int cols = g.d;
  while ((long long)g.batch * g.nkv * (g.d / cols) < LS_BLOCKS && cols % 8 == 0 && cols >= 64) cols /= 2;
  const size_t lds = (size_t)((1 + GH) * g.d + LS_THREADS / (cols / 4) * GH * cols) * sizeof(float);
  lin_step_kernel<T, GH><<<dim3(g.d / cols, g.nkv, g.batch), LS_THREADS, lds, s>>>(g, cols, pos, qkv, state_in, state_out, o);
}
template <typename T>
static void lin_step(const LinGeom& g, const int32_t* pos, const T* qkv, const float* state_in, float* state_out, T* o, hipStream_t s) {
  const int grp = g.nq / g.nkv;
  if (grp > 4) lin_step_launch<T, 8>(g, pos, qkv, state_in, state_out, o, s);
  else if (grp > 2) lin_step_launch<T, 4>(g, pos, qkv, state_in, state_out, o, s);
  else if (grp > 1) lin_step_launch<T, 2>(g, pos, qkv, state_in, state_out, o, s);
  else lin_step_launch<T, 1>(g, pos, qkv, state_in, state_out, o, s);
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
  if (dtype == DH_BF16) lin_step<bf16_t>(g, pos, (const bf16_t*)qkv, state_in, state_out, (bf16_t*)o, s);
  else lin_step<float>(g, pos, (const float*)qkv, state_in, state_out, (float*)o, s);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
