// float32 linear attention with a decay for each head, on the float32 matrix instruction (v_mfma_f32_32x32x2_f32), forward and backward: the chunks, pieces and passes of linattn_bf16.hip, with
// no rounding inside.
//
// A wave owns 32 columns of the state and of the results.  A result tile's register r holds rows 8 (r / 4) + r % 4 of one half of the wave and the row four further of the other, and the instruction's
// two k indexes may be any two rows: register r of the scores or of the state is an operand of the next product as it stands, beside the two rows of the other operand that it stands for.
// Bound by latency at the lengths of the float32 configuration: 64 tokens are two chunks.
#include <algorithm>
#include "linattn.h"

#define MFMA32(a, b, c) __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0)

// One pass: out_r = sum over tokens seen of f_score lambda^|r - j| (q_r k_j) v_j + f_read lambda^.. S^T q_r; S sums f_in lambda^.. k_j v_j^T.
struct Lin32Pass {
  const float *q, *k, *v;  // of the first head
  float* out;
  int ldq, ldk, ldv, ldo;
  const float* state;      // before each piece [batch][nkv][pieces][d][d], nullptr: zeros
  float* sum;              // sums alone: the pieces' contributions, likewise; otherwise the state at the end [batch][nkv][d][d] (or nullptr)
  int transposed;          // state and sum have their indexes exchanged
};
struct Lin32Args {
  LinGeom g;
  LinCut cut;
  Lin32Pass pass[3];
};
__device__ __forceinline__ int lin32_row(int r, int kg) { return 8 * (r >> 2) + 4 * kg + (r & 3); }

// GROUPED: the query rows are shared by the group's heads, whose keys and values are summed over (dk, dv and the states R); otherwise the other way round.  REV: from the row's end.
// OUT: results, otherwise the state's sums alone.  D: d rounded up to 32, 64 or 128; columns from d on are zeros.
template <int D, bool GROUPED, bool REV, bool OUT>
__device__ __forceinline__ void lin32_walk(const Lin32Args& a, const Lin32Pass& p, int piece, int hk, int b, float* sm) {
  constexpr int W = D / 32, LD = D + 1, TILE = LC * LD, VECS = LC * D / 4 / (W * 64);
  const LinGeom& g = a.g;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, kg = lane >> 5, d = g.d, grp = g.nq / g.nkv, col = wave * 32 + l32;
  const int chunks = (g.seq + LC - 1) / LC, c0 = piece * a.cut.per, c1 = min(chunks, c0 + a.cut.per), heads = GROUPED || OUT ? grp : 1, steps = (c1 - c0) * heads;
  const size_t t0 = (size_t)b * g.seq;
  const float l2 = g.log_decay[hk] * 1.4426950408889634f;
  const bool alone = lin_alone(l2);
  const float f_read = GROUPED ? 1.f : g.scale, f_in = GROUPED ? g.scale : 1.f;
  float *Qs = sm, *Ks = sm + TILE, *Vs = sm + 2 * TILE;
  auto chunk_of = [&](int n) { return REV ? c1 - 1 - n : c0 + n; };
  float4 nq[VECS], nk[VECS], nv[VECS];  // the next step's rows
  auto fetch1 = [&](float4 (&x)[VECS], const float* base, int ld, int head, int chunk) {
#pragma unroll
    for (int i = 0; i < VECS; i++) {
      const int e = (threadIdx.x + i * W * 64) * 4, row = e / D, c = e % D, t = chunk * LC + row;
      x[i] = t < g.seq && c < d ? *reinterpret_cast<const float4*>(base + (t0 + t) * ld + (size_t)head * d + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  };
  auto put = [&](float* to, const float4 (&x)[VECS]) {
#pragma unroll
    for (int i = 0; i < VECS; i++) {
      const int e = (threadIdx.x + i * W * 64) * 4;
      float* at = to + e / D * LD + e % D;
      at[0] = x[i].x; at[1] = x[i].y; at[2] = x[i].z; at[3] = x[i].w;
    }
  };
  auto fetch = [&](int n, int h) {
    const int chunk = chunk_of(n);
    if (OUT && (!GROUPED || h == 0)) fetch1(nq, p.q, p.ldq, GROUPED ? hk : hk * grp + h, chunk);
    if (GROUPED || h == 0) {
      fetch1(nk, p.k, p.ldk, GROUPED ? hk * grp + h : hk, chunk);
      fetch1(nv, p.v, p.ldv, GROUPED ? hk * grp + h : hk, chunk);
    }
  };
  fetch(0, 0);
  f32x16 S[W], ot;
  const size_t st = (((size_t)b * g.nkv + hk) * a.cut.pieces + piece) * d * d;
#pragma unroll
  for (int dt = 0; dt < W; dt++)
#pragma unroll
    for (int r = 0; r < 16; r++) {
      const int x = 32 * dt + lin32_row(r, kg);
      S[dt][r] = OUT && p.state && x < d && col < d && (GROUPED || !alone) ? p.state[st + (p.transposed ? (size_t)col * d + x : (size_t)x * d + col)] : 0.f;
    }
  float weight[OUT ? 16 : 1];
  if constexpr (OUT) {
#pragma unroll
    for (int r = 0; r < 16; r++) weight[r] = g.scale * lin_pow(l2, max(0, REV ? lin32_row(r, kg) - l32 : l32 - lin32_row(r, kg)));
  }
  const int lo = REV || alone ? l32 : 0, hi = !REV || alone ? l32 + 1 : LC;  // the tokens of a chunk that the lane's sees
  int n = 0, h = 0, left = 0;
  for (int s = 0; s < steps; s++) {
    const int chunk = chunk_of(n);
    left = min(LC, g.seq - chunk * LC);
    __syncthreads();  // every wave is done with the step before
    if (OUT && (!GROUPED || h == 0)) put(Qs, nq);
    if (GROUPED || h == 0) { put(Ks, nk); put(Vs, nv); }
    __syncthreads();
    if (s + 1 < steps) fetch(h + 1 == heads ? n + 1 : n, h + 1 == heads ? 0 : h + 1);
    float v[16];  // values of the 32 tokens in the wave's columns
#pragma unroll
    for (int r = 0; r < 16; r++) v[r] = Vs[lin32_row(r, kg) * LD + col];
    if constexpr (OUT) {
      const float* q = Qs + l32 * LD;
      f32x16 sc;
#pragma unroll
      for (int r = 0; r < 16; r++) sc[r] = 0.f;
      if (!GROUPED || h == 0) {
#pragma unroll
        for (int r = 0; r < 16; r++) ot[r] = 0.f;
      }
      const float* k = Ks + l32 * LD;
#pragma unroll
      for (int dt = 0; dt < W; dt++)
#pragma unroll
        for (int r = 0; r < 16; r++) {
          const int x = 32 * dt + lin32_row(r, kg);
          const float qx = q[x];
          sc = MFMA32(k[x], qx, sc);
          if (!GROUPED || h == 0) ot = MFMA32(S[dt][r], qx, ot);
        }
      if (!GROUPED || h == 0) {
        const float read = f_read * (REV ? l32 < left ? lin_pow(l2, left - 1 - l32) : 0.f : lin_pow(l2, l32 + 1));
        const bool none = GROUPED && alone && read == 0.f;
#pragma unroll
        for (int r = 0; r < 16; r++) ot[r] = none ? 0.f : ot[r] * read;
      }
      uint32_t odd = 0;  // bit r: register r's token of the lane's half holds an infinity or a NaN in some column of the wave: a zero times it would reach tokens that do not see it
#pragma unroll
      for (int r = 0; r < 16; r++) {
        const int j = lin32_row(r, kg);
        const bool seen = j >= lo && j < (REV ? min(hi, left) : hi);
        sc[r] = seen ? sc[r] * weight[r] : 0.f;
        odd |= __builtin_isfinite(v[r]) ? 0u : 1u << r;
      }
      if (!__any(odd != 0)) {
#pragma unroll
        for (int r = 0; r < 16; r++) ot = MFMA32(v[r], sc[r], ot);
      } else {
#pragma unroll
        for (int r = 0; r < 16; r++) {
          const uint64_t who = __ballot((odd >> r) & 1);
          const bool bad0 = (uint32_t)who != 0, bad1 = (who >> 32) != 0;
          ot = MFMA32((kg ? bad1 : bad0) ? 0.f : v[r], sc[r], ot);
#pragma unroll 1
          for (int half = 0; half < 2; half++) {  // such a token by itself, to those that see it
            if (!(half ? bad1 : bad0)) continue;
            f32x16 add;
#pragma unroll
            for (int x = 0; x < 16; x++) add[x] = 0.f;
            add = MFMA32(kg == half ? v[r] : 0.f, kg == half ? sc[r] : 0.f, add);
            const int j = lin32_row(r, half);
            const bool here = j >= lo && j < hi;
#pragma unroll
            for (int x = 0; x < 16; x++) ot[x] = here ? ot[x] + add[x] : ot[x];
          }
        }
      }
      if (!GROUPED || h == heads - 1) {
        float* row = p.out + (t0 + (size_t)chunk * LC + l32) * p.ldo + (size_t)(GROUPED ? hk : hk * grp + h) * d;
#pragma unroll
        for (int q4 = 0; q4 < 4; q4++) {
          const int c = wave * 32 + 8 * q4 + 4 * kg;
          if (l32 < left && c < d) *reinterpret_cast<f32x4*>(row + c) = f32x4{ot[4 * q4], ot[4 * q4 + 1], ot[4 * q4 + 2], ot[4 * q4 + 3]};
        }
      }
    }
    if ((GROUPED || h == heads - 1) && !(OUT && alone)) {  // (alone: it stays zero within the row)
      if (!GROUPED || h == 0) {
        const float f = lin_pow(l2, left);
#pragma unroll
        for (int dt = 0; dt < W; dt++)
#pragma unroll
          for (int r = 0; r < 16; r++) S[dt][r] *= f;
      }
#pragma unroll
      for (int r = 0; r < 16; r++) {  // rows behind the row's end are zeros
        const int j = lin32_row(r, kg);
        v[r] *= j < left ? f_in * lin_pow(l2, REV ? 1 + j : left - 1 - j) : 0.f;
      }
#pragma unroll
      for (int r = 0; r < 16; r++)
#pragma unroll
        for (int dt = 0; dt < W; dt++) S[dt] = MFMA32(Ks[lin32_row(r, kg) * LD + 32 * dt + l32], v[r], S[dt]);
    }
    if (++h == heads) {
      h = 0;
      n++;
      if (OUT && GROUPED && alone) {
#pragma unroll
        for (int dt = 0; dt < W; dt++)
#pragma unroll
          for (int r = 0; r < 16; r++) S[dt][r] = 0.f;
      }
    }
  }
  if (p.sum && alone) {  // the last token's k v^T, of R nothing
    float* to = p.sum + (OUT ? ((size_t)b * g.nkv + hk) * d * d : st);
    const float *k = Ks + (left - 1) * LD, *own = Vs + (left - 1) * LD;
#pragma unroll 1
    for (int e = threadIdx.x; e < d * d; e += 2 * D) to[e] = GROUPED ? 0.f : k[e / d] * own[e % d];
  } else if (p.sum) {
    float* to = p.sum + (OUT ? ((size_t)b * g.nkv + hk) * d * d : st);
#pragma unroll
    for (int dt = 0; dt < W; dt++)
#pragma unroll
      for (int r = 0; r < 16; r++) {
        const int x = 32 * dt + lin32_row(r, kg);
        if (x < d && col < d) to[(size_t)x * d + col] = S[dt][r];
      }
  }
}
// grid (pieces, nkv, batch)
template <int D, bool OUT>
__global__ __launch_bounds__(2 * D) void lin32_fwd_kernel(const Lin32Args a) {
  extern __shared__ float sm[];
  lin32_walk<D, false, false, OUT>(a, a.pass[0], blockIdx.x, blockIdx.y, blockIdx.z, sm);
}
// dk, dv and dq, or (!OUT) the sums for R and S.  grid (pieces, nkv * (OUT ? 3 : 2), batch)
template <int D, bool OUT>
__global__ __launch_bounds__(2 * D) void lin32_bwd_kernel(const Lin32Args a) {
  extern __shared__ float sm[];
  const int nkv = a.g.nkv, y = blockIdx.y;
  if (y < nkv) lin32_walk<D, true, true, OUT>(a, a.pass[0], blockIdx.x, y, blockIdx.z, sm);
  else if (y < 2 * nkv) lin32_walk<D, false, false, OUT>(a, a.pass[1], blockIdx.x, y - nkv, blockIdx.z, sm);
  else lin32_walk<D, true, true, OUT>(a, a.pass[2], blockIdx.x, y - 2 * nkv, blockIdx.z, sm);
}

// ------------------------------------------------------------------------------------ host side
// Pieces: two blocks of the forward pass for each unit of the chip, or one of each of the backward pass's three kinds, down to single chunks.  us, forward and backward, at this and at half of it: 2 x 2048
// tokens of 8:8 heads of 128 82 and 180, 73 and 202; 4 x 512 of 8:8 heads of 64 27 and 57, 29 and 50; 8192 of 4:4 42 and 82, 47 and 82.  Rows of up to three steps (a chunk of one head) stay whole, without the
// launches of sums and carry: 64 tokens of 4:4 14 and 14 whole, 17 and 21 cut; 96 19 and 20, 17 and 21; 128 25 and 25, 18 and 21.
static LinCut lin32_cut(const LinGeom& g, bool bwd) {
  const long long chunks = (g.seq + LC - 1) / LC, blocks = (long long)g.batch * g.nkv * (bwd ? 3 : 1);
  if (chunks * (g.nq / g.nkv) <= 3) return {1, (int)chunks};
  const long long want = std::max(1ll, std::min(((bwd ? 768 : 512) + blocks - 1) / blocks, chunks));
  const int per = (int)((chunks + want - 1) / want);
  return {(int)((chunks + per - 1) / per), per};
}
static size_t lin32_states(const LinGeom& g, int pieces) { return (size_t)g.batch * g.nkv * pieces * g.d * g.d; }
size_t dh_linattn_f32_ws_bytes(const LinGeom& g, bool bwd) {
  const LinCut c = lin32_cut(g, bwd);
  return c.pieces == 1 ? 0 : (bwd ? 2 : 1) * lin32_states(g, c.pieces) * sizeof(float);
}
template <int D>
static int lin32_fwd(const LinGeom& g, const float* qkv, const float* state_in, float* o, float* state_out, float* ws, hipStream_t s) {
  const int ld = (g.nq + 2 * g.nkv) * g.d;
  const size_t lds = 3 * LC * (D + 1) * sizeof(float);
  Lin32Args a = {g, lin32_cut(g, false), {}};
  a.pass[0] = {qkv, qkv + (size_t)g.nq * g.d, qkv + (size_t)(g.nq + g.nkv) * g.d, o, ld, ld, ld, g.nq * g.d, state_in, state_out, 0};
  const dim3 grid(a.cut.pieces, g.nkv, g.batch);
  if (a.cut.pieces > 1) {
    Lin32Args f = a;
    f.pass[0].sum = ws;
    lin32_fwd_kernel<D, false><<<grid, 2 * D, lds, s>>>(f);
    DH_LAUNCH_CHECK();
    if (int rc = dh_launch_lin_carry(g, a.cut.pieces, a.cut.per * LC, {ws, state_in, state_out, 0}, nullptr, s)) return rc;
    a.pass[0].state = ws;
    a.pass[0].sum = nullptr;
  }
  lin32_fwd_kernel<D, true><<<grid, 2 * D, lds, s>>>(a);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
int dh_launch_linattn_fwd_f32(const LinGeom& g, const float* qkv, const float* state_in, float* o, float* state_out, void* ws, hipStream_t s) {
  if (g.d <= 32) return lin32_fwd<32>(g, qkv, state_in, o, state_out, (float*)ws, s);
  if (g.d <= 64) return lin32_fwd<64>(g, qkv, state_in, o, state_out, (float*)ws, s);
  return lin32_fwd<128>(g, qkv, state_in, o, state_out, (float*)ws, s);
}
template <int D>
static int lin32_bwd(const LinGeom& g, const float* qkv, const float* state_in, const float* dout, const float* dstate_out, float* dqkv, float* dstate_in, float* ws, hipStream_t s) {
  const int ld = (g.nq + 2 * g.nkv) * g.d, ldo = g.nq * g.d;
  const size_t kc = (size_t)g.nq * g.d, vc = kc + (size_t)g.nkv * g.d, lds = 3 * LC * (D + 1) * sizeof(float);
  const float *q = qkv, *k = qkv + kc, *v = qkv + vc;
  Lin32Args a = {g, lin32_cut(g, true), {}};
  a.pass[0] = {k, q, dout, dqkv + vc, ld, ld, ldo, ld, dstate_out, dstate_in, 0};
  a.pass[1] = {dout, v, k, dqkv, ldo, ld, ld, ld, state_in, nullptr, 1};
  a.pass[2] = {v, dout, q, dqkv + kc, ld, ldo, ld, ld, dstate_out, nullptr, 1};
  if (a.cut.pieces > 1) {
    float* R = ws + lin32_states(g, a.cut.pieces);
    Lin32Args f = a;
    f.pass[0].sum = R;
    f.pass[1] = {nullptr, k, v, nullptr, 0, ld, ld, 0, nullptr, ws, 0};
    lin32_bwd_kernel<D, false><<<dim3(a.cut.pieces, g.nkv * 2, g.batch), 2 * D, lds, s>>>(f);
    DH_LAUNCH_CHECK();
    const LinCarry back = {R, dstate_out, dstate_in, 1};
    if (int rc = dh_launch_lin_carry(g, a.cut.pieces, a.cut.per * LC, {ws, state_in, nullptr, 0}, &back, s)) return rc;
    a.pass[0].state = a.pass[2].state = R;
    a.pass[0].sum = nullptr;
    a.pass[1].state = ws;
  }
  lin32_bwd_kernel<D, true><<<dim3(a.cut.pieces, g.nkv * 3, g.batch), 2 * D, lds, s>>>(a);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
int dh_launch_linattn_bwd_f32(const LinGeom& g, const float* qkv, const float* state_in, const float* dout, const float* dstate_out, float* dqkv, float* dstate_in, void* ws, hipStream_t s) {
  if (g.d <= 32) return lin32_bwd<32>(g, qkv, state_in, dout, dstate_out, dqkv, dstate_in, (float*)ws, s);
  if (g.d <= 64) return lin32_bwd<64>(g, qkv, state_in, dout, dstate_out, dqkv, dstate_in, (float*)ws, s);
  return lin32_bwd<128>(g, qkv, state_in, dout, dstate_out, dqkv, dstate_in, (float*)ws, s);
}
