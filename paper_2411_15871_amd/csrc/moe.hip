// Mixture-of-experts operators (paper Sec. 6.1: top-2 gating; Table 2: Router, Permute, AlltoAll,
// Group-GEMM): router, stable permutation plan, row gathers (permute, all-to-all stand-in), weighted
// combine and their backward forms.  All index work is integer and deterministic: rows are grouped by
// expert with a stable counting sort (expert ascending, then token, then k), nothing uses atomics.
#include <algorithm>
#include "common.h"

// ------------------------------------------------------------------------------------ router (M1)
// One thread per token.  Top-2 by logit, ties to the lower expert id; the two kept probabilities are the
// softmax over the two kept logits: p0 = 1/(1+exp(l1-l0)), p1 = 1-p0 computed as exp(l1-l0)/(1+exp(l1-l0)).
__global__ void moe_route_kernel(int T, int E, const float* __restrict__ logits, int32_t* __restrict__ idx,
                                 float* __restrict__ prob) {
  int t = blockIdx.x * blockDim.x + threadIdx.x;
  if (t >= T) return;
  const float* l = logits + (size_t)t * E;
  int i0 = 0, i1 = -1;
  float v0 = l[0], v1 = -INFINITY;
  for (int e = 1; e < E; e++) {
    float v = l[e];
    if (v > v0) { i1 = i0; v1 = v0; i0 = e; v0 = v; }
    else if (v > v1) { i1 = e; v1 = v; }
  }
  if (i1 < 0) {  // every other logit is minus infinity or a NaN: the lowest other expert, so that the tables stay in range
    i1 = i0 == 0 ? 1 : 0;
    v1 = l[i1];
  }
  float d = expf(v1 - v0);
  idx[2 * t] = i0;
  idx[2 * t + 1] = i1;
  prob[2 * t] = 1.0f / (1.0f + d);
  prob[2 * t + 1] = d / (1.0f + d);
}

// dlogits[t,e] = p_k (dp_k - sum_j p_j dp_j) for the two kept experts, 0 elsewhere.  A thread per element (one per token, storing E
// elements apart from its neighbours': 1500 tokens of 16 experts 3.9 us, now 2.6), up to the grid of ROUTE_BWD_BLOCKS: T * E may exceed the 2^32 - 1
// threads a launch can have (2^24 tokens of 256 experts).
#define ROUTE_BWD_BLOCKS (1u << 20)
__global__ void moe_route_bwd_kernel(int T, int E, const float* __restrict__ dprob, const int32_t* __restrict__ idx,
                                     const float* __restrict__ prob, float* __restrict__ dlogits) {
  const size_t n = (size_t)T * E, stride = (size_t)gridDim.x * blockDim.x;
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += stride) {
    const size_t t = i / E;
    const int e = (int)(i - t * E);
    const float p0 = prob[2 * t], p1 = prob[2 * t + 1], g0 = dprob[2 * t], g1 = dprob[2 * t + 1];
    const int i0 = idx[2 * t], i1 = idx[2 * t + 1];
    const float s = p0 * g0 + p1 * g1;
    dlogits[i] = e == i1 ? p1 * (g1 - s) : e == i0 ? p0 * (g0 - s) : 0.f;
  }
}

// ------------------------------------------------------------------------------------ balance loss, z loss, rows per expert
// A group of L lanes works on a token, NE logits a lane, so that a wave reads 64/L consecutive rows at once: VEC: four consecutive experts a lane in one load (E and
// the address allow it), otherwise expert = lane of the group + L * i.  A lane's experts are the same for all its tokens: it adds their probabilities in registers,
// and the block's lanes meet in LDS once at the end, in order.  The counts are integers added in LDS, in any order.  Each block leaves its sums in the
// workspace: [blocks][E] probabilities, [blocks][E] counts, [blocks] z; a block that is alone goes on to the results.  Bound by memory where there are many tokens: BAL_TOKENS
// rows a group are in flight (65536 x 256: 17.8 us, 3.8 TB/s).
#define BAL_THREADS 1024
#define BAL_BLOCKS 256
#define BAL_TOKENS 4
__device__ __forceinline__ int live_tokens(const int32_t* n_live, int T) { return n_live ? min(max(*n_live, 0), T) : T; }
// exp of a number below one by the hardware's exponential of 2: the rounding of its exponent h, up to 2^-24 |x|, is made good by the remainder x - h log 2.  Off by three half steps
// and 2^-29 |h|.  (With expf the forward pass over 65536 x 256 was bound by its arithmetic, 21 us.)  Below -150 it is zero.
__device__ __forceinline__ float bal_exp(float x) {
  x = __builtin_elementwise_maximum(x, -150.f);
  const float h = x * 1.4426950408889634f, e = __builtin_amdgcn_exp2f(h);
  return fmaf(e, fmaf(h, -0.6931471805599453f, x), e);
}
template <int L, bool VEC> __device__ __forceinline__ int bal_expert(int el, int i) { return VEC ? el * 4 + i : el + L * i; }
// A lane's logits of the row at l; -inf beyond E.
template <int L, int NE, bool VEC>
__device__ __forceinline__ void bal_load(float (&v)[NE], const float* l, int el, int E) {
  if constexpr (VEC) {
    static_assert(NE == 4, "one load");
    const bool on = el * 4 < E;
    const f32x4 x = *reinterpret_cast<const f32x4*>(l + (on ? el * 4 : 0));
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = on ? x[i] : -INFINITY;
  } else {
#pragma unroll
    for (int i = 0; i < NE; i++) v[i] = el + L * i < E ? l[el + L * i] : -INFINITY;
  }
}
// counts, prob_mean and, behind a barrier, E sum f P of experts [e0, e1) from their sums, thread e - e0 for expert e; terms: 256 floats of LDS.
__device__ __forceinline__ float bal_result(int e0, int e1, int E, int N, float p, int n, float* terms, int32_t* counts, float* prob_mean) {
  const float inv = N > 0 ? 1.f / (float)N : 0.f;
  const int e = e0 + threadIdx.x;
  if (e < e1) {
    counts[e] = n;
    prob_mean[e] = p * inv;
    terms[threadIdx.x] = (float)n * (0.5f * inv) * (p * inv);
  }
  __syncthreads();
  float b = 0.f;
  for (int k = threadIdx.x & 63; k < e1 - e0; k += 64) b += terms[k];
  return (float)E * wave_sum(b);
}
template <int L, int NE, bool VEC>
__global__ __launch_bounds__(BAL_THREADS) void moe_balance_kernel(int T, int E, const float* __restrict__ logits, const int32_t* __restrict__ idx, const int32_t* __restrict__ n_live,
                                                                  float* __restrict__ lse, float* __restrict__ part_p, int32_t* __restrict__ part_n, float* __restrict__ part_z,
                                                                  int* __restrict__ done, int32_t* __restrict__ counts, float* __restrict__ prob_mean, float* __restrict__ loss) {
  constexpr int GROUPS = BAL_THREADS / L;
  __shared__ float sums[BAL_THREADS / 64 * L * NE], zs[BAL_THREADS / 64], fp[256];
  __shared__ int hist[256];
  const int N = live_tokens(n_live, T), el = threadIdx.x % L;
  if (threadIdx.x < 256) hist[threadIdx.x] = 0;
  __syncthreads();
  for (size_t i = (size_t)blockIdx.x * BAL_THREADS + threadIdx.x; i < 2 * (size_t)N; i += (size_t)gridDim.x * BAL_THREADS) {
    const int e = idx[i];
    if (e >= 0 && e < E) atomicAdd(&hist[e], 1);
  }
  double p[NE], z = 0.0;  // a lane adds up to a few thousand tokens: BAL_TOKENS of them in float32, these in float64
#pragma unroll
  for (int i = 0; i < NE; i++) p[i] = 0.0;
  // whole waves go round together: a group without a token repeats the last one and does not count it
  const size_t stride = (size_t)gridDim.x * GROUPS;
  for (size_t t0 = (size_t)blockIdx.x * GROUPS + (threadIdx.x & ~63) / L; t0 < (size_t)N; t0 += stride * BAL_TOKENS) {
    float v[BAL_TOKENS][NE];
#pragma unroll
    for (int k = 0; k < BAL_TOKENS; k++) {
      const size_t want = t0 + k * stride + (threadIdx.x & 63) / L;
      bal_load<L, NE, VEC>(v[k], logits + (want < (size_t)N ? want : N - 1) * E, el, E);
    }
    // the rows' maxima and sums side by side: a step across lanes takes longer than its arithmetic
    float m[BAL_TOKENS], sum[BAL_TOKENS];
#pragma unroll
    for (int k = 0; k < BAL_TOKENS; k++) {
      m[k] = v[k][0];
#pragma unroll
      for (int i = 1; i < NE; i++) m[k] = fmaxf(m[k], v[k][i]);
    }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < BAL_TOKENS; k++) m[k] = fmaxf(m[k], __shfl_xor(m[k], o, 64));
#pragma unroll
    for (int k = 0; k < BAL_TOKENS; k++) {
      m[k] = m[k] == -INFINITY ? 0.f : m[k];
      sum[k] = 0.f;
#pragma unroll
      for (int i = 0; i < NE; i++) { v[k][i] = bal_exp(v[k][i] - m[k]); sum[k] += v[k][i]; }
    }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < BAL_TOKENS; k++) sum[k] += __shfl_xor(sum[k], o, 64);
    float share[NE], zs4 = 0.f;
#pragma unroll
    for (int i = 0; i < NE; i++) share[i] = 0.f;
#pragma unroll
    for (int k = 0; k < BAL_TOKENS; k++) {
      const size_t t = t0 + k * stride + (threadIdx.x & 63) / L;
      const float l = fmaf(__builtin_amdgcn_logf(sum[k]), 0.69314718055994531f, m[k]), inv = t < (size_t)N && sum[k] != 0.f ? 1.f / sum[k] : 0.f;
#pragma unroll
      for (int i = 0; i < NE; i++) share[i] = fmaf(v[k][i], inv, share[i]);
      if (el == 0 && t < (size_t)N) {
        lse[t] = l;
        zs4 = sum[k] == 0.f ? zs4 : fmaf(l, l, zs4);
      }
    }
#pragma unroll
    for (int i = 0; i < NE; i++) p[i] += (double)share[i];
    z += (double)zs4;
  }
  // the wave's groups in float32
  float q[NE];
#pragma unroll
  for (int i = 0; i < NE; i++) q[i] = (float)p[i];
#pragma unroll
  for (int o = L; o < 64; o <<= 1) {
#pragma unroll
    for (int i = 0; i < NE; i++) q[i] += __shfl_xor(q[i], o, 64);
  }
  const float zw = wave_sum(el == 0 ? (float)z : 0.f);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) < L) {
#pragma unroll
    for (int i = 0; i < NE; i++) sums[wave * (L * NE) + bal_expert<L, VEC>(el, i)] = q[i];
  }
  if ((threadIdx.x & 63) == 0) zs[wave] = zw;
  __syncthreads();
  // the 16 waves' sums, in pairs of pairs
  auto waves = [](const float* of, int step) {
    float x[BAL_THREADS / 64];
#pragma unroll
    for (int w = 0; w < BAL_THREADS / 64; w++) x[w] = of[w * step];
#pragma unroll
    for (int n = BAL_THREADS / 128; n > 0; n /= 2)
#pragma unroll
      for (int w = 0; w < n; w++) x[w] += x[w + n];
    return x[0];
  };
  const float pe = (int)threadIdx.x < L * NE ? waves(sums + threadIdx.x, L * NE) : 0.f, ze = waves(zs, 1);
  const int e = threadIdx.x;
  if (gridDim.x == 1) {
    const float b = bal_result(0, E, E, N, pe, e < E ? hist[e] : 0, fp, counts, prob_mean);
    if (e == 0) {
      loss[0] = b;
      loss[1] = N > 0 ? ze / (float)N : 0.f;
    }
    return;
  }
  if (blockIdx.x == 0 && e == 0) *done = 0;  // for the launch behind
  if (e < E) {
    part_p[(size_t)blockIdx.x * E + e] = pe;
    part_n[(size_t)blockIdx.x * E + e] = hist[e];
  }
  if (threadIdx.x == 0) part_z[blockIdx.x] = ze;
}
// A block adds the blocks' sums of 16 experts, in 16 slices of the blocks, in order; the last block to end adds the experts' terms, in order.  (One block for all experts
// fetches 256 x 256 sums in 11 us.)
#define BAL_FINISH 16
__global__ __launch_bounds__(256) void moe_balance_finish_kernel(int T, int E, int blocks, const int32_t* __restrict__ n_live, const float* __restrict__ part_p,
                                                                 const int32_t* __restrict__ part_n, const float* __restrict__ part_z, int* __restrict__ done, float* __restrict__ part_b,
                                                                 int32_t* __restrict__ counts, float* __restrict__ prob_mean, float* __restrict__ loss) {
  __shared__ double ps[256], zz[4];
  __shared__ float terms[BAL_FINISH];
  __shared__ int ns[256], last;
  const int N = live_tokens(n_live, T), e0 = blockIdx.x * BAL_FINISH, e1 = min(E, e0 + BAL_FINISH), c = threadIdx.x % BAL_FINISH, slice = threadIdx.x / BAL_FINISH;
  double p = 0.0;
  float x[BAL_BLOCKS / BAL_FINISH];
  int n = 0, y[BAL_BLOCKS / BAL_FINISH];
  const int per = (blocks + 15) / 16, b0 = slice * per, e = min(e0 + c, E - 1);
#pragma unroll
  for (int u = 0; u < BAL_BLOCKS / 16; u++) {
    const size_t at = (size_t)min(b0 + u, blocks - 1) * E + e;
    x[u] = part_p[at];
    y[u] = part_n[at];
  }
#pragma unroll
  for (int u = 0; u < BAL_BLOCKS / 16; u++)
    if (u < per && b0 + u < blocks) { p += (double)x[u]; n += y[u]; }
  ps[threadIdx.x] = p;
  ns[threadIdx.x] = n;
  __syncthreads();
  p = 0.0;
  n = 0;
  if (threadIdx.x < BAL_FINISH) {
#pragma unroll
    for (int k = 0; k < 16; k++) { p += ps[k * BAL_FINISH + threadIdx.x]; n += ns[k * BAL_FINISH + threadIdx.x]; }
  }
  const float b = bal_result(e0, e1, E, N, (float)p, n, terms, counts, prob_mean);
  if (threadIdx.x == 0) {
    part_b[blockIdx.x] = b;
    __threadfence();
    last = atomicAdd(done, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double z = (int)threadIdx.x < blocks ? (double)part_z[threadIdx.x] : 0.0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o, 64);
  if ((threadIdx.x & 63) == 0) zz[threadIdx.x >> 6] = z;
  __syncthreads();
  if (threadIdx.x == 0) {
    float sum = 0.f;
    for (unsigned k = 0; k < gridDim.x; k++) sum += __hip_atomic_load(part_b + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    loss[0] = sum;
    loss[1] = N > 0 ? (float)((zz[0] + zz[1] + zz[2] + zz[3]) / (double)N) : 0.f;
  }
}
// dlogits, in the groups of the forward pass: one read and one write of the logits' size.  Probabilities are exponentials of the logits less the whole number next to lse, over their own sum:
// logits less lse itself would be off by its rounding and by their difference's.
template <int L, int NE, bool VEC>
__global__ __launch_bounds__(256) void moe_balance_bwd_kernel(int T, int E, const float* __restrict__ logits, const float* __restrict__ lse, const int32_t* __restrict__ counts,
                                                              const int32_t* __restrict__ n_live, const float* __restrict__ dloss, int accumulate, float* __restrict__ dlogits) {
  constexpr int GROUPS = 256 / L;
  const int N = live_tokens(n_live, T), el = threadIdx.x % L;
  const float inv = N > 0 ? 1.f / (float)N : 0.f, gb = dloss[0] * (float)E * inv, gz = dloss[1] * 2.f * inv;
  float f[NE];
#pragma unroll
  for (int i = 0; i < NE; i++) {
    const int e = bal_expert<L, VEC>(el, i);
    f[i] = e < E ? (float)counts[e] * (0.5f * inv) : 0.f;
  }
  for (size_t t0 = (size_t)blockIdx.x * GROUPS + (threadIdx.x & ~63) / L; t0 < (size_t)T; t0 += (size_t)gridDim.x * GROUPS) {
    const size_t t = t0 + (threadIdx.x & 63) / L;
    const bool live = t < (size_t)N;
    const float l = live ? lse[t] : 0.f;
    const float near = rintf(l);
    float p[NE], s = 0.f, sum = 0.f;
    bal_load<L, NE, VEC>(p, logits + (t < (size_t)T ? t : T - 1) * E, el, E);
#pragma unroll
    for (int i = 0; i < NE; i++) {
      p[i] = live && l != -INFINITY && bal_expert<L, VEC>(el, i) < E ? bal_exp(p[i] - near) : 0.f;
      sum += p[i];
      s = fmaf(p[i], f[i], s);
    }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) {
      sum += __shfl_xor(sum, o, 64);
      s += __shfl_xor(s, o, 64);
    }
    const float r = live && l != -INFINITY ? 1.f / sum : 0.f;
    s *= r;
    if (t < (size_t)T && (live || !accumulate)) {
      float g[NE];
#pragma unroll
      for (int i = 0; i < NE; i++) g[i] = live && l != -INFINITY ? p[i] * r * fmaf(gb, f[i] - s, gz * l) : 0.f;
      float* to = dlogits + t * E;
      if constexpr (VEC) {
        if (el * 4 < E) {
          f32x4* q = reinterpret_cast<f32x4*>(to + el * 4);
          const f32x4 x = {g[0], g[1], g[2], g[3]};
          *q = accumulate ? *q + x : x;
        }
      } else {
#pragma unroll
        for (int i = 0; i < NE; i++)
          if (el + L * i < E) to[el + L * i] = accumulate ? to[el + L * i] + g[i] : g[i];
      }
    }
  }
}

// ------------------------------------------------------------------------------------ permutation plan (M2, M3)
// Block e ranks the assignments (a = 2t+k, ascending) that chose expert e: a wave owns a contiguous sixteenth of them, 64 at a time, counts its
// matches from the lanes' votes, and hands out ranks behind those of the waves before it.  Bound by two rounds of loads (8192 assignments: a
// thread for each 256th of them, one load after the other, took 13 us, now 4.6).
#define RANK_WAVES 16
__global__ __launch_bounds__(64 * RANK_WAVES) void moe_rank_kernel(int n_assign, const int32_t* __restrict__ idx, int32_t* __restrict__ rank,
                                                                   int32_t* __restrict__ counts) {
  __shared__ int part[RANK_WAVES];
  const int e = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = ((n_assign + RANK_WAVES - 1) / RANK_WAVES + 63) / 64 * 64, a0 = min(n_assign, wave * per), a1 = min(n_assign, a0 + per);
  int count = 0;
  for (int a = a0; a < a1; a += 64 * 8) {
    int v[8];
#pragma unroll
    for (int u = 0; u < 8; u++) v[u] = a + u * 64 + lane < a1 ? idx[a + u * 64 + lane] : -1;
#pragma unroll
    for (int u = 0; u < 8; u++) count += __popcll(__ballot(v[u] == e));
  }
  if (lane == 0) part[wave] = count;
  __syncthreads();
  int r = 0;
  for (int w = 0; w < wave; w++) r += part[w];
  for (int a = a0; a < a1; a += 64 * 8) {
    int v[8];
#pragma unroll
    for (int u = 0; u < 8; u++) v[u] = a + u * 64 + lane < a1 ? idx[a + u * 64 + lane] : -1;
#pragma unroll
    for (int u = 0; u < 8; u++) {
      const unsigned long long who = __ballot(v[u] == e);
      if (v[u] == e) rank[a + u * 64 + lane] = r + __popcll(who & ((1ull << lane) - 1));
      r += __popcll(who);
    }
  }
  if (wave == RANK_WAVES - 1 && lane == 0) counts[e] = r;
}

// Sum of the values of the threads before this one, over a block of 256; `part`: 4 ints.  Ends in a barrier.
__device__ __forceinline__ int block256_before(int v, int* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int t = __shfl_up(upto, d, 64);
    if (lane >= d) upto += t;
  }
  if (lane == 63) part[wave] = upto;
  __syncthreads();
  for (int w = 0; w < wave; w++) upto += part[w];
  __syncthreads();
  return upto - v;
}

// Prefix sums over the experts (every block for itself, thread e for expert e): offsets[e] = first send row of expert e (send order = expert
// ascending); recv_start[e] = first receive row of expert e (receive order = [local expert][source rank], logical expert
// e = source*n_local + local); group_rows[le] = rows of local expert le.  Then, with r = rank[a]: dest[a] = send row of assignment a;
// src_tok[row] = its token; send_of_recv[j] = send row copied to receive row j; recv_of_send = the inverse.  (The prefix sums as a launch of one
// thread took 2.6-4.5 us and a gap; in here they take 0.8.)
__global__ __launch_bounds__(256) void moe_tables_kernel(int n_assign, int E, int n_local, const int32_t* __restrict__ idx, const int32_t* __restrict__ rank,
                                                         const int32_t* __restrict__ counts, int32_t* __restrict__ offsets,
                                                         int32_t* __restrict__ recv_start, int32_t* __restrict__ group_rows,
                                                         int32_t* __restrict__ dest, int32_t* __restrict__ src_tok,
                                                         int32_t* __restrict__ send_of_recv, int32_t* __restrict__ recv_of_send) {
  __shared__ int send0[257], recv0[257], part[4];
  const int tid = threadIdx.x, a = blockIdx.x * 256 + tid, src = E / n_local;
  const int e = a < n_assign ? idx[a] : 0, r = a < n_assign ? rank[a] : 0;
  // thread p: expert p of the send order, and the p-th expert of the receive order
  const int pe = tid < E ? tid % src * n_local + tid / src : 0;
  const int c = tid < E ? counts[tid] : 0, pc = tid < E ? counts[pe] : 0;
  const int before = block256_before(c, part), pbefore = block256_before(pc, part);
  if (tid < E) { send0[tid] = before; recv0[pe] = pbefore; }
  if (tid == E - 1) send0[E] = before + c;
  __syncthreads();
  if (blockIdx.x == 0) {
    if (tid < E) { offsets[tid] = send0[tid]; recv_start[tid] = recv0[tid]; }
    if (tid == 0) offsets[E] = send0[E];
    if (tid < n_local) group_rows[tid] = (tid + 1 < n_local ? recv0[tid + 1] : send0[E]) - recv0[tid];  // local expert tid begins with source 0
  }
  if (a >= n_assign) return;
  const int row = send0[e] + r, rr = recv0[e] + r;
  dest[a] = row;
  src_tok[row] = a >> 1;
  send_of_recv[rr] = row;
  recv_of_send[row] = rr;
}

// ------------------------------------------------------------------------------------ row movement
// out[r,:] = in[map[r],:]  (token permute, all-to-all stand-in in both directions).  One wave per row chunk.
// Bound by memory (8192 rows of 8 KiB: 21 us, 6.4 TB/s), so two movements one behind the other are one where they may be:
// via != nullptr takes row map[via[r]].
template <typename T>
__global__ __launch_bounds__(256) void gather_rows_kernel(int n_rows, int H, const T* __restrict__ in, const int32_t* __restrict__ map,
                                                          const int32_t* __restrict__ via, T* __restrict__ out) {
  const int chunks = H / 8;
  const size_t total = (size_t)n_rows * chunks, stride = (size_t)gridDim.x * blockDim.x;
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += stride) {
    const size_t r = i / chunks;
    const int c = (int)(i % chunks) * 8;
    Vec8<T> v;
    v.load(in + (size_t)map[via ? via[r] : r] * H + c);
    v.store(out + r * H + c);
  }
}

// y[t,:] = w0*yp[dest[t,0],:] + w1*yp[dest[t,1],:] (+ res[t,:]); weights = prob[t,:] or 1 when prob == nullptr.
// via != nullptr: yp's rows lie in another order, row d at via[d].
template <typename T>
__global__ __launch_bounds__(256) void combine_kernel(int Ttok, int H, const T* __restrict__ yp, const int32_t* __restrict__ dest, const int32_t* __restrict__ via,
                                                      const float* __restrict__ prob, const T* __restrict__ res, T* __restrict__ y) {
  const int chunks = H / 8;
  const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= (size_t)Ttok * chunks) return;
  const size_t t = i / chunks;
  const int c = (int)(i % chunks) * 8;
  const float w0 = prob ? prob[2 * t] : 1.f, w1 = prob ? prob[2 * t + 1] : 1.f;
  Vec8<T> a, b;
  int r0 = dest[2 * t], r1 = dest[2 * t + 1];
  if (via != nullptr) { r0 = via[r0]; r1 = via[r1]; }
  a.load(yp + (size_t)r0 * H + c);
  b.load(yp + (size_t)r1 * H + c);
#pragma unroll
  for (int k = 0; k < 8; k++) a.v[k] = w0 * a.v[k] + w1 * b.v[k];
  if (res != nullptr) {
    b.load(res + t * H + c);
#pragma unroll
    for (int k = 0; k < 8; k++) a.v[k] += b.v[k];
  }
  a.store(y + t * H + c);
}

// Backward of the weighted combine: dyp[dest[t,k],:] = prob[t,k]*dy[t,:]; dprob[t,k] = <dy[t,:], yp[dest[t,k],:]>.
// One 256-thread block per token.
template <typename T>
__global__ __launch_bounds__(256) void combine_bwd_kernel(int H, const T* __restrict__ dy, const T* __restrict__ yp,
                                                          const int32_t* __restrict__ dest, const float* __restrict__ prob,
                                                          T* __restrict__ dyp, float* __restrict__ dprob) {
  __shared__ float red[8];
  const size_t t = blockIdx.x;
  const int r0 = dest[2 * t], r1 = dest[2 * t + 1];
  const float p0 = prob[2 * t], p1 = prob[2 * t + 1];
  float d0 = 0.f, d1 = 0.f;
  for (int c = threadIdx.x * 8; c < H; c += 256 * 8) {
    Vec8<T> g, a, b, o0, o1;
    g.load(dy + t * H + c);
    a.load(yp + (size_t)r0 * H + c);
    b.load(yp + (size_t)r1 * H + c);
#pragma unroll
    for (int k = 0; k < 8; k++) {
      d0 += g.v[k] * a.v[k];
      d1 += g.v[k] * b.v[k];
      o0.v[k] = p0 * g.v[k];
      o1.v[k] = p1 * g.v[k];
    }
    o0.store(dyp + (size_t)r0 * H + c);
    o1.store(dyp + (size_t)r1 * H + c);
  }
  d0 = block256_sum(d0, red);
  d1 = block256_sum(d1, red);
  if (threadIdx.x == 0) { dprob[2 * t] = d0; dprob[2 * t + 1] = d1; }
}

// ------------------------------------------------------------------------------------ host side
extern "C" int dh_moe_route(int T, int E, const float* logits, int32_t* idx, float* prob, void* stream) {
  if (T < 0 || E < 2 || E > 256) DH_FAIL(DH_ERR_SHAPE, "moe_route: T=%d E=%d (E must be 2..256)", T, E);
  if (T == 0) return DH_OK;
  if (!logits || !idx || !prob) DH_FAIL(DH_ERR_INVALID_ARG, "moe_route: null pointer");
  moe_route_kernel<<<(T + 255) / 256, 256, 0, (hipStream_t)stream>>>(T, E, logits, idx, prob);
  DH_LAUNCH_CHECK();
  return DH_OK;
}

extern "C" int dh_moe_route_bwd(int T, int E, const float* dprob, const int32_t* idx, const float* prob, float* dlogits,
                                void* stream) {
  if (T < 0 || E < 2 || E > 256) DH_FAIL(DH_ERR_SHAPE, "moe_route_bwd: T=%d E=%d (E must be 2..256)", T, E);
  if (T == 0) return DH_OK;
  if (!dprob || !idx || !prob || !dlogits) DH_FAIL(DH_ERR_INVALID_ARG, "moe_route_bwd: null pointer");
  moe_route_bwd_kernel<<<(unsigned)std::min<size_t>(((size_t)T * E + 255) / 256, ROUTE_BWD_BLOCKS), 256, 0, (hipStream_t)stream>>>(T, E, dprob, idx, prob, dlogits);
  DH_LAUNCH_CHECK();
  return DH_OK;
}

// GO(L, NE, VEC) for E experts: four experts a lane where rows of logits allow 16-byte loads; otherwise as many lanes as experts (a power of two), 64 with several
// logits a lane.
#define BALANCE_FOR(E, VEC, GO)                                                       \
  do {                                                                                \
    if (VEC) {                                                                        \
      if ((E) <= 4) GO(1, 4, true);                                                   \
      else if ((E) <= 8) GO(2, 4, true);                                              \
      else if ((E) <= 16) GO(4, 4, true);                                             \
      else if ((E) <= 32) GO(8, 4, true);                                             \
      else if ((E) <= 64) GO(16, 4, true);                                            \
      else if ((E) <= 128) GO(32, 4, true);                                           \
      else GO(64, 4, true);                                                           \
    } else if ((E) <= 2) GO(2, 1, false);                                             \
    else if ((E) <= 4) GO(4, 1, false);                                               \
    else if ((E) <= 8) GO(8, 1, false);                                               \
    else if ((E) <= 16) GO(16, 1, false);                                             \
    else if ((E) <= 32) GO(32, 1, false);                                             \
    else if ((E) <= 64) GO(64, 1, false);                                             \
    else if ((E) <= 128) GO(64, 2, false);                                            \
    else GO(64, 4, false);                                                            \
  } while (0)
static int balance_lanes(int E, bool vec) {  // of a group, as above
  int l = vec ? 1 : 2;
  while (l * (vec ? 4 : 1) < E && l < 64) l *= 2;
  return l;
}
static bool balance_vec(int E, const void* a, const void* b) { return E % 4 == 0 && (((uintptr_t)a | (uintptr_t)b) & 15) == 0; }
// Blocks of the forward launch: one up to BAL_ALONE rounds of its groups (it goes on to the results: 1500 x 16, 6 rounds, 10.1 us by several blocks and 7.9 by one; 4000 x 16, 16
// rounds, 10.8 and 13.2), else two rounds a block.
#define BAL_ALONE 8
static int balance_blocks(int T, int E, bool vec) {
  const size_t groups = BAL_THREADS / balance_lanes(E, vec), rounds = ((size_t)T + groups - 1) / groups;
  return rounds <= BAL_ALONE ? 1 : (int)std::min<size_t>(BAL_BLOCKS, (rounds + 1) / 2);
}

extern "C" size_t dh_moe_balance_ws_bytes(int T, int E) {
  if (T < 0 || E < 2 || E > 256) return 0;
  return ((size_t)std::max(balance_blocks(T, E, false), balance_blocks(T, E, true)) * (2 * (size_t)E + 1) + 1 + (E + BAL_FINISH - 1) / BAL_FINISH) * 4;
}

extern "C" int dh_moe_balance_fwd(int T, int E, const float* logits, const int32_t* idx, const int32_t* n_live, int32_t* counts, float* prob_mean, float* lse, float* loss, void* ws,
                                  size_t ws_bytes, void* stream) {
  if (T < 0 || E < 2 || E > 256) DH_FAIL(DH_ERR_SHAPE, "moe_balance_fwd: T=%d E=%d (E must be 2..256)", T, E);
  if (!counts || !prob_mean || !loss || (T > 0 && (!logits || !idx || !lse))) DH_FAIL(DH_ERR_INVALID_ARG, "moe_balance_fwd: null pointer");
  const size_t need = dh_moe_balance_ws_bytes(T, E);
  if (!ws || ws_bytes < need) DH_FAIL(DH_ERR_WORKSPACE_TOO_SMALL, "moe_balance_fwd: workspace %zu < %zu bytes", ws_bytes, need);
  if ((uintptr_t)ws & 3) DH_FAIL(DH_ERR_INVALID_ARG, "moe_balance_fwd: ws must be 4-byte aligned");
  const bool vec = balance_vec(E, logits, nullptr);
  const int blocks = balance_blocks(T, E, vec);
  float* part_p = (float*)ws;
  int32_t* part_n = (int32_t*)(part_p + (size_t)blocks * E);
  float* part_z = (float*)(part_n + (size_t)blocks * E);
  int* done = (int*)(part_z + blocks);
  float* part_b = (float*)(done + 1);
  hipStream_t s = (hipStream_t)stream;
#define GO(L, NE, V) moe_balance_kernel<L, NE, V><<<blocks, BAL_THREADS, 0, s>>>(T, E, logits, idx, n_live, lse, part_p, part_n, part_z, done, counts, prob_mean, loss)
  BALANCE_FOR(E, vec, GO);
#undef GO
  DH_LAUNCH_CHECK();
  if (blocks == 1) return DH_OK;
  moe_balance_finish_kernel<<<(E + BAL_FINISH - 1) / BAL_FINISH, 256, 0, s>>>(T, E, blocks, n_live, part_p, part_n, part_z, done, part_b, counts, prob_mean, loss);
  DH_LAUNCH_CHECK();
  return DH_OK;
}

extern "C" int dh_moe_balance_bwd(int T, int E, const float* logits, const float* lse, const int32_t* counts, const int32_t* n_live, const float* dloss, int accumulate, float* dlogits,
                                  void* stream) {
  if (T < 0 || E < 2 || E > 256) DH_FAIL(DH_ERR_SHAPE, "moe_balance_bwd: T=%d E=%d (E must be 2..256)", T, E);
  if (T == 0) return DH_OK;
  if (!logits || !lse || !counts || !dloss || !dlogits) DH_FAIL(DH_ERR_INVALID_ARG, "moe_balance_bwd: null pointer");
  const bool vec = balance_vec(E, logits, dlogits);
  const unsigned blocks = (unsigned)std::min<size_t>(2048, ((size_t)T * balance_lanes(E, vec) + 255) / 256);
#define GO(L, NE, V) moe_balance_bwd_kernel<L, NE, V><<<blocks, 256, 0, (hipStream_t)stream>>>(T, E, logits, lse, counts, n_live, dloss, accumulate, dlogits)
  BALANCE_FOR(E, vec, GO);
#undef GO
  DH_LAUNCH_CHECK();
  return DH_OK;
}

extern "C" int dh_moe_plan(int T, int E, int n_local, const int32_t* idx, const dh_moe_tables* tb, void* stream) {
  if (T < 0 || E < 2 || E > 256 || n_local < 1 || E % n_local) DH_FAIL(DH_ERR_SHAPE, "moe_plan: T=%d E=%d n_local=%d", T, E, n_local);
  if (!tb || !tb->rank || !tb->dest || !tb->src_tok || !tb->send_of_recv || !tb->recv_of_send || !tb->counts || !tb->offsets ||
      !tb->recv_start || !tb->group_rows || (T > 0 && !idx))
    DH_FAIL(DH_ERR_INVALID_ARG, "moe_plan: null pointer");
  const int n = 2 * T;
  hipStream_t s = (hipStream_t)stream;
  moe_rank_kernel<<<E, 64 * RANK_WAVES, 0, s>>>(n, idx, tb->rank, tb->counts);
  DH_LAUNCH_CHECK();
  moe_tables_kernel<<<std::max(1, (n + 255) / 256), 256, 0, s>>>(n, E, n_local, idx, tb->rank, tb->counts, tb->offsets, tb->recv_start, tb->group_rows,
                                                                 tb->dest, tb->src_tok, tb->send_of_recv, tb->recv_of_send);
  DH_LAUNCH_CHECK();
  return DH_OK;
}

extern "C" int dh_moe_gather_rows(int dtype, int n_rows, int H, const void* in, const int32_t* map, void* out, int n_blocks,
                                  void* stream) {
  return dh_launch_moe_gather_rows(dtype, n_rows, H, in, map, nullptr, out, n_blocks, (hipStream_t)stream);
}
int dh_launch_moe_gather_rows(int dtype, int n_rows, int H, const void* in, const int32_t* map, const int32_t* via, void* out, int n_blocks,
                              hipStream_t stream) {
  if (n_rows < 0 || H <= 0 || H % 8) DH_FAIL(DH_ERR_SHAPE, "moe_gather_rows: rows=%d H=%d (H must be a positive multiple of 8)", n_rows, H);
  if (n_blocks < 0 || n_blocks > 65536) DH_FAIL(DH_ERR_INVALID_ARG, "moe_gather_rows: n_blocks %d outside 0..65536", n_blocks);
  if (n_rows == 0) return DH_OK;
  if (!in || !map || !out) DH_FAIL(DH_ERR_INVALID_ARG, "moe_gather_rows: null pointer");
  size_t want = ((size_t)n_rows * (H / 8) + 255) / 256, cap = n_blocks > 0 ? (size_t)n_blocks : 4096;
  unsigned grid = (unsigned)(want < cap ? want : cap);
  if (dtype == DH_BF16) gather_rows_kernel<bf16_t><<<grid, 256, 0, stream>>>(n_rows, H, (const bf16_t*)in, map, via, (bf16_t*)out);
  else gather_rows_kernel<float><<<grid, 256, 0, stream>>>(n_rows, H, (const float*)in, map, via, (float*)out);
  DH_LAUNCH_CHECK();
  return DH_OK;
}

extern "C" int dh_moe_combine(int dtype, int T, int H, const void* yp, const int32_t* dest, const float* prob,
                              const void* residual, void* y, void* stream) {
  return dh_launch_moe_combine(dtype, T, H, yp, dest, nullptr, prob, residual, y, (hipStream_t)stream);
}
int dh_launch_moe_combine(int dtype, int T, int H, const void* yp, const int32_t* dest, const int32_t* via, const float* prob,
                          const void* residual, void* y, hipStream_t stream) {
  if (T < 0 || H <= 0 || H % 8) DH_FAIL(DH_ERR_SHAPE, "moe_combine: T=%d H=%d (H must be a positive multiple of 8)", T, H);
  if (T == 0) return DH_OK;
  if (!yp || !dest || !y) DH_FAIL(DH_ERR_INVALID_ARG, "moe_combine: null pointer");
  unsigned grid = (unsigned)(((size_t)T * (H / 8) + 255) / 256);
  if (dtype == DH_BF16) combine_kernel<bf16_t><<<grid, 256, 0, stream>>>(T, H, (const bf16_t*)yp, dest, via, prob, (const bf16_t*)residual, (bf16_t*)y);
  else combine_kernel<float><<<grid, 256, 0, stream>>>(T, H, (const float*)yp, dest, via, prob, (const float*)residual, (float*)y);
  DH_LAUNCH_CHECK();
  return DH_OK;
}

extern "C" int dh_moe_combine_bwd(int dtype, int T, int H, const void* dy, const void* yp, const int32_t* dest, const float* prob,
                                  void* dyp, float* dprob, void* stream) {
  if (T < 0 || H <= 0 || H % 8) DH_FAIL(DH_ERR_SHAPE, "moe_combine_bwd: T=%d H=%d (H must be a positive multiple of 8)", T, H);
  if (T == 0) return DH_OK;
  if (!dy || !yp || !dest || !prob || !dyp || !dprob) DH_FAIL(DH_ERR_INVALID_ARG, "moe_combine_bwd: null pointer");
  if (dtype == DH_BF16)
    combine_bwd_kernel<bf16_t><<<T, 256, 0, (hipStream_t)stream>>>(H, (const bf16_t*)dy, (const bf16_t*)yp, dest, prob, (bf16_t*)dyp, dprob);
  else
    combine_bwd_kernel<float><<<T, 256, 0, (hipStream_t)stream>>>(H, (const float*)dy, (const float*)yp, dest, prob, (float*)dyp, dprob);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
