// Attention with a sliding window and sinks: what its sources share.
#pragma once
#include "mixers.h"

// The queries that see key j are rows j .. end - 1.
__device__ __forceinline__ int window_queries_end(const WindowGeom& g, int j) { return j < g.sinks ? g.seq : (int)min((long long)g.seq, (long long)j + g.window); }

int dh_launch_window_fwd_bf16(const WindowGeom& g, const bf16_t* qkv, bf16_t* o, float* lse, void* ws, hipStream_t stream);
size_t dh_window_fwd_bf16_ws_bytes(const WindowGeom& g);
int dh_launch_window_bwd_bf16(const WindowGeom& g, const bf16_t* qkv, const bf16_t* o, const bf16_t* dout, const float* lse, bf16_t* dqkv, float* delta, void* ws, hipStream_t stream);
size_t dh_window_bwd_bf16_ws_bytes(const WindowGeom& g);
int dh_launch_window_fwd_f32(const WindowGeom& g, const float* qkv, float* o, float* lse, hipStream_t stream);
int dh_launch_window_bwd_f32(const WindowGeom& g, const float* qkv, const float* o, const float* dout, const float* lse, float* dqkv, float* delta, hipStream_t stream);
