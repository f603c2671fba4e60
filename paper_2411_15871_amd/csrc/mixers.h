// Token mixers that are linear in the row's length: what their sources share.
#pragma once
#include "common.h"

#define MIX_MAX_BATCH 65535
#define MIX_MAX_SEQ (1 << 26)     // blocks of 16 rows with 512 threads: a launch counts threads along x in 32 bits
#define MIX_MAX_TOKENS (1 << 28)
#define MIX_MAX_HEADS 1024
static inline bool mix_unaligned(const void* p, size_t a = 16) { return ((uintptr_t)p & (a - 1)) != 0; }
static inline int mix_check(const char* who, int dtype, int batch, int seq, int nq, int nkv, int d) {
  if (dtype != DH_F32 && dtype != DH_BF16) DH_FAIL(DH_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (batch < 0 || seq < 0 || nq <= 0 || nkv <= 0 || nq % nkv) DH_FAIL(DH_ERR_SHAPE, "%s: batch=%d seq=%d nq=%d nkv=%d", who, batch, seq, nq, nkv);
  if (batch > MIX_MAX_BATCH || seq > MIX_MAX_SEQ || (long long)batch * seq > MIX_MAX_TOKENS || nq > MIX_MAX_HEADS)
    DH_FAIL(DH_ERR_SHAPE, "%s: batch=%d seq=%d nq=%d (at most %d, %d, %d tokens and %d)", who, batch, seq, nq, MIX_MAX_BATCH, MIX_MAX_SEQ, MIX_MAX_TOKENS, MIX_MAX_HEADS);
  if (dtype == DH_F32 && (d <= 0 || d % 8 || d > 128)) DH_FAIL(DH_ERR_SHAPE, "%s: head_dim %d must be a multiple of 8, at most 128", who, d);
  if (dtype == DH_BF16 && d != 64 && d != 128) DH_FAIL(DH_ERR_SHAPE, "%s: head_dim %d must be 64 or 128", who, d);
  return DH_OK;
}
static inline bool mix_sized(int dtype, int batch, int seq, int nq, int nkv, int d) {  // for the workspace queries, which report nothing
  return (dtype == DH_F32 || dtype == DH_BF16) && batch > 0 && batch <= MIX_MAX_BATCH && seq > 0 && seq <= MIX_MAX_SEQ && (long long)batch * seq <= MIX_MAX_TOKENS && nkv > 0 && nq > 0 &&
         nq <= MIX_MAX_HEADS && nq % nkv == 0 && (dtype == DH_F32 ? d > 0 && d % 8 == 0 && d <= 128 : d == 64 || d == 128);
}

// Attention with a window and sinks: the row at position i of its sequence sees j <= i with j > i - window or j < sinks.
struct WindowGeom {
  int batch, seq, window, sinks, nq, nkv, d;
  float scale;
};
