// Attention under masks (mslt_op_attention_masked): what its kernels share.
#pragma once
#include "common.cuh"
#include "../../include/mslt.h"

namespace mslt {

// The mask and the scores' form, as the kernels read them.
struct AttnMask {
  int S, causal;
  float scale, cap;
  const float* slopes;
  const int32_t *prefix, *docs, *lens;
};

// ---- which loop blocks a row tile visits --------------------------------------------------------------
namespace {

struct Seq { int len, prefix; };
__device__ __forceinline__ Seq sequence(const AttnMask& m, int b) {
  Seq s;
  s.len = m.lens ? min(max(m.lens[b], 0), m.S) : m.S;
  s.prefix = m.causal ? (m.prefix ? min(max(m.prefix[b], 0), m.S) : 0) : m.S;
  return s;
}

// Called by the whole block.  list[i] receives 2 * block + (pairs to test); returns their number.  Rows r0 .. r0 + kRows - 1 are
// queries (and the blocks keys), or with kKeys the other way round.  red: 16 words of shared memory.
template <bool kKeys, int kWarps, int kRows, int kCols>
__device__ __forceinline__ int list_blocks(const AttnMask& m, const Seq& s, int b, int r0, uint16_t* list, int* red) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int* docs = m.docs ? m.docs + (long long)b * m.S : nullptr;
  const int r1 = min(r0 + kRows, s.len) - 1;  // last live row
  int lo = 0, hi = 0;
  if (docs) {
    if (warp < kRows / 32) {
      const int r = r0 + (int)threadIdx.x;
      const bool live = r < s.len;
      const int d = live ? docs[r] : 0;
      const int mn = __reduce_min_sync(0xffffffffu, live ? d : 0x7fffffff), mx = __reduce_max_sync(0xffffffffu, live ? d : (int)0x80000000);
      if (lane == 0) {
        red[warp] = mn;
        red[4 + warp] = mx;
      }
    }
    __syncthreads();
    lo = red[0];
    hi = red[4];
    for (int i = 1; i < kRows / 32; i++) {
      lo = min(lo, red[i]);
      hi = max(hi, red[4 + i]);
    }
  }
  int first = 0, last = 0;
  if (r0 < s.len) {
    last = kKeys ? s.len : min(s.len, max(r1 + 1, s.prefix));
    first = kKeys && r0 >= s.prefix ? r0 / kCols : 0;
    last = (last + kCols - 1) / kCols;
  }
  // whole by positions: every pair of live rows counts
  auto whole = [&](int c0) {
    if (c0 + kCols > s.len) return false;
    return kKeys ? (c0 >= r1 || r1 < s.prefix) : (c0 + kCols - 1 <= r0 || c0 + kCols <= s.prefix);
  };
  if (docs) {
    constexpr int kAhead = 256 / kCols;  // blocks whose documents are asked for together
    for (int base = first + warp; base < last; base += kWarps * kAhead) {
      int d[kAhead][kCols / 32];
#pragma unroll
      for (int u = 0; u < kAhead; u++)
#pragma unroll
        for (int e = 0; e < kCols / 32; e++) {
          const int c = (base + u * kWarps) * kCols + 32 * e + lane;
          d[u][e] = c < s.len ? docs[c] : 0;
        }
#pragma unroll
      for (int u = 0; u < kAhead; u++) {
        const int blk = base + u * kWarps;
        int mn = 0x7fffffff, mx = (int)0x80000000;
#pragma unroll
        for (int e = 0; e < kCols / 32; e++)
          if (blk * kCols + 32 * e + lane < s.len) {
            mn = min(mn, d[u][e]);
            mx = max(mx, d[u][e]);
          }
        mn = __reduce_min_sync(0xffffffffu, mn);
        mx = __reduce_max_sync(0xffffffffu, mx);
        if (lane == 0 && blk < last)
          list[blk] = mn > hi || mx < lo ? 0 : (lo == hi && mn == lo && mx == lo && whole(blk * kCols)) ? 1 : 2;
      }
    }
    __syncthreads();
  }
  if (warp == 0) {
    int n = 0;
    for (int base = first; base < last; base += 32) {
      const int blk = base + lane;
      int kind = 0;
      if (blk < last) kind = docs ? list[blk] : whole(blk * kCols) ? 1 : 2;
      const uint32_t take = __ballot_sync(0xffffffffu, kind != 0);
      __syncwarp();
      if (kind) list[n + __popc(take & ((1u << lane) - 1))] = (uint16_t)(blk * 2 + (kind == 2));
      n += __popc(take);
      __syncwarp();
    }
    if (lane == 0) red[8] = n;
  }
  __syncthreads();
  return red[8];
}

}  // namespace

// fp32 (attn_masked_f32.cu) and bf16 (attn_masked_tc.cu); err: 256 bytes
int attn_masked_f32_fwd(const mslt_attention_desc& d, cudaStream_t st, char* err);
int attn_masked_f32_bwd(const mslt_attention_desc& d, float* delta, cudaStream_t st, char* err);
int attn_masked_tc_fwd(const mslt_attention_desc& d, int* status, cudaStream_t st, char* err);
int attn_masked_tc_bwd(const mslt_attention_desc& d, float* delta, int* next, int* status, cudaStream_t st, char* err);

}  // namespace mslt
