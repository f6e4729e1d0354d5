// Attention under masks in fp32, forward and backward, on the CUDA cores (a tolerance of 1e-4 and less rules the
// tensor cores' formats out, and the split of operands into bf16 planes costs more than it gains on scores that are
// used once).  The scores never reach memory:
//   forward   a block of 32 queries walks over the key tiles that its mask leaves, with the running maximum and sum
//   backward  P = e^(z - lse), dS = P (dP - delta) dz/ds, delta = rowsum(dC C); dQ = scale dS K by blocks of queries,
//             dK = scale dS^T Q and dV = P^T dC by blocks of keys, over all query heads that share them, in one launch
// A block owns 32 rows, 128 threads hold 4 x 4 scores each, then 4 rows x 4 (8) columns of the accumulators, as packed
// multiply-adds.  32 rows and not 64 because full precision is used on small batches, whose blocks have to fill the device:
// 2 x 12 heads x 509 keys in 3 documents, forward | backward, 81 | 264 us with 64 rows and plain loads, 65 | 165 us with 32 and
// two launches for the backward, 65 | 132 us so.  What bounds it: where the device is full (4 x 12 x 512) half of the
// multiply-adds' issue slots (110 | 311 us of 46 | 140), on small batches the longest blocks' steps one after the other, 3 us
// each for a block alone on its SM (5500 cycles, 2050 of them multiply-adds).  The
// other side's tiles of 64 rows are asked for by asynchronous copies as soon as the product before is done with their memory.
// A tile is left out where the mask leaves none of its pairs (attn_masked.h).  Rows beyond a sequence are zero in shared memory.
// delta is summed in the order in which dP is, so that where a query sees a single key dP - delta is exactly zero.
#include <math.h>
#include <stdio.h>

#include <mutex>

#include "attn_masked.h"

namespace mslt {
namespace {

constexpr int MF_R = 32;         // rows of a block
constexpr int MF_C = 64;         // rows of a tile of the other side
constexpr int MF_RPT = 4;        // rows of a thread (2 on twice the threads: backward 38 % slower, the reads of operands decide)
constexpr int MF_NT = 16 * MF_R / MF_RPT;
constexpr int MF_PP = MF_C + 4;  // floats between rows of a tile of scores

struct Rows { const float* p; int64_t batch, row, head; };
struct MaskedParams {
  AttnMask m;
  Rows q, k, v, dc, c;
  Rows o, dk, dv;     // forward: ctx; backward: dq, dk, dv
  float *lse, *delta;
  int batch, heads, kv_heads, D, tiles, rows;
  unsigned kv_blocks;
};

__device__ __forceinline__ const float* row_ptr(const Rows& r, int64_t b, int64_t i, int h) {
  return r.p + b * r.batch + i * r.row + h * r.head;
}

// Tile, head and sequence of a block.  causal: the tiles with the longest loops start first, the last queries or the first keys;
// else the tiles of a head side by side, which read the same rows.
struct Place { int tile, h, b; };
__device__ __forceinline__ Place place_of(const MaskedParams& p, int block, int heads, bool keys) {
  Place a;
  int head;
  if (p.m.causal) {
    const int per = heads * p.batch, t = block / per;
    head = block - t * per;
    a.tile = keys ? t : p.tiles - 1 - t;
  } else {
    head = block / p.tiles;
    a.tile = block - head * p.tiles;
  }
  a.b = head / heads;
  a.h = head - a.b * heads;
  return a;
}

// Asks for rows [r0, r0 + kRows) of a head; rows from `rows` on and columns from D on are zero.
template <int DP, int kRows>
__device__ __forceinline__ void ask_tile(float* dst, const Rows& src, int b, int r0, int h, int rows, int D) {
#pragma unroll
  for (int i = 0; i < kRows * (DP / 4) / MF_NT; i++) {
    const int idx = threadIdx.x + i * MF_NT, r = idx / (DP / 4), c = idx % (DP / 4) * 4;
    const bool live = r0 + r < rows && c < D;
    const float* g = live ? row_ptr(src, b, r0 + r, h) + c : src.p;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst + r * (DP + 4) + c)),
                 "l"(g), "r"(live ? 16 : 0)
                 : "memory");
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
}
// all but the last N groups asked for have landed, for the whole block
template <int N>
__device__ __forceinline__ void landed() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
  __syncthreads();
}

// s[i][c] = row MF_RPT ty + i of A . row tx + 16 c of B, even and odd elements summed apart
template <int DP>
__device__ __forceinline__ void products(const float* A, const float* B, int ty, int tx, float (&s)[MF_RPT][4]) {
  float2 acc[MF_RPT][4];
#pragma unroll
  for (int i = 0; i < MF_RPT; i++)
#pragma unroll
    for (int c = 0; c < 4; c++) acc[i][c] = make_float2(0.f, 0.f);
#pragma unroll 4
  for (int e = 0; e < DP; e += 4) {
    float4 a[MF_RPT], b[4];
#pragma unroll
    for (int i = 0; i < MF_RPT; i++) a[i] = *reinterpret_cast<const float4*>(A + (MF_RPT * ty + i) * (DP + 4) + e);
#pragma unroll
    for (int c = 0; c < 4; c++) b[c] = *reinterpret_cast<const float4*>(B + (tx + 16 * c) * (DP + 4) + e);
#pragma unroll
    for (int i = 0; i < MF_RPT; i++)
#pragma unroll
      for (int c = 0; c < 4; c++) {
        acc[i][c] = __ffma2_rn(make_float2(a[i].x, a[i].y), make_float2(b[c].x, b[c].y), acc[i][c]);
        acc[i][c] = __ffma2_rn(make_float2(a[i].z, a[i].w), make_float2(b[c].z, b[c].w), acc[i][c]);
      }
  }
#pragma unroll
  for (int i = 0; i < MF_RPT; i++)
#pragma unroll
    for (int c = 0; c < 4; c++) s[i][c] = acc[i][c].x + acc[i][c].y;
}

// acc row MF_RPT ty + i, columns 4 tx + 64 j.. += sum over the rows of B of P[row][n] B[n][column]
template <int DP>
__device__ __forceinline__ void accumulate(const float* P, const float* B, int ty, int tx, float2 (&acc)[MF_RPT][DP / 64][2]) {
#pragma unroll 4
  for (int n = 0; n < MF_C; n += 4) {
    float4 p[MF_RPT];
#pragma unroll
    for (int i = 0; i < MF_RPT; i++) p[i] = *reinterpret_cast<const float4*>(P + (MF_RPT * ty + i) * MF_PP + n);
#pragma unroll
    for (int k = 0; k < 4; k++)
#pragma unroll
      for (int j = 0; j < DP / 64; j++) {
        const float4 b = *reinterpret_cast<const float4*>(B + (n + k) * (DP + 4) + 64 * j + 4 * tx);
#pragma unroll
        for (int i = 0; i < MF_RPT; i++) {
          const float w = k == 0 ? p[i].x : k == 1 ? p[i].y : k == 2 ? p[i].z : p[i].w;
          acc[i][j][0] = __ffma2_rn(make_float2(w, w), make_float2(b.x, b.y), acc[i][j][0]);
          acc[i][j][1] = __ffma2_rn(make_float2(w, w), make_float2(b.z, b.w), acc[i][j][1]);
        }
      }
  }
}

__device__ __forceinline__ float half_max(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float half_sum(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

__device__ __forceinline__ bool sees(const Seq& s, int i, int j, int di, int dj) {
  return i < s.len && j < s.len && di == dj && (j <= i || j < s.prefix);
}
// The scores behind cap, bias and mask (where test: others -infinity); bend: the cap's derivative.  Rows i0 + i, columns
// j0 + 16 c.  Exponentials further down are 2^x of the hardware (relative error 2^-22) of a rounded x log2(e): what that
// costs grows with |x|, as the probability falls.
template <bool kKeys>
__device__ __forceinline__ void scores(const AttnMask& m, const Seq& s, float slope, bool test, int i0, int j0, const int* idocs,
                                       const int* jdocs, float (&z)[MF_RPT][4], float (&bend)[MF_RPT][4]) {
#pragma unroll
  for (int i = 0; i < MF_RPT; i++)
#pragma unroll
    for (int c = 0; c < 4; c++) {
      z[i][c] *= m.scale;
      bend[i][c] = 1.f;
    }
  if (m.cap > 0.f) {
#pragma unroll
    for (int i = 0; i < MF_RPT; i++)
#pragma unroll
      for (int c = 0; c < 4; c++) {
        const float t = tanhf(z[i][c] / m.cap);
        z[i][c] = m.cap * t;
        bend[i][c] = 1.f - t * t;
      }
  }
  if (m.slopes) {
#pragma unroll
    for (int i = 0; i < MF_RPT; i++)
#pragma unroll
      for (int c = 0; c < 4; c++) z[i][c] -= slope * fabsf((float)(i0 + i - j0 - 16 * c));
  }
  if (test) {
#pragma unroll
    for (int i = 0; i < MF_RPT; i++)
#pragma unroll
      for (int c = 0; c < 4; c++) {
        const int a = i0 + i, b = j0 + 16 * c;
        const bool ok = kKeys ? sees(s, b, a, jdocs[16 * c], idocs[i]) : sees(s, a, b, idocs[i], jdocs[16 * c]);
        z[i][c] = ok ? z[i][c] : -INFINITY;
      }
  }
}

__device__ __forceinline__ int document(const AttnMask& m, const Seq& s, int b, int r) {
  return m.docs && r < s.len ? m.docs[(int64_t)b * m.S + r] : 0;
}

template <int DP>
__device__ __forceinline__ void store_rows(const Rows& dst, int b, int r0, int h, int S, int D, int ty, int tx,
                                           const float2 (&acc)[MF_RPT][DP / 64][2], const float (&f)[MF_RPT]) {
#pragma unroll
  for (int i = 0; i < MF_RPT; i++) {
    const int r = r0 + MF_RPT * ty + i;
    if (r >= S) continue;
    float* out = const_cast<float*>(row_ptr(dst, b, r, h));
#pragma unroll
    for (int j = 0; j < DP / 64; j++) {
      const int c = 64 * j + 4 * tx;
      if (c >= D) continue;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);  // f = 0: whatever the accumulator holds
      if (f[i] != 0.f) v = make_float4(acc[i][j][0].x * f[i], acc[i][j][0].y * f[i], acc[i][j][1].x * f[i], acc[i][j][1].y * f[i]);
      *reinterpret_cast<float4*>(out + c) = v;
    }
  }
}

// Shared memory of both kernels: row tiles, two loop tiles, scores, then the list of loop blocks.
template <int DP> __host__ __device__ constexpr size_t tile_floats(int row_tiles) {
  return (size_t)(row_tiles * MF_R + 2 * MF_C) * (DP + 4) + (size_t)MF_R * MF_PP;
}

template <int DP>
__global__ void __launch_bounds__(MF_NT)
masked_fwd_kernel(const MaskedParams p) {
  extern __shared__ __align__(16) float sm[];
  __shared__ int qdocs[MF_R], kdocs[MF_C], red[16];
  float* Qs = sm;
  float* Ks = Qs + MF_R * (DP + 4);
  float* Vs = Ks + MF_C * (DP + 4);
  float* Ps = Vs + MF_C * (DP + 4);
  uint16_t* list = (uint16_t*)(sm + tile_floats<DP>(1));
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const Place place = place_of(p, blockIdx.x, p.heads, false);
  const int h = place.h, b = place.b;
  const int hk = h / (p.heads / p.kv_heads), q0 = place.tile * MF_R;
  pdl_begin();
  const Seq s = sequence(p.m, b);
  const float slope = p.m.slopes ? p.m.slopes[h] : 0.f;
  ask_tile<DP, MF_R>(Qs, p.q, b, q0, h, s.len, p.D);
  if (threadIdx.x < MF_R) qdocs[threadIdx.x] = document(p.m, s, b, q0 + threadIdx.x);
  const int n = list_blocks<false, MF_NT / 32, MF_R, MF_C>(p.m, s, b, q0, list, red);
  float2 acc[MF_RPT][DP / 64][2];
  float top[MF_RPT], sum[MF_RPT];
#pragma unroll
  for (int i = 0; i < MF_RPT; i++) {
    top[i] = -INFINITY;
    sum[i] = 0.f;
#pragma unroll
    for (int j = 0; j < DP / 64; j++) acc[i][j][0] = acc[i][j][1] = make_float2(0.f, 0.f);
  }
  int doc = 0;
  auto ask_k = [&](int j) {
    const int k0 = (list[j] >> 1) * MF_C;
    ask_tile<DP, MF_C>(Ks, p.k, b, k0, hk, s.len, p.D);
    if (threadIdx.x < MF_C) doc = document(p.m, s, b, k0 + threadIdx.x);
  };
  auto ask_v = [&](int j) { ask_tile<DP, MF_C>(Vs, p.v, b, (list[j] >> 1) * MF_C, hk, s.len, p.D); };
  if (n > 0) {
    ask_k(0);
    ask_v(0);
  }
  for (int j = 0; j < n; j++) {
    const int k0 = (list[j] >> 1) * MF_C;
    const bool test = list[j] & 1;
    if (threadIdx.x < MF_C) kdocs[threadIdx.x] = doc;
    landed<1>();
    float z[MF_RPT][4];
    products<DP>(Qs, Ks, ty, tx, z);
    __syncthreads();
    if (j + 1 < n) ask_k(j + 1);
    else asm volatile("cp.async.commit_group;" ::: "memory");
    float bend[MF_RPT][4];
    scores<false>(p.m, s, slope, test, q0 + MF_RPT * ty, k0 + tx, qdocs + MF_RPT * ty, kdocs + tx, z, bend);
#pragma unroll
    for (int i = 0; i < MF_RPT; i++) {
      float t = top[i];
#pragma unroll
      for (int c = 0; c < 4; c++) t = fmaxf(t, z[i][c]);
      t = half_max(t);
      const float base = t == -INFINITY ? 0.f : t;
      const float keep = __expf(top[i] - base);
      top[i] = t;
      float part = 0.f;
#pragma unroll
      for (int c = 0; c < 4; c++) {
        const float e = __expf(z[i][c] - base);
        part += e;
        Ps[(MF_RPT * ty + i) * MF_PP + tx + 16 * c] = e;
      }
      sum[i] = sum[i] * keep + half_sum(part);
#pragma unroll
      for (int e = 0; e < DP / 64; e++) {
        acc[i][e][0] = __fmul2_rn(acc[i][e][0], make_float2(keep, keep));
        acc[i][e][1] = __fmul2_rn(acc[i][e][1], make_float2(keep, keep));
      }
    }
    landed<1>();
    accumulate<DP>(Ps, Vs, ty, tx, acc);
    __syncthreads();
    if (j + 1 < n) ask_v(j + 1);
  }
  float f[MF_RPT];
#pragma unroll
  for (int i = 0; i < MF_RPT; i++) {
    f[i] = sum[i] == 0.f ? 0.f : 1.f / sum[i];
    const int r = q0 + MF_RPT * ty + i;
    const bool dead = r >= s.len;  // its row of Q is zero and may have been given scores where nothing is tested
    if (dead) f[i] = 0.f;
    if (tx == 0 && p.lse && r < p.m.S) p.lse[((int64_t)b * p.heads + h) * p.m.S + r] = dead ? -INFINITY : top[i] + logf(sum[i]);
  }
  store_rows<DP>(p.o, b, q0, h, p.m.S, p.D, ty, tx, acc, f);
}

// delta_i = dC_i . C_i, even and odd elements summed apart, one thread a row and head
__global__ void __launch_bounds__(MF_NT)
masked_delta_kernel(const MaskedParams p) {
  pdl_begin();
  const int64_t n = (int64_t)blockIdx.x * MF_NT + threadIdx.x;
  if (n >= p.rows) return;
  const int S = p.m.S, h = (int)(n % p.heads), i = (int)(n / p.heads % S);  // head fastest: neighbours in memory
  const int64_t b = n / p.heads / S;
  float2 acc = make_float2(0.f, 0.f);
  const float *dc = row_ptr(p.dc, b, i, h), *c = row_ptr(p.c, b, i, h);
#pragma unroll 4
  for (int e = 0; e < p.D; e += 4) {
    const float4 x = *reinterpret_cast<const float4*>(dc + e), y = *reinterpret_cast<const float4*>(c + e);
    acc = __ffma2_rn(make_float2(x.x, x.y), make_float2(y.x, y.y), acc);
    acc = __ffma2_rn(make_float2(x.z, x.w), make_float2(y.z, y.w), acc);
  }
  p.delta[(b * p.heads + h) * S + i] = acc.x + acc.y;
}

// what a block keeps beside its tiles
struct Beside { int fixed_docs[MF_R], docs[MF_C], red[16]; float lses[MF_C], deltas[MF_C]; };

// dQ of 32 queries
template <int DP>
__device__ __forceinline__ void gradient_q(const MaskedParams& p, int block, float* sm, Beside& at_side) {
  int *qdocs = at_side.fixed_docs, *kdocs = at_side.docs, *red = at_side.red;
  float* Qs = sm;
  float* Cs = Qs + MF_R * (DP + 4);
  float* Ks = Cs + MF_R * (DP + 4);
  float* Vs = Ks + MF_C * (DP + 4);
  float* Ps = Vs + MF_C * (DP + 4);
  uint16_t* list = (uint16_t*)(sm + tile_floats<DP>(2));
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const Place place = place_of(p, block, p.heads, false);
  const int h = place.h, b = place.b;
  const int hk = h / (p.heads / p.kv_heads), q0 = place.tile * MF_R;
  const Seq s = sequence(p.m, b);
  const float slope = p.m.slopes ? p.m.slopes[h] : 0.f;
  ask_tile<DP, MF_R>(Qs, p.q, b, q0, h, s.len, p.D);
  ask_tile<DP, MF_R>(Cs, p.dc, b, q0, h, s.len, p.D);
  if (threadIdx.x < MF_R) qdocs[threadIdx.x] = document(p.m, s, b, q0 + threadIdx.x);
  const int n = list_blocks<false, MF_NT / 32, MF_R, MF_C>(p.m, s, b, q0, list, red);
  float2 acc[MF_RPT][DP / 64][2];
  float lse[MF_RPT], delta[MF_RPT];
#pragma unroll
  for (int i = 0; i < MF_RPT; i++) {
    const int r = q0 + MF_RPT * ty + i;
    const int64_t at = ((int64_t)b * p.heads + h) * p.m.S + r;
    lse[i] = r < s.len ? p.lse[at] : INFINITY;  // no probability
    delta[i] = r < s.len ? p.delta[at] : 0.f;
#pragma unroll
    for (int j = 0; j < DP / 64; j++) acc[i][j][0] = acc[i][j][1] = make_float2(0.f, 0.f);
  }
  int doc = 0;
  auto ask_k = [&](int j) {
    const int k0 = (list[j] >> 1) * MF_C;
    ask_tile<DP, MF_C>(Ks, p.k, b, k0, hk, s.len, p.D);
    if (threadIdx.x < MF_C) doc = document(p.m, s, b, k0 + threadIdx.x);
  };
  auto ask_v = [&](int j) { ask_tile<DP, MF_C>(Vs, p.v, b, (list[j] >> 1) * MF_C, hk, s.len, p.D); };
  if (n > 0) {
    ask_v(0);
    ask_k(0);
  }
  for (int j = 0; j < n; j++) {
    const int k0 = (list[j] >> 1) * MF_C;
    const bool test = list[j] & 1;
    if (threadIdx.x < MF_C) kdocs[threadIdx.x] = doc;
    float z[MF_RPT][4], dp[MF_RPT][4];
    landed<1>();
    products<DP>(Cs, Vs, ty, tx, dp);
    landed<0>();
    if (j + 1 < n) ask_v(j + 1);
    products<DP>(Qs, Ks, ty, tx, z);
    float bend[MF_RPT][4];
    scores<false>(p.m, s, slope, test, q0 + MF_RPT * ty, k0 + tx, qdocs + MF_RPT * ty, kdocs + tx, z, bend);
#pragma unroll
    for (int i = 0; i < MF_RPT; i++)
#pragma unroll
      for (int c = 0; c < 4; c++) {
        const float w = __expf(z[i][c] - lse[i]);
        Ps[(MF_RPT * ty + i) * MF_PP + tx + 16 * c] = w == 0.f ? 0.f : w * (dp[i][c] - delta[i]) * bend[i][c];
      }
    __syncwarp();  // the scores of a thread's rows are its half warp's
    accumulate<DP>(Ps, Ks, ty, tx, acc);
    __syncthreads();
    if (j + 1 < n) ask_k(j + 1);
  }
  float f[MF_RPT];
#pragma unroll
  for (int i = 0; i < MF_RPT; i++) f[i] = p.m.scale;
  store_rows<DP>(p.o, b, q0, h, p.m.S, p.D, ty, tx, acc, f);
}

// dK and dV of 32 keys: rows of the thread's tiles are keys, columns queries
template <int DP>
__device__ __forceinline__ void gradient_kv(const MaskedParams& p, int block, float* sm, Beside& at_side) {
  int *kdocs = at_side.fixed_docs, *qdocs = at_side.docs, *red = at_side.red;
  float *lses = at_side.lses, *deltas = at_side.deltas;
  float* Ks = sm;
  float* Vs = Ks + MF_R * (DP + 4);
  float* Qs = Vs + MF_R * (DP + 4);
  float* Cs = Qs + MF_C * (DP + 4);
  float* Ps = Cs + MF_C * (DP + 4);
  uint16_t* list = (uint16_t*)(sm + tile_floats<DP>(2));
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const Place place = place_of(p, block, p.kv_heads, true);
  const int hk = place.h, b = place.b;
  const int group = p.heads / p.kv_heads, k0 = place.tile * MF_R;
  const Seq s = sequence(p.m, b);
  ask_tile<DP, MF_R>(Ks, p.k, b, k0, hk, s.len, p.D);
  ask_tile<DP, MF_R>(Vs, p.v, b, k0, hk, s.len, p.D);
  if (threadIdx.x < MF_R) kdocs[threadIdx.x] = document(p.m, s, b, k0 + threadIdx.x);
  const int n = list_blocks<true, MF_NT / 32, MF_R, MF_C>(p.m, s, b, k0, list, red);
  float2 dk[MF_RPT][DP / 64][2], dv[MF_RPT][DP / 64][2];
#pragma unroll
  for (int i = 0; i < MF_RPT; i++)
#pragma unroll
    for (int j = 0; j < DP / 64; j++) dk[i][j][0] = dk[i][j][1] = dv[i][j][0] = dv[i][j][1] = make_float2(0.f, 0.f);
  // steps: the list once for every query head that shares the keys
  int doc = 0;
  float lse = 0.f, delta = 0.f;
  auto ask_q = [&](int j) {
    const int q0 = (list[j % n] >> 1) * MF_C, h = hk * group + j / n;
    ask_tile<DP, MF_C>(Qs, p.q, b, q0, h, s.len, p.D);
    if (threadIdx.x < MF_C) {
      const int r = q0 + threadIdx.x;
      const int64_t at = ((int64_t)b * p.heads + h) * p.m.S + r;
      doc = document(p.m, s, b, r);
      lse = r < s.len ? p.lse[at] : 0.f;
      delta = r < s.len ? p.delta[at] : 0.f;
    }
  };
  auto ask_c = [&](int j) { ask_tile<DP, MF_C>(Cs, p.dc, b, (list[j % n] >> 1) * MF_C, hk * group + j / n, s.len, p.D); };
  if (n > 0) {
    ask_c(0);
    ask_q(0);
  }
  for (int j = 0; j < n * group; j++) {
    const int entry = list[j % n], q0 = (entry >> 1) * MF_C;
    const bool test = entry & 1;
    const float slope = p.m.slopes ? p.m.slopes[hk * group + j / n] : 0.f;
    if (threadIdx.x < MF_C) {
      qdocs[threadIdx.x] = doc;
      lses[threadIdx.x] = lse;
      deltas[threadIdx.x] = delta;
    }
    float z[MF_RPT][4], dp[MF_RPT][4];
    landed<1>();
    products<DP>(Vs, Cs, ty, tx, dp);
    landed<0>();
    products<DP>(Ks, Qs, ty, tx, z);
    float bend[MF_RPT][4];
    scores<true>(p.m, s, slope, test, k0 + MF_RPT * ty, q0 + tx, kdocs + MF_RPT * ty, qdocs + tx, z, bend);
#pragma unroll
    for (int i = 0; i < MF_RPT; i++)
#pragma unroll
      for (int c = 0; c < 4; c++) {
        const int m = tx + 16 * c;
        const float w = __expf(z[i][c] - lses[m]);
        Ps[(MF_RPT * ty + i) * MF_PP + m] = w;
        z[i][c] = w == 0.f ? 0.f : w * (dp[i][c] - deltas[m]) * bend[i][c];
      }
    __syncwarp();
    accumulate<DP>(Ps, Cs, ty, tx, dv);
    __syncthreads();
    if (j + 1 < n * group) ask_c(j + 1);
#pragma unroll
    for (int i = 0; i < MF_RPT; i++)
#pragma unroll
      for (int c = 0; c < 4; c++) Ps[(MF_RPT * ty + i) * MF_PP + tx + 16 * c] = z[i][c];
    __syncwarp();
    accumulate<DP>(Ps, Qs, ty, tx, dk);
    __syncthreads();
    if (j + 1 < n * group) ask_q(j + 1);
  }
  // keys beyond the sequence are zero rows that may have been given scores where nothing is tested
  float one[MF_RPT], f[MF_RPT];
#pragma unroll
  for (int i = 0; i < MF_RPT; i++) {
    one[i] = k0 + MF_RPT * ty + i < s.len ? 1.f : 0.f;
    f[i] = p.m.scale * one[i];
  }
  store_rows<DP>(p.dk, b, k0, hk, p.m.S, p.D, ty, tx, dk, f);
  store_rows<DP>(p.dv, b, k0, hk, p.m.S, p.D, ty, tx, dv, one);
}

// Both in one launch, blocks of keys first, which have the longer steps: full precision is used on small batches, where either
// alone is less than a wave of blocks and the device idles behind its longest ones.
template <int DP>
__global__ void __launch_bounds__(MF_NT, DP == 64 ? 3 : 2)
masked_bwd_kernel(const MaskedParams p) {
  extern __shared__ __align__(16) float sm[];
  __shared__ Beside at_side;
  pdl_begin();
  if (blockIdx.x < p.kv_blocks) gradient_kv<DP>(p, blockIdx.x, sm, at_side);
  else gradient_q<DP>(p, blockIdx.x - p.kv_blocks, sm, at_side);
}

constexpr int kMaxDevices = 64;
std::mutex g_mf_mu;
int opt_in(const void* kernel, bool (&done)[kMaxDevices], size_t smem, char* err) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev < 0 || dev >= kMaxDevices)) e = cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_mf_mu);
  if (e == cudaSuccess && !done[dev]) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) {
    snprintf(err, 256, "attention_masked: %s", cudaGetErrorString(e));
    return MSLT_ERR_CUDA;
  }
  done[dev] = true;
  return 0;
}

Rows rows_of(const mslt_heads& h) { return Rows{(const float*)h.data, h.batch, h.row, h.head}; }

MaskedParams params_of(const mslt_attention_desc& d) {
  MaskedParams p = {};
  p.m = AttnMask{d.S, d.causal != 0, d.scale, d.cap, d.slopes, d.prefix, d.docs, d.lens};
  p.q = rows_of(d.q); p.k = rows_of(d.k); p.v = rows_of(d.v);
  p.lse = d.lse; p.batch = d.B; p.heads = d.heads; p.kv_heads = d.kv_heads; p.D = d.head_dim;
  p.tiles = (d.S + MF_R - 1) / MF_R;
  return p;
}

template <int DP> size_t smem_bytes(int row_tiles, int S) {
  return tile_floats<DP>(row_tiles) * sizeof(float) + ((size_t)(S + MF_C - 1) / MF_C * 2 + 15) / 16 * 16;
}
constexpr int kMostS = 131072;

template <int DP>
int forward(const mslt_attention_desc& d, cudaStream_t st, char* err) {
  static bool done[kMaxDevices];
  if (opt_in((const void*)masked_fwd_kernel<DP>, done, smem_bytes<DP>(1, kMostS), err)) return MSLT_ERR_CUDA;
  MaskedParams p = params_of(d);
  p.o = rows_of(d.ctx);
  launch_pdl(masked_fwd_kernel<DP>, d.B * d.heads * p.tiles, MF_NT, smem_bytes<DP>(1, d.S), st, p);
  return 0;
}

template <int DP>
int backward(const mslt_attention_desc& d, float* delta, cudaStream_t st, char* err) {
  static bool done[kMaxDevices];
  if (opt_in((const void*)masked_bwd_kernel<DP>, done, smem_bytes<DP>(2, kMostS), err)) return MSLT_ERR_CUDA;
  MaskedParams p = params_of(d);
  p.dc = rows_of(d.dctx); p.c = rows_of(d.ctx); p.delta = delta;
  p.rows = d.B * d.heads * d.S;
  launch_pdl(masked_delta_kernel, (int)(((int64_t)p.rows + MF_NT - 1) / MF_NT), MF_NT, 0, st, p);
  p.o = rows_of(d.dq); p.dk = rows_of(d.dk); p.dv = rows_of(d.dv);
  p.kv_blocks = (unsigned)d.B * d.kv_heads * p.tiles;
  launch_pdl(masked_bwd_kernel<DP>, p.kv_blocks + (unsigned)d.B * d.heads * p.tiles, MF_NT, smem_bytes<DP>(2, d.S), st, p);
  return 0;
}

}  // namespace

int attn_masked_f32_fwd(const mslt_attention_desc& d, cudaStream_t st, char* err) {
  return d.head_dim <= 64 ? forward<64>(d, st, err) : forward<128>(d, st, err);
}
int attn_masked_f32_bwd(const mslt_attention_desc& d, float* delta, cudaStream_t st, char* err) {
  return d.head_dim <= 64 ? backward<64>(d, delta, st, err) : backward<128>(d, delta, st, err);
}

}  // namespace mslt
