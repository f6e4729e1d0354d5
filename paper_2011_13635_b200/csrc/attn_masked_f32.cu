// Attention under masks in fp32, forward and backward, on the CUDA cores (a tolerance of 1e-4 and less rules the
// tensor cores' formats out, and the split of operands into bf16 planes costs more than it gains on scores that are
// used once).  The scores never reach memory:
//   forward   a block of 64 queries walks over the key tiles that its mask leaves, with the running maximum and sum
//   backward  P = e^(z - lse), dS = P (dP - delta) dz/ds, delta = rowsum(dC C); dQ = scale dS K by blocks of queries,
//             dK = scale dS^T Q and dV = P^T dC by blocks of keys, over all query heads that share them
// 256 threads hold 4 x 4 scores each, then 4 rows x 4 (8) columns of the accumulators, as packed multiply-adds.
// A tile is left out where the mask leaves none of its pairs by the rules on positions, or where no key's document lies
// between the least and the greatest document of the queries.  Rows beyond a sequence are zero in shared memory.
// delta is summed in the order in which dP is, so that where a query sees a single key dP - delta is exactly zero.
#include <math.h>
#include <stdio.h>

#include <mutex>

#include "attn_masked.h"

namespace mslt {
namespace {

constexpr int MF_T = 64;        // rows of a tile
constexpr int MF_NT = 256;
constexpr int MF_PP = MF_T + 4; // floats between rows of a tile of scores

struct Rows { const void* p; int64_t batch, row, head; };
struct MaskedParams {
  AttnMask m;
  Rows q, k, v, dc, c;
  void* rest;         // bf16, laid out like ctx
  Rows o0, o1;        // forward: ctx; queries: dq; keys: dk, dv
  float *lse, *delta;
  int heads, kv_heads, D, tiles;
};

template <typename T>
__device__ __forceinline__ const T* row_ptr(const Rows& r, int b, int64_t i, int h) {
  return (const T*)r.p + b * r.batch + i * r.row + h * r.head;
}

// rows [r0, r0 + 64) of a head as fp32; rows from `rows` on and columns from D on are zero
template <typename T, int DP>
__device__ __forceinline__ void load_tile(float* dst, const Rows& src, int b, int r0, int h, int rows, int D) {
  constexpr int V = VecT<T>::N;
  for (int idx = threadIdx.x; idx < MF_T * (DP / V); idx += MF_NT) {
    const int r = idx / (DP / V), c = idx % (DP / V) * V;
    float v[V];
#pragma unroll
    for (int j = 0; j < V; j++) v[j] = 0.f;
    if (r0 + r < rows && c < D) VecT<T>::load(row_ptr<T>(src, b, r0 + r, h) + c, v);
#pragma unroll
    for (int j = 0; j < V; j += 4)
      *reinterpret_cast<float4*>(dst + r * (DP + 4) + c + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
  }
}

// s[i][c] = row 4 ty + i of A . row tx + 16 c of B, even and odd elements summed apart
template <int DP>
__device__ __forceinline__ void products(const float* A, const float* B, int ty, int tx, float (&s)[4][4]) {
  float2 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; i++)
#pragma unroll
    for (int c = 0; c < 4; c++) acc[i][c] = make_float2(0.f, 0.f);
#pragma unroll 4
  for (int e = 0; e < DP; e += 4) {
    float4 a[4], b[4];
#pragma unroll
    for (int i = 0; i < 4; i++) a[i] = *reinterpret_cast<const float4*>(A + (4 * ty + i) * (DP + 4) + e);
#pragma unroll
    for (int c = 0; c < 4; c++) b[c] = *reinterpret_cast<const float4*>(B + (tx + 16 * c) * (DP + 4) + e);
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int c = 0; c < 4; c++) {
        acc[i][c] = __ffma2_rn(make_float2(a[i].x, a[i].y), make_float2(b[c].x, b[c].y), acc[i][c]);
        acc[i][c] = __ffma2_rn(make_float2(a[i].z, a[i].w), make_float2(b[c].z, b[c].w), acc[i][c]);
      }
  }
#pragma unroll
  for (int i = 0; i < 4; i++)
#pragma unroll
    for (int c = 0; c < 4; c++) s[i][c] = acc[i][c].x + acc[i][c].y;
}

// acc row 4 ty + i, columns 4 tx + 64 j.. += sum over the 64 rows of B of P[row][n] B[n][column]
template <int DP>
__device__ __forceinline__ void accumulate(const float* P, const float* B, int ty, int tx, float2 (&acc)[4][DP / 64][2]) {
#pragma unroll 4
  for (int n = 0; n < MF_T; n += 4) {
    float4 p[4];
#pragma unroll
    for (int i = 0; i < 4; i++) p[i] = *reinterpret_cast<const float4*>(P + (4 * ty + i) * MF_PP + n);
#pragma unroll
    for (int k = 0; k < 4; k++)
#pragma unroll
      for (int j = 0; j < DP / 64; j++) {
        const float4 b = *reinterpret_cast<const float4*>(B + (n + k) * (DP + 4) + 64 * j + 4 * tx);
#pragma unroll
        for (int i = 0; i < 4; i++) {
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

struct Seq { int len, prefix; float slope; };
__device__ __forceinline__ Seq sequence(const AttnMask& m, int b, int h) {
  Seq s;
  s.len = m.lens ? min(max(m.lens[b], 0), m.S) : m.S;
  s.prefix = m.causal ? (m.prefix ? min(max(m.prefix[b], 0), m.S) : 0) : m.S;
  s.slope = m.slopes ? m.slopes[h] : 0.f;
  return s;
}
__device__ __forceinline__ bool sees(const Seq& s, int i, int j, int di, int dj) {
  return i < s.len && j < s.len && di == dj && (j <= i || j < s.prefix);
}
// the score behind cap and bias; bend: the cap's derivative
__device__ __forceinline__ float score(const AttnMask& m, const Seq& s, float dot, int i, int j, float* bend) {
  float z = dot * m.scale;
  *bend = 1.f;
  if (m.cap > 0.f) {
    const float t = tanhf(z / m.cap);
    z = m.cap * t;
    *bend = 1.f - t * t;
  }
  return z - s.slope * fabsf((float)(i - j));
}

// Documents of a tile's rows into shared memory; returns whether any of them lies in [lo, hi] (and is not beyond len).
__device__ __forceinline__ bool tile_documents(const AttnMask& m, const Seq& s, int b, int r0, int* docs, int lo, int hi) {
  bool any = false;
  if (threadIdx.x < MF_T) {
    const int r = r0 + threadIdx.x;
    const int d = m.docs && r < s.len ? m.docs[(int64_t)b * m.S + r] : 0;
    docs[threadIdx.x] = d;
    any = r < s.len && d >= lo && d <= hi;
  }
  return __syncthreads_or(any) != 0;
}
// least and greatest document of the live rows of a tile already in shared memory
__device__ __forceinline__ void document_range(const Seq& s, int r0, const int* docs, int* lo, int* hi) {
  *lo = 0x7fffffff;
  *hi = (int)0x80000000;
  for (int r = 0; r < MF_T && r0 + r < s.len; r++) {
    *lo = min(*lo, docs[r]);
    *hi = max(*hi, docs[r]);
  }
}

template <typename T, int DP>
__device__ __forceinline__ void store_rows(const Rows& dst, int b, int r0, int h, int S, int D, int ty, int tx,
                                           const float2 (&acc)[4][DP / 64][2], const float (&f)[4], T* rest = nullptr) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int r = r0 + 4 * ty + i;
    if (r >= S) continue;
    T* out = const_cast<T*>(row_ptr<T>(dst, b, r, h));
#pragma unroll
    for (int j = 0; j < DP / 64; j++) {
      const int c = 64 * j + 4 * tx;
      if (c >= D) continue;
      const float o[4] = {acc[i][j][0].x * f[i], acc[i][j][0].y * f[i], acc[i][j][1].x * f[i], acc[i][j][1].y * f[i]};
#pragma unroll
      for (int n = 0; n < 4; n++) {
        out[c + n] = from_f<T>(o[n]);
        if (rest) rest[out - (const T*)dst.p + c + n] = from_f<T>(o[n] - to_f(out[c + n]));
      }
    }
  }
}

template <typename T, int DP>
__global__ void __launch_bounds__(MF_NT)
masked_fwd_kernel(const MaskedParams p) {
  extern __shared__ float sm[];
  __shared__ int qdocs[MF_T], kdocs[MF_T];
  float* Qs = sm;
  float* Ks = Qs + MF_T * (DP + 4);
  float* Vs = Ks + MF_T * (DP + 4);
  float* Ps = Vs + MF_T * (DP + 4);
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const int tile = blockIdx.x % p.tiles, h = blockIdx.x / p.tiles % p.heads, b = blockIdx.x / p.tiles / p.heads;
  const int hk = h / (p.heads / p.kv_heads), q0 = tile * MF_T;
  pdl_begin();
  const Seq s = sequence(p.m, b, h);
  float2 acc[4][DP / 64][2];
  float top[4], sum[4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    top[i] = -INFINITY;
    sum[i] = 0.f;
#pragma unroll
    for (int j = 0; j < DP / 64; j++) acc[i][j][0] = acc[i][j][1] = make_float2(0.f, 0.f);
  }
  load_tile<T, DP>(Qs, p.q, b, q0, h, s.len, p.D);
  tile_documents(p.m, s, b, q0, qdocs, 0, 0);
  int lo, hi;
  document_range(s, q0, qdocs, &lo, &hi);
  const int last = q0 >= s.len ? 0 : min(s.len, max(q0 + MF_T, s.prefix));
  for (int k0 = 0; k0 < last; k0 += MF_T) {
    __syncthreads();
    if (!tile_documents(p.m, s, b, k0, kdocs, lo, hi)) continue;
    load_tile<T, DP>(Ks, p.k, b, k0, hk, s.len, p.D);
    load_tile<T, DP>(Vs, p.v, b, k0, hk, s.len, p.D);
    __syncthreads();
    float z[4][4];
    products<DP>(Qs, Ks, ty, tx, z);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      float t = top[i];
#pragma unroll
      for (int c = 0; c < 4; c++) {
        const int qi = q0 + 4 * ty + i, kj = k0 + tx + 16 * c;
        float bend;
        z[i][c] = sees(s, qi, kj, qdocs[4 * ty + i], kdocs[tx + 16 * c]) ? score(p.m, s, z[i][c], qi, kj, &bend) : -INFINITY;
        t = fmaxf(t, z[i][c]);
      }
      t = half_max(t);
      const float base = t == -INFINITY ? 0.f : t;
      const float keep = expf(top[i] - base);
      top[i] = t;
      float part = 0.f;
#pragma unroll
      for (int c = 0; c < 4; c++) {
        const float e = expf(z[i][c] - base);
        part += e;
        Ps[(4 * ty + i) * MF_PP + tx + 16 * c] = e;
      }
      sum[i] = sum[i] * keep + half_sum(part);
#pragma unroll
      for (int j = 0; j < DP / 64; j++) {
        acc[i][j][0] = __fmul2_rn(acc[i][j][0], make_float2(keep, keep));
        acc[i][j][1] = __fmul2_rn(acc[i][j][1], make_float2(keep, keep));
      }
    }
    __syncwarp();
    accumulate<DP>(Ps, Vs, ty, tx, acc);
  }
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    f[i] = sum[i] > 0.f ? 1.f / sum[i] : 0.f;
    const int r = q0 + 4 * ty + i;
    if (tx == 0 && p.lse && r < p.m.S) p.lse[((int64_t)b * p.heads + h) * p.m.S + r] = top[i] + logf(sum[i]);
  }
  store_rows<T, DP>(p.o0, b, q0, h, p.m.S, p.D, ty, tx, acc, f, (T*)p.rest);
}

// delta_i = dC_i . C_i, even and odd elements summed apart, one thread a row and head
template <typename T>
__global__ void __launch_bounds__(MF_NT)
masked_delta_kernel(const MaskedParams p) {
  pdl_begin();
  const int64_t n = (int64_t)blockIdx.x * MF_NT + threadIdx.x;
  const int S = p.m.S;
  const int i = (int)(n % S), h = (int)(n / S % p.heads);
  const int64_t b = n / S / p.heads;
  if (n >= (int64_t)p.tiles) return;
  constexpr int V = VecT<T>::N;
  float2 acc = make_float2(0.f, 0.f);
  const T *dc = row_ptr<T>(p.dc, b, i, h), *c = row_ptr<T>(p.c, b, i, h);
  for (int e = 0; e < p.D; e += V) {
    float x[V], y[V];
    VecT<T>::load(dc + e, x);
    VecT<T>::load(c + e, y);
    if (p.rest) {
      float z[V];
      VecT<T>::load((const T*)p.rest + (c - (const T*)p.c.p) + e, z);
#pragma unroll
      for (int j = 0; j < V; j++) y[j] += z[j];
    }
#pragma unroll
    for (int j = 0; j < V; j += 2) acc = __ffma2_rn(make_float2(x[j], x[j + 1]), make_float2(y[j], y[j + 1]), acc);
  }
  p.delta[n] = acc.x + acc.y;
}

// dQ of 64 queries
template <typename T, int DP>
__global__ void __launch_bounds__(MF_NT)
masked_dq_kernel(const MaskedParams p) {
  extern __shared__ float sm[];
  __shared__ int qdocs[MF_T], kdocs[MF_T];
  float* Qs = sm;
  float* Cs = Qs + MF_T * (DP + 4);
  float* Ks = Cs + MF_T * (DP + 4);
  float* Vs = Ks + MF_T * (DP + 4);
  float* Ps = Vs + MF_T * (DP + 4);
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const int tile = blockIdx.x % p.tiles, h = blockIdx.x / p.tiles % p.heads, b = blockIdx.x / p.tiles / p.heads;
  const int hk = h / (p.heads / p.kv_heads), q0 = tile * MF_T;
  pdl_begin();
  const Seq s = sequence(p.m, b, h);
  float2 acc[4][DP / 64][2];
  float lse[4], delta[4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int r = q0 + 4 * ty + i;
    const int64_t at = ((int64_t)b * p.heads + h) * p.m.S + r;
    lse[i] = r < s.len ? p.lse[at] : 0.f;
    delta[i] = r < s.len ? p.delta[at] : 0.f;
#pragma unroll
    for (int j = 0; j < DP / 64; j++) acc[i][j][0] = acc[i][j][1] = make_float2(0.f, 0.f);
  }
  load_tile<T, DP>(Qs, p.q, b, q0, h, s.len, p.D);
  load_tile<T, DP>(Cs, p.dc, b, q0, h, s.len, p.D);
  tile_documents(p.m, s, b, q0, qdocs, 0, 0);
  int lo, hi;
  document_range(s, q0, qdocs, &lo, &hi);
  const int last = q0 >= s.len ? 0 : min(s.len, max(q0 + MF_T, s.prefix));
  for (int k0 = 0; k0 < last; k0 += MF_T) {
    __syncthreads();
    if (!tile_documents(p.m, s, b, k0, kdocs, lo, hi)) continue;
    load_tile<T, DP>(Ks, p.k, b, k0, hk, s.len, p.D);
    load_tile<T, DP>(Vs, p.v, b, k0, hk, s.len, p.D);
    __syncthreads();
    float z[4][4], dp[4][4];
    products<DP>(Qs, Ks, ty, tx, z);
    products<DP>(Cs, Vs, ty, tx, dp);
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int c = 0; c < 4; c++) {
        const int qi = q0 + 4 * ty + i, kj = k0 + tx + 16 * c;
        float ds = 0.f;
        if (sees(s, qi, kj, qdocs[4 * ty + i], kdocs[tx + 16 * c])) {
          float bend;
          const float w = expf(score(p.m, s, z[i][c], qi, kj, &bend) - lse[i]);
          ds = w * (dp[i][c] - delta[i]) * bend;
        }
        Ps[(4 * ty + i) * MF_PP + tx + 16 * c] = ds;
      }
    __syncwarp();
    accumulate<DP>(Ps, Ks, ty, tx, acc);
  }
  const float f[4] = {p.m.scale, p.m.scale, p.m.scale, p.m.scale};
  store_rows<T, DP>(p.o0, b, q0, h, p.m.S, p.D, ty, tx, acc, f);
}

// dK and dV of 64 keys: rows of the thread's tiles are keys, columns queries
template <typename T, int DP>
__global__ void __launch_bounds__(MF_NT)
masked_dkv_kernel(const MaskedParams p) {
  extern __shared__ float sm[];
  __shared__ int qdocs[MF_T], kdocs[MF_T];
  __shared__ float lses[MF_T], deltas[MF_T];
  float* Ks = sm;
  float* Vs = Ks + MF_T * (DP + 4);
  float* Qs = Vs + MF_T * (DP + 4);
  float* Cs = Qs + MF_T * (DP + 4);
  float* Ps = Cs + MF_T * (DP + 4);
  float* Ds = Ps + MF_T * MF_PP;
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const int tile = blockIdx.x % p.tiles, hk = blockIdx.x / p.tiles % p.kv_heads, b = blockIdx.x / p.tiles / p.kv_heads;
  const int group = p.heads / p.kv_heads, k0 = tile * MF_T;
  pdl_begin();
  Seq s = sequence(p.m, b, hk * group);
  float2 dk[4][DP / 64][2], dv[4][DP / 64][2];
#pragma unroll
  for (int i = 0; i < 4; i++)
#pragma unroll
    for (int j = 0; j < DP / 64; j++) dk[i][j][0] = dk[i][j][1] = dv[i][j][0] = dv[i][j][1] = make_float2(0.f, 0.f);
  load_tile<T, DP>(Ks, p.k, b, k0, hk, s.len, p.D);
  load_tile<T, DP>(Vs, p.v, b, k0, hk, s.len, p.D);
  tile_documents(p.m, s, b, k0, kdocs, 0, 0);
  int lo, hi;
  document_range(s, k0, kdocs, &lo, &hi);
  const int first = k0 < s.prefix ? 0 : k0, last = k0 >= s.len ? 0 : s.len;
  for (int h = hk * group; h < (hk + 1) * group; h++) {
    s = sequence(p.m, b, h);
    for (int q0 = first; q0 < last; q0 += MF_T) {
      __syncthreads();
      if (!tile_documents(p.m, s, b, q0, qdocs, lo, hi)) continue;
      load_tile<T, DP>(Qs, p.q, b, q0, h, s.len, p.D);
      load_tile<T, DP>(Cs, p.dc, b, q0, h, s.len, p.D);
      if (threadIdx.x < MF_T) {
        const int r = q0 + threadIdx.x;
        const int64_t at = ((int64_t)b * p.heads + h) * p.m.S + r;
        lses[threadIdx.x] = r < s.len ? p.lse[at] : 0.f;
        deltas[threadIdx.x] = r < s.len ? p.delta[at] : 0.f;
      }
      __syncthreads();
      float z[4][4], dp[4][4];
      products<DP>(Ks, Qs, ty, tx, z);
      products<DP>(Vs, Cs, ty, tx, dp);
#pragma unroll
      for (int i = 0; i < 4; i++)
#pragma unroll
        for (int c = 0; c < 4; c++) {
          const int n = tx + 16 * c, qi = q0 + n, kj = k0 + 4 * ty + i;
          float w = 0.f, ds = 0.f;
          if (sees(s, qi, kj, qdocs[n], kdocs[4 * ty + i])) {
            float bend;
            w = expf(score(p.m, s, z[i][c], qi, kj, &bend) - lses[n]);
            ds = w * (dp[i][c] - deltas[n]) * bend;
          }
          Ps[(4 * ty + i) * MF_PP + n] = w;
          Ds[(4 * ty + i) * MF_PP + n] = ds;
        }
      __syncwarp();
      accumulate<DP>(Ps, Cs, ty, tx, dv);
      accumulate<DP>(Ds, Qs, ty, tx, dk);
    }
  }
  const float one[4] = {1.f, 1.f, 1.f, 1.f};
  const float f[4] = {p.m.scale, p.m.scale, p.m.scale, p.m.scale};
  store_rows<T, DP>(p.o0, b, k0, hk, p.m.S, p.D, ty, tx, dk, f);
  store_rows<T, DP>(p.o1, b, k0, hk, p.m.S, p.D, ty, tx, dv, one);
}

template <int DP> constexpr size_t smem_bytes(int operands, int scores) {
  return ((size_t)operands * MF_T * (DP + 4) + (size_t)scores * MF_T * MF_PP) * sizeof(float);
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

Rows rows_of(const mslt_heads& h) { return Rows{h.data, h.batch, h.row, h.head}; }

MaskedParams params_of(const mslt_attention_desc& d) {
  MaskedParams p = {};
  p.m = AttnMask{d.S, d.causal != 0, d.scale, d.cap, d.slopes, d.prefix, d.docs, d.lens};
  p.q = rows_of(d.q); p.k = rows_of(d.k); p.v = rows_of(d.v);
  p.rest = d.rest;
  p.lse = d.lse; p.heads = d.heads; p.kv_heads = d.kv_heads; p.D = d.head_dim;
  p.tiles = (d.S + MF_T - 1) / MF_T;
  return p;
}

template <typename T, int DP>
int forward(const mslt_attention_desc& d, cudaStream_t st, char* err) {
  static bool done[kMaxDevices];
  constexpr size_t smem = smem_bytes<DP>(3, 1);
  if (opt_in((const void*)masked_fwd_kernel<T, DP>, done, smem, err)) return MSLT_ERR_CUDA;
  MaskedParams p = params_of(d);
  p.o0 = rows_of(d.ctx);
  launch_pdl(masked_fwd_kernel<T, DP>, d.B * d.heads * p.tiles, MF_NT, smem, st, p);
  return 0;
}

template <typename T, int DP>
int backward(const mslt_attention_desc& d, float* delta, cudaStream_t st, char* err) {
  static bool done_q[kMaxDevices], done_kv[kMaxDevices];
  constexpr size_t smem_q = smem_bytes<DP>(4, 1), smem_kv = smem_bytes<DP>(4, 2);
  if (opt_in((const void*)masked_dq_kernel<T, DP>, done_q, smem_q, err)) return MSLT_ERR_CUDA;
  if (opt_in((const void*)masked_dkv_kernel<T, DP>, done_kv, smem_kv, err)) return MSLT_ERR_CUDA;
  MaskedParams p = params_of(d);
  p.dc = rows_of(d.dctx); p.c = rows_of(d.ctx); p.delta = delta;
  const int tiles = p.tiles, rows = d.B * d.heads * d.S;
  p.tiles = rows;
  launch_pdl(masked_delta_kernel<T>, (int)(((int64_t)rows + MF_NT - 1) / MF_NT), MF_NT, 0, st, p);
  p.tiles = tiles;
  p.o0 = rows_of(d.dq);
  launch_pdl(masked_dq_kernel<T, DP>, d.B * d.heads * tiles, MF_NT, smem_q, st, p);
  p.o0 = rows_of(d.dk); p.o1 = rows_of(d.dv);
  launch_pdl(masked_dkv_kernel<T, DP>, d.B * d.kv_heads * tiles, MF_NT, smem_kv, st, p);
  return 0;
}

}  // namespace

int attn_masked_f32_fwd(const mslt_attention_desc& d, cudaStream_t st, char* err) {
  if (d.dtype == 1) return d.head_dim <= 64 ? forward<bf16, 64>(d, st, err) : forward<bf16, 128>(d, st, err);
  return d.head_dim <= 64 ? forward<float, 64>(d, st, err) : forward<float, 128>(d, st, err);
}
int attn_masked_f32_bwd(const mslt_attention_desc& d, float* delta, cudaStream_t st, char* err) {
  if (d.dtype == 1) return d.head_dim <= 64 ? backward<bf16, 64>(d, delta, st, err) : backward<bf16, 128>(d, delta, st, err);
  return d.head_dim <= 64 ? backward<float, 64>(d, delta, st, err) : backward<float, 128>(d, delta, st, err);
}

}  // namespace mslt
