// Rotary positions of query and key heads, alone or behind a normalisation of every head, and the backward pass of both.
//   rope       y = R x: pairs (x_u, x_w) turned by P f_i, scaled by a magnitude
//   norm       n = gain xh + bias, xh = (x - mean) r, r = 1 / sqrt(var + eps) over a head (mean 0 without center), y = R n
//   backward   g = R^T dy, dgain = sum g xh, dbias = sum g, h = gain g, dx = r (h - xh mean(h xh) - [center] mean(h))
// One pass: a head is read once, its statistics are sums over the few lanes that hold it, and the backward forms them
// again from x instead of reading them.  Bound by HBM: 2 (rope, norm) or 3 (backward) passes over the heads.
//
// A lane holds two pieces of W elements of a head such that both elements of every pair are its own: pieces half a rotation
// apart, or side by side where neighbours are paired (and the rest of the head likewise).  So nothing is exchanged but
// the norm's sums, and the lane's pairs are W neighbours of the table in either layout.  W is 4 in either type: 8 bf16 a
// piece measure the same for the rotation alone (19.0 against 19.1 us at 16384 rows x 24 heads x 64) and leave the norm's
// backward too few registers (77 against 55 us at the time).  The angle of a pair depends on row and pair only: a warp works three
// groups of heads of a row with one set of cosines and sines, asks for all of their bytes before it forms them, and takes
// the three sums of a norm side by side.  (One 16-byte piece a lane and the partner's values through shuffles: twice the
// sines, 32 us.)  Angles: the table holds turns a position as 64-bit fractions, position times table modulo 2^64 is the turn's
// fraction without any rounding that grows with the position, and its upper 32 bits go to the sine.  In bf16 the sine is
// the hardware's (absolute error 2^-21 on [-pi, pi], an eighth of a thousandth of the result's rounding 2^-9); in fp32
// the library's sincospif.
#include <math.h>

#include "common.cuh"
#include "op_check.h"

namespace mslt {
namespace {

constexpr int RO_WARPS = 8;
constexpr int RO_MAX_BLOCKS = 1184;  // blocks of the backward pass that leave partial sums

struct RotaryParams {
  const void *x, *dy;
  void *y, *dx;
  int64_t x_row, x_head, y_row, y_head, dy_row, dy_head, dx_row, dx_head;
  const int32_t* positions;
  const uint64_t* turns;
  const float *gain, *bias;
  float* partial;  // backward: [blocks][2][D]: dgain, dbias
  int rows, heads, q_heads, D, seq, rot, log_lanes, passes, q_slots, center;
  float magnitude, sign, eps;
};

constexpr int W = 4;  // elements of a piece, in pairs for packed arithmetic

template <typename T> struct Piece;
template <> struct Piece<float> {
  typedef float4 Raw;
  static __device__ __forceinline__ void unpack(const Raw& r, float2 (&v)[2]) {
    v[0] = make_float2(r.x, r.y);
    v[1] = make_float2(r.z, r.w);
  }
  static __device__ __forceinline__ void store(float* p, const float2 (&v)[2]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
  }
};
template <> struct Piece<bf16> {
  typedef uint2 Raw;
  static __device__ __forceinline__ void unpack(const Raw& r, float2 (&v)[2]) {
    v[0] = make_float2(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u));
    v[1] = make_float2(__uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u));
  }
  static __device__ __forceinline__ void store(bf16* p, const float2 (&v)[2]) {
    uint2 r;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&r);
    h[0] = __floats2bfloat162_rn(v[0].x, v[0].y);
    h[1] = __floats2bfloat162_rn(v[1].x, v[1].y);
    *reinterpret_cast<uint2*>(p) = r;
  }
};
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 pair_at(const float* p) { return *reinterpret_cast<const float2*>(p); }

__device__ __forceinline__ void turn_of(int pos, uint64_t turns, bool exact, float& s, float& c) {
  const int32_t f = (int32_t)(((uint64_t)(int64_t)pos * turns) >> 32);
  const float t = (float)f * 2.3283064365386963e-10f;  // 2^-32: in [-1/2, 1/2)
  if (exact) {
    sincospif(2.0f * t, &s, &c);
  } else {
    const float a = t * 6.2831853071795865f;
    s = __sinf(a);
    c = __cosf(a);
  }
}

// Sums over the lanes of a head, of all passes side by side
template <int N>
__device__ __forceinline__ void lanes_sum(float (&v)[N], int lanes) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < lanes) {
#pragma unroll
      for (int k = 0; k < N; k++) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    }
}

// The lane's pairs turned: (a_j, b_j), or the neighbours in a and in b; c, s, minus s by pair.  What does not turn is left as it is.
// kPacked: two pairs an instruction, where the norms' instructions count; the rotation alone has no registers for minus s.
template <bool INTER, bool kPacked>
__device__ __forceinline__ void rotate(float2 (&a)[2], float2 (&b)[2], const float2 (&c)[2], const float2 (&s)[2], const float2 (&ms)[2],
                                       bool turn_a, bool turn_b) {
  if (INTER) {
    auto turn = [](float2& v, float cs, float sn) { v = make_float2(fmaf(-v.y, sn, v.x * cs), fmaf(v.x, sn, v.y * cs)); };
    if (turn_a) {
      turn(a[0], c[0].x, s[0].x);
      turn(a[1], c[0].y, s[0].y);
    }
    if (turn_b) {
      turn(b[0], c[1].x, s[1].x);
      turn(b[1], c[1].y, s[1].y);
    }
  } else if (turn_a) {
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const float2 u = a[j], w = b[j];
      if (kPacked) {
        a[j] = __ffma2_rn(w, ms[j], __fmul2_rn(u, c[j]));
        b[j] = __ffma2_rn(u, s[j], __fmul2_rn(w, c[j]));
      } else {
        a[j] = make_float2(fmaf(-w.x, s[j].x, u.x * c[j].x), fmaf(-w.y, s[j].y, u.y * c[j].y));
        b[j] = make_float2(fmaf(u.x, s[j].x, w.x * c[j].x), fmaf(u.y, s[j].y, w.y * c[j].y));
      }
    }
  }
}

// OP 0: rotation, 1: norm and rotation, 2: backward of 1.  A warp takes the heads of a row in passes of `together`; in the
// backward queries and keys are taken by different blocks (grid y), each with one set of sums in registers.
// PASSES, and BLOCKS of 256 threads on an SM (80 or 128 registers), were tried together; 16384 rows x 24 heads x 64 and 8144 x 20
// x 128, us: rotation 3 x 4 18.9 and 16.0, 3 x 3 19.7 and 18.5, 2 x 3 20.3 and 16.1; norm 2 x 3 24.9 and 21.5, 3 x 3 29 and
// 22.5, 2 x 4 27 and 19.8; backward 3 x 2 40.0 and 39.4 (43.6 and 42.1 without packed arithmetic), 2 x 3 63 and 43.  Rotation in
// fp32, 8168 x 32 x 64: 4 x 2 24.5, 2 x 3 24.9, 4 x 3 28.4, 3 x 4 31.1.  Asking for a row ahead gained nothing at any of them.
template <typename T, int OP> struct Shape {
  static constexpr bool wide = sizeof(T) == 4 && OP == 0;
  static constexpr int PASSES = wide ? 4 : OP == 1 ? 2 : 3, BLOCKS = wide ? 2 : OP == 0 ? 4 : OP == 1 ? 3 : 2;
};

template <typename T, bool INTER, int OP>
__global__ void __launch_bounds__(32 * RO_WARPS, (Shape<T, OP>::BLOCKS))
rotary_kernel(const RotaryParams p) {
  constexpr bool kExact = sizeof(T) == 4;
  constexpr int PASSES = Shape<T, OP>::PASSES;
  typedef Piece<T> Pc;
  typedef typename Pc::Raw Raw;
  __shared__ __align__(16) uint64_t turns[64];
  __shared__ __align__(16) float gains[OP >= 1 ? 2 : 1][128], biases[OP == 1 ? 2 : 1][128];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int lanes = 1 << p.log_lanes, o = (lane & (lanes - 1)) * W, half = p.rot >> 1;
  const int sub = lane >> p.log_lanes, together = 32 >> p.log_lanes;
  const bool live = o < p.D / 2;
  const int ea = INTER ? 2 * o : o < half ? o : half + o;                        // half + o = rot + (o - half)
  const int eb = INTER ? 2 * o + W : o < half ? half + o : p.D / 2 + o;          // rot + (D - rot) / 2 + (o - half)
  const bool turn_a = live && (INTER ? ea < p.rot : o < half), turn_b = live && (INTER ? eb < p.rot : o < half);
  const int slot = blockIdx.y, kind = OP == 2 && slot >= p.q_slots;
  const int h0 = (kind ? p.q_heads + (slot - p.q_slots) * together * p.passes : slot * together * p.passes) + sub;
  const int h1 = OP < 2 || kind ? p.heads : p.q_heads;
  const float inv_d = 1.0f / (float)p.D;
  pdl_begin();
  for (int i = threadIdx.x; i < 64; i += 32 * RO_WARPS) turns[i] = i < half ? p.turns[i] : 0;
  if (OP >= 1) {
    for (int i = threadIdx.x; i < 2 * p.D; i += 32 * RO_WARPS) {
      const int k = i >= p.D;
      gains[k][i - k * p.D] = p.gain[i];
      if (OP == 1) biases[k][i - k * p.D] = p.bias ? p.bias[i] : 0.f;
    }
  }
  __syncthreads();
  float2 dga[2], dgb[2], dba[2], dbb[2];
#pragma unroll
  for (int j = 0; j < 2; j++) dga[j] = dgb[j] = dba[j] = dbb[j] = make_float2(0.f, 0.f);

  const T* x0 = (const T*)p.x + h0 * p.x_head;
  const T* d0 = (const T*)p.dy + h0 * p.dy_head;
  T* out0 = OP == 2 ? (T*)p.dx + h0 * p.dx_head : (T*)p.y + h0 * p.y_head;
  const int64_t x_step = together * p.x_head, d_step = together * p.dy_head;
  const int64_t out_row = OP == 2 ? p.dx_row : p.y_row, out_step = together * (OP == 2 ? p.dx_head : p.y_head);
  bool here[PASSES];
#pragma unroll
  for (int k = 0; k < PASSES; k++) here[k] = k < p.passes && live && h0 + k * together < h1;

  for (int row = (int)blockIdx.x * RO_WARPS + warp; row < p.rows; row += (int)gridDim.x * RO_WARPS) {
    Raw xa[PASSES], xb[PASSES], da[PASSES], db[PASSES];
    const int pos = p.positions ? p.positions[row] : row % p.seq;
#pragma unroll
    for (int k = 0; k < PASSES; k++) {
      xa[k] = xb[k] = da[k] = db[k] = Raw();
      if (here[k]) {
        const T* x = x0 + row * p.x_row + k * x_step;
        xa[k] = *reinterpret_cast<const Raw*>(x + ea);
        xb[k] = *reinterpret_cast<const Raw*>(x + eb);
        if (OP == 2) {
          const T* d = d0 + row * p.dy_row + k * d_step;
          da[k] = *reinterpret_cast<const Raw*>(d + ea);
          db[k] = *reinterpret_cast<const Raw*>(d + eb);
        }
      }
    }
    float2 c[2], s[2], ms[2];
#pragma unroll
    for (int j = 0; j < 2; j++) {
      turn_of(pos, turns[(o + 2 * j) & 63], kExact, s[j].x, c[j].x);
      turn_of(pos, turns[(o + 2 * j + 1) & 63], kExact, s[j].y, c[j].y);
      ms[j] = __fmul2_rn(s[j], both(-p.sign * p.magnitude));
      s[j] = __fmul2_rn(s[j], both(p.sign * p.magnitude));
      c[j] = __fmul2_rn(c[j], both(p.magnitude));
    }
    float mean[PASSES], r[PASSES];
    if (OP >= 1) {
#pragma unroll
      for (int k = 0; k < PASSES; k++) mean[k] = r[k] = 0.f;
      if (p.center) {
#pragma unroll
        for (int k = 0; k < PASSES; k++) {
          float2 a[2], b[2];
          Pc::unpack(xa[k], a);
          Pc::unpack(xb[k], b);
          const float2 t = __fadd2_rn(__fadd2_rn(a[0], a[1]), __fadd2_rn(b[0], b[1]));
          mean[k] = t.x + t.y;
        }
        lanes_sum(mean, lanes);
#pragma unroll
        for (int k = 0; k < PASSES; k++) mean[k] = here[k] ? mean[k] * inv_d : 0.f;  // an idle lane's zeros stay zeros
      }
#pragma unroll
      for (int k = 0; k < PASSES; k++) {
        float2 a[2], b[2], t = make_float2(0.f, 0.f);
        Pc::unpack(xa[k], a);
        Pc::unpack(xb[k], b);
#pragma unroll
        for (int j = 0; j < 2; j++) {
          a[j] = __fadd2_rn(a[j], both(-mean[k]));
          b[j] = __fadd2_rn(b[j], both(-mean[k]));
          t = __ffma2_rn(a[j], a[j], t);
          t = __ffma2_rn(b[j], b[j], t);
        }
        r[k] = t.x + t.y;
      }
      lanes_sum(r, lanes);
#pragma unroll
      for (int k = 0; k < PASSES; k++) r[k] = rsqrtf(fmaf(r[k], inv_d, p.eps));
    }
    if (OP == 2) {
      float2 a[PASSES][2], b[PASSES][2], u[PASSES][2], w[PASSES][2], ga[2], gb[2];
      float m1[PASSES], m2[PASSES];
#pragma unroll
      for (int j = 0; j < 2; j++) {
        ga[j] = live ? pair_at(&gains[kind][ea + 2 * j]) : make_float2(0.f, 0.f);
        gb[j] = live ? pair_at(&gains[kind][eb + 2 * j]) : make_float2(0.f, 0.f);
      }
#pragma unroll
      for (int k = 0; k < PASSES; k++) {
        Pc::unpack(xa[k], a[k]);
        Pc::unpack(xb[k], b[k]);
        Pc::unpack(da[k], u[k]);
        Pc::unpack(db[k], w[k]);
        rotate<INTER, (OP >= 1)>(u[k], w[k], c, s, ms, turn_a, turn_b);
        float2 t1 = make_float2(0.f, 0.f), t2 = t1;
#pragma unroll
        for (int j = 0; j < 2; j++) {
          a[k][j] = __fmul2_rn(__fadd2_rn(a[k][j], both(-mean[k])), both(r[k]));  // xh
          b[k][j] = __fmul2_rn(__fadd2_rn(b[k][j], both(-mean[k])), both(r[k]));
          dga[j] = __ffma2_rn(u[k][j], a[k][j], dga[j]);
          dgb[j] = __ffma2_rn(w[k][j], b[k][j], dgb[j]);
          dba[j] = __fadd2_rn(dba[j], u[k][j]);
          dbb[j] = __fadd2_rn(dbb[j], w[k][j]);
          u[k][j] = __fmul2_rn(u[k][j], ga[j]);
          w[k][j] = __fmul2_rn(w[k][j], gb[j]);
          t1 = __ffma2_rn(u[k][j], a[k][j], t1);
          t1 = __ffma2_rn(w[k][j], b[k][j], t1);
          t2 = __fadd2_rn(t2, __fadd2_rn(u[k][j], w[k][j]));
        }
        m1[k] = t1.x + t1.y;
        m2[k] = t2.x + t2.y;
      }
      lanes_sum(m1, lanes);
      if (p.center) lanes_sum(m2, lanes);
#pragma unroll
      for (int k = 0; k < PASSES; k++) {
        m1[k] *= -inv_d;
        m2[k] = p.center ? m2[k] * -inv_d : 0.f;
#pragma unroll
        for (int j = 0; j < 2; j++) {
          a[k][j] = __fmul2_rn(both(r[k]), __ffma2_rn(a[k][j], both(m1[k]), __fadd2_rn(u[k][j], both(m2[k]))));
          b[k][j] = __fmul2_rn(both(r[k]), __ffma2_rn(b[k][j], both(m1[k]), __fadd2_rn(w[k][j], both(m2[k]))));
        }
        if (here[k]) {
          T* out = out0 + row * out_row + k * out_step;
          Pc::store(out + ea, a[k]);
          Pc::store(out + eb, b[k]);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < PASSES; k++) {
        if (!here[k]) continue;
        float2 a[2], b[2];
        Pc::unpack(xa[k], a);
        Pc::unpack(xb[k], b);
        if (OP == 1) {
          const int kd = h0 + k * together >= p.q_heads;
#pragma unroll
          for (int j = 0; j < 2; j++) {
            a[j] = __fmul2_rn(__fadd2_rn(a[j], both(-mean[k])), both(r[k]));
            b[j] = __fmul2_rn(__fadd2_rn(b[j], both(-mean[k])), both(r[k]));
            const float2 ga = pair_at(&gains[kd][ea + 2 * j]), gb = pair_at(&gains[kd][eb + 2 * j]);
            if (p.bias) {
              a[j] = __ffma2_rn(a[j], ga, pair_at(&biases[kd][ea + 2 * j]));
              b[j] = __ffma2_rn(b[j], gb, pair_at(&biases[kd][eb + 2 * j]));
            } else {
              a[j] = __fmul2_rn(a[j], ga);
              b[j] = __fmul2_rn(b[j], gb);
            }
          }
        }
        rotate<INTER, (OP >= 1)>(a, b, c, s, ms, turn_a, turn_b);
        T* out = out0 + row * out_row + k * out_step;
        Pc::store(out + ea, a);
        Pc::store(out + eb, b);
      }
    }
  }

  if (OP == 2) {  // the block's sums, warps and groups in order
    __shared__ __align__(16) float part[RO_WARPS][2][64 * W];  // together * D <= 64 W
    if (live) {
#pragma unroll
      for (int j = 0; j < 2; j++) {
        *reinterpret_cast<float2*>(&part[warp][0][sub * p.D + ea + 2 * j]) = dga[j];
        *reinterpret_cast<float2*>(&part[warp][0][sub * p.D + eb + 2 * j]) = dgb[j];
        *reinterpret_cast<float2*>(&part[warp][1][sub * p.D + ea + 2 * j]) = dba[j];
        *reinterpret_cast<float2*>(&part[warp][1][sub * p.D + eb + 2 * j]) = dbb[j];
      }
    }
    __syncthreads();
    float* out = p.partial + (int64_t)(blockIdx.y * gridDim.x + blockIdx.x) * 2 * p.D;
    for (int i = threadIdx.x; i < 2 * p.D; i += 32 * RO_WARPS) {
      const int which = i >= p.D, col = i - which * p.D;
      float sum = 0.f;
      for (int w = 0; w < RO_WARPS; w++)
        for (int t = 0; t < together; t++) sum += part[w][which][t * p.D + col];
      out[i] = sum;
    }
  }
}

// Sums of the blocks' sums, in order: 32 columns a block, 32 threads each, added in double.
__global__ void __launch_bounds__(1024) rotary_sum_kernel(const float* partial, int D, int q_blocks, int blocks, float* dgain,
                                                          float* dbias) {
  __shared__ double part[32][33];
  pdl_begin();
  const int col = (int)blockIdx.x * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5, kind = blockIdx.y;
  const int b1 = kind ? blocks : q_blocks;
  double sum = 0.;
  if (col < 2 * D)
#pragma unroll 4
    for (int b = (kind ? q_blocks : 0) + lane; b < b1; b += 32) sum += (double)partial[(int64_t)b * 2 * D + col];
  part[lane][threadIdx.x & 31] = sum;
  __syncthreads();
  if (lane == 0 && col < 2 * D) {
    sum = 0.;
    for (int i = 0; i < 32; i++) sum += part[i][threadIdx.x];
    float* out = col < D ? dgain : dbias;
    if (out) out[kind * D + (col < D ? col : col - D)] = (float)sum;
  }
}

int ceil_div(int a, int b) { return (a + b - 1) / b; }

// passes: a warp takes up to PASSES groups of heads, fewer where the launch would have too few warps to fill the
// device (latency counts there, and the angles cost little).
struct RotaryLaunch { dim3 grid; int q_blocks; };
RotaryLaunch plan_rotary(RotaryParams& p, int most_passes, int blocks_per_sm, int sms, bool by_kind) {
  p.log_lanes = 0;
  while ((2 * W << p.log_lanes) < p.D) p.log_lanes++;
  const int together = 32 >> p.log_lanes;
  const int first = by_kind ? p.q_heads : p.heads, second = p.heads - first;
  int slots = 0;
  for (p.passes = most_passes; p.passes >= 1; p.passes--) {
    p.q_slots = ceil_div(first, together * p.passes);
    slots = p.q_slots + ceil_div(second, together * p.passes);
    if (p.passes == 1 || (int64_t)p.rows * slots >= (int64_t)sms * RO_WARPS * blocks_per_sm) break;
  }
  const int most = sms * blocks_per_sm > RO_MAX_BLOCKS ? RO_MAX_BLOCKS : sms * blocks_per_sm;
  int gx = most / slots;
  if (gx < 1) gx = 1;
  if (gx > ceil_div(p.rows, RO_WARPS)) gx = ceil_div(p.rows, RO_WARPS);
  RotaryLaunch l;
  l.grid = dim3(gx, slots);
  l.q_blocks = gx * p.q_slots;
  return l;
}

template <int OP>
RotaryLaunch run_rotary(const mslt_rope_desc& d, RotaryParams& p, int sms, cudaStream_t st) {
  const RotaryLaunch l = d.dtype == 1 ? plan_rotary(p, Shape<bf16, OP>::PASSES, Shape<bf16, OP>::BLOCKS, sms, OP == 2)
                                      : plan_rotary(p, Shape<float, OP>::PASSES, Shape<float, OP>::BLOCKS, sms, OP == 2);
  if (d.dtype == 1) {
    if (d.interleaved) launch_pdl(rotary_kernel<bf16, true, OP>, l.grid, 32 * RO_WARPS, 0, st, p);
    else launch_pdl(rotary_kernel<bf16, false, OP>, l.grid, 32 * RO_WARPS, 0, st, p);
  } else {
    if (d.interleaved) launch_pdl(rotary_kernel<float, true, OP>, l.grid, 32 * RO_WARPS, 0, st, p);
    else launch_pdl(rotary_kernel<float, false, OP>, l.grid, 32 * RO_WARPS, 0, st, p);
  }
  return l;
}

// the strides of a single row and of a single head are not used
int check_strided(const char* what, const char* name, const mslt_rope_desc& d, const void* ptr, int64_t row, int64_t head, bool output) {
  const int dtype = d.dtype;
  if (d.rows == 1) row = 0;
  if (d.heads == 1) head = 0;
  const int unit = dtype == 1 ? 8 : 4;
  if (!ptr) return op_refuse(MSLT_ERR_ARG, "%s: %s is null", what, name);
  if ((uintptr_t)ptr & 15) return op_refuse(MSLT_ERR_ARG, "%s: %s must be 16-byte aligned", what, name);
  if (row % unit || head % unit || row < 0 || head < 0)
    return op_refuse(MSLT_ERR_ARG, "%s: strides of %s must be multiples of 16 bytes", what, name);
  if (output && ((d.rows > 1 && row < d.head_dim) || (d.heads > 1 && head < d.head_dim)))
    return op_refuse(MSLT_ERR_ARG, "%s: strides of %s must be at least head_dim", what, name);
  return 0;
}

int check_rope(const char* what, const mslt_rope_desc* d, int rot_min) {
  if (!d) return op_refuse(MSLT_ERR_ARG, "%s: null descriptor", what);
  if (d->dtype != 0 && d->dtype != 1) return op_refuse(MSLT_ERR_ARG, "%s: dtype must be 0 or 1", what);
  if (d->rows < 1 || d->heads < 1) return op_refuse(MSLT_ERR_ARG, "%s: rows and heads must be >= 1", what);
  if (d->heads > 4096 || d->rows > (1 << 30)) return op_refuse(MSLT_ERR_SIZE, "%s: at most 4096 heads and 2^30 rows", what);
  if (d->head_dim < 8 || d->head_dim > 128 || d->head_dim % 8)
    return op_refuse(MSLT_ERR_ARG, "%s: head_dim must be a multiple of 8 in [8, 128]", what);
  if (d->rot_dim < rot_min || d->rot_dim > d->head_dim || d->rot_dim % 8)
    return op_refuse(MSLT_ERR_ARG, "%s: rot_dim must be a multiple of 8 in [%d, head_dim]", what, rot_min);
  if (d->rot_dim > 0 && (!d->turns || ((uintptr_t)d->turns & 15)))
    return op_refuse(MSLT_ERR_ARG, "%s: turns must be 16-byte aligned and not null", what);
  if (!d->positions && d->seq < 1) return op_refuse(MSLT_ERR_ARG, "%s: without positions seq must be >= 1", what);
  if (!isfinite(d->magnitude)) return op_refuse(MSLT_ERR_ARG, "%s: magnitude must be finite", what);
  return check_strided(what, "x", *d, d->x, d->x_row, d->x_head, false);
}

void fill_rope(const mslt_rope_desc& d, RotaryParams& p) {
  p = RotaryParams();
  p.x = d.x; p.y = d.y;
  p.x_row = d.x_row; p.x_head = d.x_head; p.y_row = d.y_row; p.y_head = d.y_head;
  p.positions = d.positions; p.turns = d.turns;
  p.rows = d.rows; p.heads = p.q_heads = d.heads; p.D = d.head_dim; p.seq = d.seq > 0 ? d.seq : 1; p.rot = d.rot_dim;
  p.magnitude = d.magnitude; p.sign = d.inverse ? -1.f : 1.f;
}

int check_norm(const char* what, const mslt_qk_norm_desc* d) {
  if (!d) return op_refuse(MSLT_ERR_ARG, "%s: null descriptor", what);
  int rc = check_rope(what, &d->rope, 0);
  if (rc) return rc;
  if (d->rope.inverse) return op_refuse(MSLT_ERR_ARG, "%s: inverse must be 0", what);
  if (d->q_heads < 0 || d->q_heads > d->rope.heads) return op_refuse(MSLT_ERR_ARG, "%s: q_heads must be in [0, heads]", what);
  if (!(d->eps > 0) || !isfinite(d->eps)) return op_refuse(MSLT_ERR_ARG, "%s: eps must be > 0", what);
  if (!d->gain) return op_refuse(MSLT_ERR_ARG, "%s: gain is null", what);
  return 0;
}

void fill_norm(const mslt_qk_norm_desc& d, RotaryParams& p) {
  fill_rope(d.rope, p);
  p.q_heads = d.q_heads; p.center = d.center != 0; p.eps = d.eps; p.gain = d.gain; p.bias = d.bias;
}

int sm_count(int* sms) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return op_refuse(MSLT_ERR_CUDA, "device attributes: %s", cudaGetErrorString(e));
  return 0;
}

}  // namespace
}  // namespace mslt

using namespace mslt;

extern "C" {

int mslt_rope_turns(int32_t rot_dim, double base, int32_t scaling, double factor, int32_t trained_len, uint64_t* host_turns,
                    float* magnitude) {
  if (!host_turns || !magnitude) return op_refuse(MSLT_ERR_ARG, "rope_turns: null pointer");
  if (rot_dim < 8 || rot_dim % 8 || rot_dim > 128) return op_refuse(MSLT_ERR_ARG, "rope_turns: rot_dim must be a multiple of 8 in [8, 128]");
  if (!(base > 1.0) || !isfinite(base)) return op_refuse(MSLT_ERR_ARG, "rope_turns: base must be > 1");
  if (scaling < 0 || scaling > 3) return op_refuse(MSLT_ERR_ARG, "rope_turns: scaling must be in [0, 3]");
  if (!(factor >= 1.0) || !isfinite(factor)) return op_refuse(MSLT_ERR_ARG, "rope_turns: factor must be >= 1");
  if (scaling == 3 && trained_len < 1) return op_refuse(MSLT_ERR_ARG, "rope_turns: trained_len must be >= 1");
  const double two_pi = 6.283185307179586476925;
  if (scaling == 2) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
  for (int i = 0; i < rot_dim / 2; i++) {
    double f = pow(base, -2.0 * i / rot_dim);
    if (scaling == 1) f /= factor;
    if (scaling == 3) {
      double keep = (trained_len * f / two_pi - 1.0) / 31.0;
      keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
      f = f * keep + f / factor * (1 - keep);
    }
    host_turns[i] = (uint64_t)llround(ldexp(f / two_pi, 64));  // f <= 1: below 2^62
  }
  *magnitude = scaling == 3 ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
  return 0;
}

int mslt_op_rope(const mslt_rope_desc* desc, void* cuda_stream, int32_t sync) {
  int rc = check_rope("rope", desc, 8);
  if (rc) return rc;
  rc = check_strided("rope", "y", *desc, desc->y, desc->y_row, desc->y_head, true);
  if (rc) return rc;
  int sms = 0;
  if ((rc = op_need_device()) || (rc = sm_count(&sms))) return rc;
  RotaryParams p;
  fill_rope(*desc, p);
  run_rotary<0>(*desc, p, sms, (cudaStream_t)cuda_stream);
  return op_end("rope", (cudaStream_t)cuda_stream, sync);
}

int mslt_op_qk_norm_rope(const mslt_qk_norm_desc* desc, void* cuda_stream, int32_t sync) {
  int rc = check_norm("qk_norm_rope", desc);
  if (rc) return rc;
  rc = check_strided("qk_norm_rope", "y", desc->rope, desc->rope.y, desc->rope.y_row, desc->rope.y_head, true);
  if (rc) return rc;
  int sms = 0;
  if ((rc = op_need_device()) || (rc = sm_count(&sms))) return rc;
  RotaryParams p;
  fill_norm(*desc, p);
  run_rotary<1>(desc->rope, p, sms, (cudaStream_t)cuda_stream);
  return op_end("qk_norm_rope", (cudaStream_t)cuda_stream, sync);
}

size_t mslt_op_qk_norm_rope_bwd_scratch_bytes(int32_t rows, int32_t heads, int32_t head_dim) {
  if (rows < 1 || heads < 1 || head_dim < 1) return 0;
  // at least one block for every group of heads, and there are no more groups than heads
  const size_t blocks = heads > RO_MAX_BLOCKS ? heads : RO_MAX_BLOCKS;
  return blocks * 2 * (size_t)head_dim * sizeof(float);
}

int mslt_op_qk_norm_rope_bwd(const mslt_qk_norm_desc* desc, void* d_scratch, size_t scratch_bytes, void* cuda_stream,
                             int32_t sync) {
  const char* what = "qk_norm_rope_bwd";
  int rc = check_norm(what, desc);
  if (rc) return rc;
  if ((rc = check_strided(what, "dy", desc->rope, desc->dy, desc->dy_row, desc->dy_head, false))) return rc;
  if ((rc = check_strided(what, "dx", desc->rope, desc->dx, desc->dx_row, desc->dx_head, true))) return rc;
  if (!desc->dgain) return op_refuse(MSLT_ERR_ARG, "%s: dgain is null", what);
  const size_t need = mslt_op_qk_norm_rope_bwd_scratch_bytes(desc->rope.rows, desc->rope.heads, desc->rope.head_dim);
  if (!d_scratch || scratch_bytes < need || ((uintptr_t)d_scratch & 15))
    return op_refuse(MSLT_ERR_SIZE, "%s: scratch must be 16-byte aligned and hold %zu bytes", what, need);
  int sms = 0;
  if ((rc = op_need_device()) || (rc = sm_count(&sms))) return rc;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  RotaryParams p;
  fill_norm(*desc, p);
  p.sign = -1.f;
  p.dy = desc->dy; p.dy_row = desc->dy_row; p.dy_head = desc->dy_head;
  p.dx = desc->dx; p.dx_row = desc->dx_row; p.dx_head = desc->dx_head;
  p.partial = (float*)d_scratch;
  const RotaryLaunch l = run_rotary<2>(desc->rope, p, sms, st);
  launch_pdl(rotary_sum_kernel, dim3(ceil_div(2 * p.D, 32), 2), 1024, 0, st, (const float*)p.partial, p.D, l.q_blocks,
             (int)(l.grid.x * l.grid.y), desc->dgain, desc->dbias);
  return op_end(what, st, sync);
}

}  // extern "C"
