// Rotary positions of query and key heads, alone or behind a normalisation of every head, and the backward pass of both.
//   rope       y = R x: pairs (x_u, x_w) turned by P f_i, scaled by a magnitude
//   norm       n = gain xh + bias, xh = (x - mean) r, r = 1 / sqrt(var + eps) over a head (mean 0 without center), y = R n
//   backward   g = R^T dy, dgain = sum g xh, dbias = sum g, h = gain g, dx = r (h - xh mean(h xh) - [center] mean(h))
// One pass: a head is read once, its statistics are sums over the few lanes that hold it, and the backward forms them
// again from x instead of reading them.  Bound by HBM: 2 (rope, norm) or 3 (backward) passes over the heads.
//
// A lane holds 16 bytes of a head, the next power of two of lanes a head, so a warp has 32 / lanes heads of one row at a
// time.  The angle of a pair depends on row and pair only: a warp works up to four such groups of heads with one set of
// cosines and sines, and asks for all of their bytes before it forms them.  Angles: the table holds turns a position as
// 64-bit fractions, position times table modulo 2^64 is the turn's fraction without any rounding that grows with the
// position, and its upper 32 bits go to the sine.  In bf16 the sine is the hardware's (absolute error 2^-21 on
// [-pi, pi], an eighth of a thousandth of the result's rounding 2^-9); in fp32 the library's sincospif.
// Pairs at distance rot / 2 exchange their values through shuffles.  rot is a multiple of 8, so that distance is a number
// of four-element quads and a lane's quads each come from one lane.
#include <math.h>

#include "common.cuh"
#include "op_check.h"

namespace mslt {
namespace {

constexpr int RO_WARPS = 8;
constexpr int RO_PASSES = 4;         // groups of heads that a warp has under way
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

__device__ __forceinline__ float lanes_sum(float v, int log_lanes) {
  for (int o = (1 << log_lanes) >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// v <- c v + s (partner of v): the rotation, with the sign of each element's side in s
template <int V, bool INTER>
__device__ __forceinline__ void rotate(float (&v)[V], const float (&c)[V], const float (&s)[V], const int (&src)[V / 4], bool odd) {
  float w[V];
  if (INTER) {
#pragma unroll
    for (int j = 0; j < V; j++) w[j] = v[j ^ 1];
  } else {
#pragma unroll
    for (int q = 0; q < V / 4; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        // an odd distance in quads: the partner lies in the other quad of its lane
        const float give = V == 8 && odd ? v[(4 * q + j) ^ (V - 4)] : v[4 * q + j];
        w[4 * q + j] = __shfl_sync(0xffffffffu, give, src[q]);
      }
  }
#pragma unroll
  for (int j = 0; j < V; j++) v[j] = fmaf(s[j], w[j], c[j] * v[j]);
}

// OP 0: rotation, 1: norm and rotation, 2: backward of 1
template <typename T, bool INTER, int OP>
__global__ void __launch_bounds__(32 * RO_WARPS, 2)
rotary_kernel(const RotaryParams p) {
  constexpr int V = VecT<T>::N, NT = INTER ? V / 2 : V;
  constexpr bool kExact = sizeof(T) == 4;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int lanes = 1 << p.log_lanes, g = lane & (lanes - 1), e = g * V;
  const int sub = lane >> p.log_lanes, together = 32 >> p.log_lanes;
  const bool live = e < p.D, turned = live && e < p.rot;
  const int slot = blockIdx.y, kind = slot >= p.q_slots;
  const int h0 = (kind ? p.q_heads + (slot - p.q_slots) * together * p.passes : slot * together * p.passes) + sub;
  const int h1 = kind ? p.heads : p.q_heads;
  const float inv_d = 1.0f / (float)p.D;
  const int half = p.rot >> 1;
  int src[V / 4];
#pragma unroll
  for (int q = 0; q < V / 4; q++) {
    const int e0 = e + 4 * q;
    const int pe = e0 < half ? e0 + half : e0 - half;
    src[q] = live && e0 < p.rot ? (lane - g) + pe / V : lane;
  }
  const bool odd = (half & 4) != 0;
  pdl_begin();

  uint64_t turns[NT];
#pragma unroll
  for (int j = 0; j < NT; j += 2) {
    int i;
    bool act;
    if (INTER) {
      i = e / 2 + j;
      act = turned;
    } else {
      const int e0 = e + (j & ~3);
      act = live && e0 < p.rot;
      i = (e0 < half ? e0 : e0 - half) + (j & 3);
    }
    ulonglong2 t = make_ulonglong2(0, 0);
    if (act) t = *reinterpret_cast<const ulonglong2*>(p.turns + i);
    turns[j] = t.x;
    turns[j + 1] = t.y;
  }
  float gain[V], bias[V], dgain[V], dbias[V];
  if (OP >= 1) {
#pragma unroll
    for (int j = 0; j < V; j++) {
      gain[j] = live ? p.gain[kind * p.D + e + j] : 0.f;
      bias[j] = OP == 1 && live && p.bias ? p.bias[kind * p.D + e + j] : 0.f;
      dgain[j] = dbias[j] = 0.f;
    }
  }

  for (int row = (int)blockIdx.x * RO_WARPS + warp; row < p.rows; row += (int)gridDim.x * RO_WARPS) {
    typename VecT<T>::Raw rx[RO_PASSES], rd[RO_PASSES];
    const int pos = p.positions ? p.positions[row] : row % p.seq;
#pragma unroll
    for (int k = 0; k < RO_PASSES; k++) {
      const int h = h0 + k * together;
      if (k < p.passes && live && h < h1) {
        rx[k] = VecT<T>::load_raw((const T*)p.x + row * p.x_row + h * p.x_head + e);
        if (OP == 2) rd[k] = VecT<T>::load_raw((const T*)p.dy + row * p.dy_row + h * p.dy_head + e);
      }
    }
    float c[V], s[V];
#pragma unroll
    for (int j = 0; j < NT; j++) {
      float sn, cs;
      turn_of(pos, turns[j], kExact, sn, cs);
      sn *= p.sign * p.magnitude;
      cs *= p.magnitude;
      if (INTER) {
        c[2 * j] = turned ? cs : 1.f;
        c[2 * j + 1] = c[2 * j];
        s[2 * j + 1] = turned ? sn : 0.f;
        s[2 * j] = -s[2 * j + 1];
      } else {
        const int e0 = e + (j & ~3);
        const bool act = e0 < p.rot;
        c[j] = act ? cs : 1.f;
        s[j] = !act ? 0.f : e0 < half ? -sn : sn;
      }
    }
#pragma unroll
    for (int k = 0; k < RO_PASSES; k++) {
      if (k >= p.passes) break;
      const int h = h0 + k * together;
      const bool here = live && h < h1;
      float v[V];
#pragma unroll
      for (int j = 0; j < V; j++) v[j] = 0.f;
      if (here) VecT<T>::unpack(rx[k], v);
      if (OP >= 1) {
        float mean = 0.f, sum = 0.f;
        if (p.center) {
#pragma unroll
          for (int j = 0; j < V; j++) sum += v[j];
          mean = lanes_sum(sum, p.log_lanes) * inv_d;
        }
        sum = 0.f;
#pragma unroll
        for (int j = 0; j < V; j++) {
          if (here) v[j] -= mean;
          sum = fmaf(v[j], v[j], sum);
        }
        const float r = 1.0f / sqrtf(fmaf(lanes_sum(sum, p.log_lanes), inv_d, p.eps));
#pragma unroll
        for (int j = 0; j < V; j++) v[j] *= r;  // xh
        if (OP == 1) {
#pragma unroll
          for (int j = 0; j < V; j++) v[j] = fmaf(v[j], gain[j], bias[j]);
        } else {
          float d[V];
#pragma unroll
          for (int j = 0; j < V; j++) d[j] = 0.f;
          if (here) VecT<T>::unpack(rd[k], d);
          rotate<V, INTER>(d, c, s, src, odd);
          float m1 = 0.f, m2 = 0.f;
#pragma unroll
          for (int j = 0; j < V; j++) {
            dgain[j] = fmaf(d[j], v[j], dgain[j]);
            dbias[j] += d[j];
            d[j] *= gain[j];
            m1 = fmaf(d[j], v[j], m1);
            m2 += d[j];
          }
          m1 = lanes_sum(m1, p.log_lanes) * inv_d;
          m2 = p.center ? lanes_sum(m2, p.log_lanes) * inv_d : 0.f;
#pragma unroll
          for (int j = 0; j < V; j++) v[j] = r * (d[j] - m2 - v[j] * m1);
          if (here) VecT<T>::store((T*)p.dx + row * p.dx_row + h * p.dx_head + e, v);
        }
      }
      if (OP <= 1) {
        rotate<V, INTER>(v, c, s, src, odd);
        if (here) VecT<T>::store((T*)p.y + row * p.y_row + h * p.y_head + e, v);
      }
    }
  }

  if (OP == 2) {  // the block's sums, warps and groups in order
    __shared__ float part[RO_WARPS][2][32 * V];
#pragma unroll
    for (int j = 0; j < V; j++) {
      part[warp][0][lane * V + j] = dgain[j];
      part[warp][1][lane * V + j] = dbias[j];
    }
    __syncthreads();
    float* out = p.partial + (int64_t)(blockIdx.y * gridDim.x + blockIdx.x) * 2 * p.D;
    for (int i = threadIdx.x; i < 2 * p.D; i += 32 * RO_WARPS) {
      const int which = i >= p.D, col = i - which * p.D;
      float sum = 0.f;
      for (int w = 0; w < RO_WARPS; w++)
        for (int t = 0; t < together; t++) sum += part[w][which][t * lanes * V + col];
      out[i] = sum;
    }
  }
}

// Sums of the blocks' sums, in order: 32 columns a block, 32 threads each, added in double at the end.
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

// The launch of all three forms.  passes: a warp takes up to four groups of heads, fewer where the launch would have too
// few warps to fill the device (latency counts there, and the angles cost little).
struct RotaryLaunch { dim3 grid; int q_blocks; };
RotaryLaunch plan_rotary(RotaryParams& p, int vec, int blocks_per_sm, int sms) {
  p.log_lanes = 0;
  while ((vec << p.log_lanes) < p.D) p.log_lanes++;
  const int together = 32 >> p.log_lanes, k_heads = p.heads - p.q_heads;
  int slots = 0;
  for (p.passes = RO_PASSES; p.passes >= 1; p.passes--) {
    p.q_slots = ceil_div(p.q_heads, together * p.passes);
    slots = p.q_slots + ceil_div(k_heads, together * p.passes);
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
  // blocks of 256 threads that an SM holds at the kernels' registers
  const RotaryLaunch l = plan_rotary(p, d.dtype == 1 ? 8 : 4, OP == 2 ? 2 : 3, sms);
  if (d.dtype == 1) {
    if (d.interleaved) launch_pdl(rotary_kernel<bf16, true, OP>, l.grid, 32 * RO_WARPS, 0, st, p);
    else launch_pdl(rotary_kernel<bf16, false, OP>, l.grid, 32 * RO_WARPS, 0, st, p);
  } else {
    if (d.interleaved) launch_pdl(rotary_kernel<float, true, OP>, l.grid, 32 * RO_WARPS, 0, st, p);
    else launch_pdl(rotary_kernel<float, false, OP>, l.grid, 32 * RO_WARPS, 0, st, p);
  }
  return l;
}

int check_strided(const char* what, const char* name, int dtype, const void* ptr, int64_t row, int64_t head) {
  const int unit = dtype == 1 ? 8 : 4;
  if (!ptr) return op_refuse(MSLT_ERR_ARG, "%s: %s is null", what, name);
  if ((uintptr_t)ptr & 15) return op_refuse(MSLT_ERR_ARG, "%s: %s must be 16-byte aligned", what, name);
  if (row % unit || head % unit || row < 0 || head < 0)
    return op_refuse(MSLT_ERR_ARG, "%s: strides of %s must be multiples of 16 bytes", what, name);
  return 0;
}

int check_rope(const char* what, const mslt_rope_desc* d, int rot_min) {
  if (!d) return op_refuse(MSLT_ERR_ARG, "%s: null descriptor", what);
  if (d->dtype != 0 && d->dtype != 1) return op_refuse(MSLT_ERR_ARG, "%s: dtype must be 0 or 1", what);
  if (d->rows < 1 || d->heads < 1) return op_refuse(MSLT_ERR_ARG, "%s: rows and heads must be >= 1", what);
  if (d->heads > 4096) return op_refuse(MSLT_ERR_SIZE, "%s: at most 4096 heads", what);
  if (d->head_dim < 8 || d->head_dim > 128 || d->head_dim % 8)
    return op_refuse(MSLT_ERR_ARG, "%s: head_dim must be a multiple of 8 in [8, 128]", what);
  if (d->rot_dim < rot_min || d->rot_dim > d->head_dim || d->rot_dim % 8)
    return op_refuse(MSLT_ERR_ARG, "%s: rot_dim must be a multiple of 8 in [%d, head_dim]", what, rot_min);
  if (d->rot_dim > 0 && (!d->turns || ((uintptr_t)d->turns & 15)))
    return op_refuse(MSLT_ERR_ARG, "%s: turns must be 16-byte aligned and not null", what);
  if (!d->positions && d->seq < 1) return op_refuse(MSLT_ERR_ARG, "%s: without positions seq must be >= 1", what);
  if (!isfinite(d->magnitude)) return op_refuse(MSLT_ERR_ARG, "%s: magnitude must be finite", what);
  return check_strided(what, "x", d->dtype, d->x, d->x_row, d->x_head);
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
  rc = check_strided("rope", "y", desc->dtype, desc->y, desc->y_row, desc->y_head);
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
  rc = check_strided("qk_norm_rope", "y", desc->rope.dtype, desc->rope.y, desc->rope.y_row, desc->rope.y_head);
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
  if ((rc = check_strided(what, "dy", desc->rope.dtype, desc->dy, desc->dy_row, desc->dy_head))) return rc;
  if ((rc = check_strided(what, "dx", desc->rope.dtype, desc->dx, desc->dx_row, desc->dx_head))) return rc;
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
