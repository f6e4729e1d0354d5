// Attention under masks in bf16 on the tensor cores, forward and backward, for head widths up to 128 (formulas: attn_masked.h).
// The scores never reach memory.  Three kernels of one build: a block owns 128 rows of one head (queries in the
// forward and for dQ, keys for dK and dV), a thread of its four softmax warps owns a row, and the loop runs over blocks
// of 64 rows of the other side that the mask leaves:
//   forward  S = Q K^T                 P = 2^(S' - m)                               O += P V
//   dQ       S = Q K^T, dP = dC V^T    dS = P (dP - delta) dz/ds                    dQ += dS K
//   dK, dV   S^T = K Q^T, dP^T = V dC^T, the same transposed                        dV += P^T dC, dK += dS^T Q
// P and dS are the A operand of the second product and never leave tensor memory: they are written over the scores they
// come from.  dQ and dK/dV are two launches that form S and dP twice (7 products in the place of 5): in return no sum
// crosses blocks, so every run gives the same bits and nothing is added by atomics.
//   warp 0: TMA producer; warp 1: one thread issues the products; warps 2-5: softmax
// Two blocks share an SM where 256 columns of tensor memory and half of the shared memory do (all but the backward of
// heads wider than 64): while one waits for its products, the other has the exponential unit, which bounds heads of 64 (a
// 128 x 128 tile takes 1024 cycles of exponentials, its products 512 in the forward).
//
// Which blocks a row tile visits is worked out once, at its start, from positions, length, prefix and the least and
// greatest document of either side: left out, whole, or with pairs to test.  Documents may be in any order; where they
// are sorted, as in a packed batch, exactly the blocks that hold a common document are visited.  Only blocks with pairs
// to test pay for it: a 64-bit word per row says which pairs count.
// Rows beyond a sequence may hold anything: those of the row tile give rows that are not stored, those of the other
// side are cleared in shared memory (zero times NaN is NaN) by the softmax warps before the product that contracts over
// them.
#include <math.h>

#include <atomic>

#include "attn_masked.h"
#include "tc_common.cuh"

namespace mslt {
bool attn_take_starve();  // whether the next attention launch was asked to run out of time (attn_tc.cu)

namespace {

constexpr int AM_ROWS = 128;      // rows of a block
constexpr int AM_COLS = 64;       // rows of a loop block
constexpr int AM_THREADS = 192;
constexpr int AM_SOFT = 4;        // softmax warps
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// The running maximum of a row is followed only where it grows by more than 2^8: until then the probabilities stay
// below 2^8, which costs bf16 nothing, and the accumulator in tensor memory need not be read and written.
constexpr float AM_SLACK = 8.0f;

struct View { bf16* p; long long batch, row, head; };
struct TcParams {
  AttnMask m;
  int heads, kv_heads, D, tiles;
  View o0, o1;          // ctx | dq | dk, dv
  bf16* rest;
  float* lse;
  const float* delta;
  int a_perm[3], b_perm[3], c_perm[3], d_perm[3];
  long long wait_limit;
  int starve;           // test hook: the producer issues no copies, so the first wait runs out
  int* status;
};

__device__ __forceinline__ void tc_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tc_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tc_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// ---- which loop blocks a row tile visits --------------------------------------------------------------

struct Seq { int len, prefix; };
__device__ __forceinline__ Seq sequence(const AttnMask& m, int b) {
  Seq s;
  s.len = m.lens ? min(max(m.lens[b], 0), m.S) : m.S;
  s.prefix = m.causal ? (m.prefix ? min(max(m.prefix[b], 0), m.S) : 0) : m.S;
  return s;
}

// Called by the whole block.  list[i] receives 2 * block + (pairs to test); returns their number.  Rows r0 .. r0 + 127 are
// queries (and the blocks keys), or with kKeys the other way round.  red: 16 words of shared memory.
template <bool kKeys>
__device__ __forceinline__ int list_blocks(const AttnMask& m, const Seq& s, int b, int r0, uint16_t* list, int* red) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int* docs = m.docs ? m.docs + (long long)b * m.S : nullptr;
  const int r1 = min(r0 + AM_ROWS, s.len) - 1;  // last live row
  int lo = 0, hi = 0;
  if (docs) {
    if (warp < 4) {
      const int r = r0 + (int)threadIdx.x;
      const bool live = r < s.len;
      const int d = live ? docs[r] : 0;
      const int mn = __reduce_min_sync(0xffffffffu, live ? d : 0x7fffffff), mx = __reduce_max_sync(0xffffffffu, live ? d : (int)0x80000000);
      if (lane == 0) { red[warp] = mn; red[4 + warp] = mx; }
    }
    __syncthreads();
    lo = min(min(red[0], red[1]), min(red[2], red[3]));
    hi = max(max(red[4], red[5]), max(red[6], red[7]));
  }
  int first = 0, last = 0;
  if (r0 < s.len) {
    last = kKeys ? s.len : min(s.len, max(r1 + 1, s.prefix));
    first = kKeys && r0 >= s.prefix ? r0 / AM_COLS : 0;
    last = (last + AM_COLS - 1) / AM_COLS;
  }
  // whole by positions: every pair of live rows counts
  auto whole = [&](int c0) {
    if (c0 + AM_COLS > s.len) return false;
    return kKeys ? (c0 >= r1 || r1 < s.prefix) : (c0 + AM_COLS - 1 <= r0 || c0 + AM_COLS <= s.prefix);
  };
  if (docs) {
    constexpr int kAhead = 4;  // blocks whose documents are asked for together
    for (int base = first + warp; base < last; base += (AM_THREADS / 32) * kAhead) {
      int d0[kAhead], d1[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; u++) {
        const int c = (base + u * (AM_THREADS / 32)) * AM_COLS + lane;
        d0[u] = c < s.len ? docs[c] : 0;
        d1[u] = c + 32 < s.len ? docs[c + 32] : 0;
      }
#pragma unroll
      for (int u = 0; u < kAhead; u++) {
        const int blk = base + u * (AM_THREADS / 32), c = blk * AM_COLS + lane;
        int mn = min(c < s.len ? d0[u] : 0x7fffffff, c + 32 < s.len ? d1[u] : 0x7fffffff);
        int mx = max(c < s.len ? d0[u] : (int)0x80000000, c + 32 < s.len ? d1[u] : (int)0x80000000);
        mn = __reduce_min_sync(0xffffffffu, mn);
        mx = __reduce_max_sync(0xffffffffu, mx);
        if (lane == 0 && blk < last)
          list[blk] = mn > hi || mx < lo ? 0 : (lo == hi && mn == lo && mx == lo && whole(blk * AM_COLS)) ? 1 : 2;
      }
    }
    __syncthreads();
  }
  if (warp == 0) {
    int n = 0;
    for (int base = first; base < last; base += 32) {
      const int blk = base + lane;
      int kind = 0;
      if (blk < last) kind = docs ? list[blk] : whole(blk * AM_COLS) ? 1 : 2;
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

// Which of the 64 loop rows from c0 on row r counts a pair with.  docs: the 64 loop rows' documents in shared memory.
template <bool kKeys>
__device__ __forceinline__ uint64_t visible(const Seq& s, int r, int c0, bool has_docs, int doc, const int* docs) {
  const int end = (kKeys ? s.len : min(s.len, max(r + 1, s.prefix))) - c0;
  const int begin = (kKeys && r >= s.prefix ? r : 0) - c0;
  uint64_t w = end >= 64 ? ~0ull : end <= 0 ? 0ull : (1ull << end) - 1;
  if (begin > 0) w = begin >= 64 ? 0ull : w & ~((1ull << begin) - 1);
  if (has_docs) {
    uint32_t a = 0, b = 0;
#pragma unroll
    for (int c = 0; c < 32; c += 4) {
      const int4 x = *reinterpret_cast<const int4*>(docs + c), y = *reinterpret_cast<const int4*>(docs + 32 + c);
      a |= (x.x == doc ? 1u << c : 0) | (x.y == doc ? 2u << c : 0) | (x.z == doc ? 4u << c : 0) | (x.w == doc ? 8u << c : 0);
      b |= (y.x == doc ? 1u << c : 0) | (y.y == doc ? 2u << c : 0) | (y.z == doc ? 4u << c : 0) | (y.w == doc ? 8u << c : 0);
    }
    w &= (uint64_t)b << 32 | a;
  }
  return w;
}

// ---- scores ---------------------------------------------------------------------------------------------

// How a score becomes an exponent of two: 0: s scale log2(e), scale > 0; 1: a bias by distance, or a scale <= 0; 2: capped
// (and perhaps biased).
struct Form { float sl2, z_by, cap2, slope2; };
__device__ __forceinline__ Form form_of(const AttnMask& m, int h) {
  Form f;
  f.sl2 = m.scale * LOG2E;
  f.z_by = m.cap > 0.f ? m.scale / m.cap * (2.f * LOG2E) : 0.f;  // 2^(s z_by) = e^(2 z / cap)
  f.cap2 = m.cap * LOG2E;
  f.slope2 = m.slopes ? m.slopes[h] * LOG2E : 0.f;
  return f;
}
// dist: distance of the pair.  bend: derivative of the cap.  tanh u = 1 - 2 / (1 + e^(2u)): two special functions and an
// absolute error of 2e-7, where the hardware's tanh has 2^-11 of the value (a probability off by 2 % at a score of 50).
template <int kForm>
__device__ __forceinline__ float exponent(const Form& f, float s, float dist, float* bend) {
  if (kForm == 0) return s * f.sl2;
  if (kForm == 1) return fmaf(s, f.sl2, -f.slope2 * dist);
  const float t = fmaf(-2.f, rcp(1.f + ex2(s * f.z_by)), 1.f);
  *bend = fmaf(-t, t, 1.f);
  return fmaf(f.cap2, t, -f.slope2 * dist);
}

// ---- pieces of the roles ----------------------------------------------------------------------------------

struct Ring { uint64_t *full, *empty; };

__device__ __forceinline__ uint32_t addr16(uint32_t a) { return (a & 0x3FFFFu) >> 4; }

// D (+)= A B^T, both with the contraction contiguous, over DP; a_kb, b_kb: 16-byte units between 64-wide tiles of it
template <int DP>
__device__ __forceinline__ void product_ss(uint32_t d, uint32_t a, uint32_t a_kb, uint32_t b, uint32_t b_kb, uint32_t idesc) {
  const uint32_t hi = (uint32_t)(make_smem_desc(0, 16) >> 32), lo = (uint32_t)make_smem_desc(0, 16);
#pragma unroll
  for (int kb = 0; kb < DP / 64; kb++)
#pragma unroll
    for (int k = 0; k < 4; k++) {
      const uint64_t ad = ((uint64_t)hi << 32) | (lo + addr16(a) + kb * a_kb + k * 2);
      const uint64_t bd = ((uint64_t)hi << 32) | (lo + addr16(b) + kb * b_kb + k * 2);
      tc_mma(d, ad, bd, idesc, kb + k > 0 ? 1u : 0u);
    }
}
// D (+)= A B, A 64 wide in tensor memory, B 64 rows (the contraction) of DP contiguous elements
__device__ __forceinline__ void product_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  const uint32_t hi = (uint32_t)(make_smem_desc(0, 16) >> 32), lo = (uint32_t)make_smem_desc(0, 8192);
#pragma unroll
  for (int k = 0; k < 4; k++)
    tc_mma_ts(d, a + k * 8, ((uint64_t)hi << 32) | (lo + addr16(b) + k * 128), idesc, accumulate | (k > 0));
}

template <int DP>
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* map, const int (&perm)[3], uint32_t bar, int row, int head,
                                          int batch, int tile_bytes) {
  int c[4];
  c[perm[0]] = row; c[perm[1]] = head; c[perm[2]] = batch;
#pragma unroll
  for (int kb = 0; kb < DP / 64; kb++) {
    c[0] = kb * 64;
    tma_load_4d(dst + kb * tile_bytes, map, bar, c[0], c[1], c[2], c[3]);
  }
}

// The producer gave up: what it has issued must have landed before the block leaves.
__device__ __forceinline__ void drain(uint64_t* bar, uint32_t parity) {
  const long long t0 = now_cycles();
  while (!mbar_try_wait(smem_u32(bar), parity) && now_cycles() - t0 < 200000000ll) {}
}

// Rows `from` .. 63 of a loop block's tiles become zero; the whole softmax group, thread t of 128.
template <int DP>
__device__ __forceinline__ void clear_rows(uint8_t* tile, int from, int t) {
#pragma unroll
  for (int kb = 0; kb < DP / 64; kb++)
    for (int v = from * 8 + t; v < AM_COLS * 8; v += AM_SOFT * 32)
      reinterpret_cast<uint4*>(tile + kb * 8192)[v] = make_uint4(0, 0, 0, 0);
}

// 32 columns of a row, scaled, to bf16; optionally what the rounding took off
__device__ __forceinline__ void store32(bf16* dst, bf16* rest, const uint32_t (&r)[32], float f, int cols) {
#pragma unroll
  for (int c = 0; c < 32; c += 8) {
    if (c >= cols) break;
    uint4 hi, lo;
    uint32_t *h = reinterpret_cast<uint32_t*>(&hi), *l = reinterpret_cast<uint32_t*>(&lo);
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const float x = __uint_as_float(r[c + 2 * e]) * f, y = __uint_as_float(r[c + 2 * e + 1]) * f;
      h[e] = pack2(x, y);
      const float2 b = bf162_to_f2(h[e]);
      l[e] = pack2(x - b.x, y - b.y);
    }
    *reinterpret_cast<uint4*>(dst + c) = hi;
    if (rest) *reinterpret_cast<uint4*>(rest + c) = lo;
  }
}
// A row of an accumulator (DP columns from taddr on) to memory; f = 0 stores zeros whatever the accumulator holds.
template <int DP>
__device__ __forceinline__ void store_row(uint32_t taddr, bf16* dst, bf16* rest, float f, bool zero, bool have, bool write, int D) {
#pragma unroll
  for (int c = 0; c < DP; c += 32) {
    uint32_t r[32];
    if (have) {
      tc_ld32_issue(taddr + c, r);
      tc_ld32_wait(r);
    }
    if (zero || !have) {
#pragma unroll
      for (int e = 0; e < 32; e++) r[e] = 0;
    }
    if (write) store32(dst + c, rest ? rest + c : nullptr, r, f, D - c);
  }
}

__host__ __device__ constexpr uint32_t idesc_of(int n, bool b_rows_are_k) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (b_rows_are_k ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

template <int COLS>
__device__ __forceinline__ void tmem_alloc(uint32_t* slot) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(COLS) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
template <int COLS>
__device__ __forceinline__ void tmem_free(uint32_t base) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(COLS) : "memory");
}

// The issuing thread gave up: products in flight must be over before tensor memory is freed.
__device__ __forceinline__ void settle(uint64_t* bar) {
  tc_commit(smem_u32(bar));
  const long long t0 = now_cycles();
  while (now_cycles() - t0 < 2000000ll) {}
}

// ---- forward ----------------------------------------------------------------------------------------------

template <int DP> struct FwdShape {
  static constexpr int STAGES = DP == 64 ? 4 : 2;
  static constexpr int Q_BYTES = AM_ROWS * DP * 2, KV_BYTES = AM_COLS * DP * 2;
  static constexpr int SMEM = Q_BYTES + 2 * STAGES * KV_BYTES;
};

template <int DP, int kForm>
__global__ void __launch_bounds__(AM_THREADS, 2)
masked_fwd_tc(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
              const __grid_constant__ CUtensorMap tmV, const TcParams p) {
  typedef FwdShape<DP> Sh;
  constexpr int NS = Sh::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* Ks = smem + Sh::Q_BYTES;
  uint8_t* Vs = Ks + NS * Sh::KV_BYTES;
  uint16_t* list = (uint16_t*)(Vs + NS * Sh::KV_BYTES);
  __shared__ uint64_t qfull, kfull[NS], kempty[NS], vfull[NS], vempty[NS], sfull[2], pready[2], odone[2], oall;
  __shared__ uint32_t tmem_slot;
  __shared__ int red[16];
  __shared__ __align__(16) int docs_of[AM_SOFT][AM_COLS];
  __shared__ __align__(8) int flag_mem[4];
  volatile int* abort_flag = flag_mem + 1;   // the limit, 8 bytes, follows
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&qfull), 1);
    for (int i = 0; i < NS; i++) {
      mbar_init(smem_u32(&kfull[i]), 1);
      mbar_init(smem_u32(&kempty[i]), 1);
      mbar_init(smem_u32(&vfull[i]), 1);
      mbar_init(smem_u32(&vempty[i]), 1);
    }
    for (int i = 0; i < 2; i++) {
      mbar_init(smem_u32(&sfull[i]), 1);
      mbar_init(smem_u32(&pready[i]), AM_SOFT);
      mbar_init(smem_u32(&odone[i]), 1);
    }
    mbar_init(smem_u32(&oall), 1);
    *abort_flag = 0;
    *reinterpret_cast<volatile long long*>(abort_flag + 1) = p.wait_limit;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0 && elect_one()) {
    prefetch_map(&tmQ);
    prefetch_map(&tmK);
    prefetch_map(&tmV);
  }
  if (warp == 1) tmem_alloc<256>(&tmem_slot);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_begin();

  const int idx = blockIdx.x % p.tiles, h = blockIdx.x / p.tiles % p.heads, b = blockIdx.x / p.tiles / p.heads;
  const int tile = p.m.causal ? p.tiles - 1 - idx : idx;  // causal: the tiles with the most keys start first
  const int hk = h / (p.heads / p.kv_heads), r0 = tile * AM_ROWS;
  const Seq s = sequence(p.m, b);
  const int n = list_blocks<false>(p.m, s, b, r0, list, red);
  constexpr uint32_t O_COL = 128;

  if (warp == 0 && n > 0 && !p.starve && elect_one()) {
    // ------------------------------- TMA producer -------------------------------
    mbar_expect_tx(smem_u32(&qfull), Sh::Q_BYTES);
    load_rows<DP>(smem_u32(smem), &tmQ, p.a_perm, smem_u32(&qfull), r0, h, b, 16384);
    int k_issued = 0, v_issued = 0;
    for (int j = 0; j < n; j++) {
      const int st = j % NS, row = (list[j] >> 1) * AM_COLS;
      const uint32_t par = (uint32_t)(j / NS & 1) ^ 1;
      if (!mbar_wait(smem_u32(&kempty[st]), par, abort_flag, p.status)) break;
      mbar_expect_tx(smem_u32(&kfull[st]), Sh::KV_BYTES);
      load_rows<DP>(smem_u32(Ks + st * Sh::KV_BYTES), &tmK, p.b_perm, smem_u32(&kfull[st]), row, hk, b, 8192);
      k_issued = j + 1;
      if (!mbar_wait(smem_u32(&vempty[st]), par, abort_flag, p.status)) break;
      mbar_expect_tx(smem_u32(&vfull[st]), Sh::KV_BYTES);
      load_rows<DP>(smem_u32(Vs + st * Sh::KV_BYTES), &tmV, p.c_perm, smem_u32(&vfull[st]), row, hk, b, 8192);
      v_issued = j + 1;
    }
    if (v_issued < n || *abort_flag) {
      drain(&qfull, 0);
      for (int j = max(0, k_issued - NS); j < k_issued; j++) drain(&kfull[j % NS], (j / NS) & 1);
      for (int j = max(0, v_issued - NS); j < v_issued; j++) drain(&vfull[j % NS], (j / NS) & 1);
    }
  } else if (warp == 1 && n > 0 && elect_one()) {
    // ------------------------------- products -------------------------------
    constexpr uint32_t id_s = idesc_of(AM_COLS, false), id_o = idesc_of(DP, true);
    auto scores = [&](int j) {
      const int st = j % NS;
      if (!mbar_wait(smem_u32(&kfull[st]), j / NS & 1, abort_flag, p.status)) return false;
      tc_fence_after();
      product_ss<DP>(tmem + (j & 1) * 64, smem_u32(smem), 1024, smem_u32(Ks + st * Sh::KV_BYTES), 512, id_s);
      tc_commit(smem_u32(&sfull[j & 1]));
      tc_commit(smem_u32(&kempty[st]));
      return true;
    };
    bool ok = mbar_wait(smem_u32(&qfull), 0, abort_flag, p.status) && scores(0);
    for (int j = 0; j < n && ok; j++) {
      if (j + 1 < n && !scores(j + 1)) { ok = false; break; }
      const int st = j % NS;
      ok = mbar_wait(smem_u32(&vfull[st]), j / NS & 1, abort_flag, p.status) &&
           mbar_wait(smem_u32(&pready[j & 1]), j >> 1 & 1, abort_flag, p.status);
      if (!ok) break;
      tc_fence_after();
      product_ts(tmem + O_COL, tmem + (j & 1) * 64, smem_u32(Vs + st * Sh::KV_BYTES), id_o, j > 0);
      tc_commit(smem_u32(&odone[j & 1]));
      tc_commit(smem_u32(&vempty[st]));
    }
    if (ok) tc_commit(smem_u32(&oall));
    if (!ok || *abort_flag) settle(&oall);
  } else if (warp >= 2) {
    // ------------------------------- softmax: a thread owns a query -------------------------------
    const int quarter = warp & 3, row = quarter * 32 + lane, r = r0 + row;
    const uint32_t trow = tmem + ((uint32_t)(quarter * 32) << 16);
    const Form f = form_of(p.m, h);
    const int* docs = p.m.docs ? p.m.docs + (long long)b * p.m.S : nullptr;
    const int doc = docs && r < s.len ? docs[r] : 0;
    float top = -INFINITY;               // reference of the row's exponents
    float sum = 0.f, exact = 0.f;        // of the rounded probabilities, and of the unrounded ones
    bool ok = true;
    for (int j = 0; j < n; j++) {
      const int entry = list[j], c0 = (entry >> 1) * AM_COLS;
      uint64_t see = ~0ull;
      if (entry & 1) {
        if (docs) {
          __syncwarp();
          docs_of[warp - 2][lane] = c0 + lane < s.len ? docs[c0 + lane] : 0;
          docs_of[warp - 2][lane + 32] = c0 + lane + 32 < s.len ? docs[c0 + lane + 32] : 0;
          __syncwarp();
        }
        see = visible<false>(s, r, c0, docs != nullptr, doc, docs_of[warp - 2]);
      }
      if (!mbar_wait(smem_u32(&sfull[j & 1]), j >> 1 & 1, abort_flag, p.status)) { ok = false; break; }
      tc_fence_after();
      uint32_t a0[32], a1[32];
      tc_ld32_issue(trow + (j & 1) * 64, a0);
      tc_ld32_issue(trow + (j & 1) * 64 + 32, a1);
      tc_ld32_wait(a0);
      tc_ld32_wait(a1);
      float x[64];
#pragma unroll
      for (int c = 0; c < 32; c++) {
        x[c] = __uint_as_float(a0[c]);
        x[c + 32] = __uint_as_float(a1[c]);
      }
      if (kForm != 0) {
        const float off = (float)(c0 - r);
#pragma unroll
        for (int c = 0; c < 64; c++) {
          float bend;
          x[c] = exponent<kForm>(f, x[c], fabsf(off + (float)c), &bend);
        }
      }
      if (entry & 1) {
        const uint32_t w0 = (uint32_t)see, w1 = (uint32_t)(see >> 32);
#pragma unroll
        for (int c = 0; c < 32; c++) {
          x[c] = w0 >> c & 1 ? x[c] : -INFINITY;
          x[c + 32] = w1 >> c & 1 ? x[c + 32] : -INFINITY;
        }
      }
      float mx[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
      for (int c = 4; c < 64; c += 8)
#pragma unroll
        for (int e = 0; e < 4; e++) mx[e] = c + 4 + e < 64 ? fmaxf(fmaxf(mx[e], x[c + e]), x[c + 4 + e]) : fmaxf(mx[e], x[c + e]);
      float big = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
      if (kForm == 0) big *= f.sl2;
      const bool grow = big > top + AM_SLACK || (top == -INFINITY && big > top);
      if (__any_sync(0xffffffffu, grow)) {
        const float by = grow ? ex2(top - big) : 1.f;
        if (grow) top = big;
        sum *= by;
        exact *= by;
        if (j > 0) {
          // two barriers: the scores at hand say that the product before the last is complete, so neither can be a phase ahead
          if (!mbar_wait(smem_u32(&odone[(j - 1) & 1]), (j - 1) >> 1 & 1, abort_flag, p.status)) { ok = false; break; }
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < DP; c += 32) {
            uint32_t o[32];
            tc_ld32_issue(trow + O_COL + c, o);
            tc_ld32_wait(o);
#pragma unroll
            for (int e = 0; e < 32; e++) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
            tc_st32(trow + O_COL + c, o);
          }
          tc_st_wait();
        }
      }
      const float base = top == -INFINITY ? 0.f : top;
      uint32_t pk[32];
      float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)}, part_r[2] = {part[0], part[0]};
#pragma unroll
      for (int c = 0; c < 32; c++) {
        float2 e = make_float2(x[2 * c], x[2 * c + 1]);
        e = kForm == 0 ? __ffma2_rn(e, splat2(f.sl2), splat2(-base)) : __fadd2_rn(e, splat2(-base));
        e.x = ex2(e.x);
        e.y = ex2(e.y);
        pk[c] = pack2(e.x, e.y);
        part[c & 1] = __fadd2_rn(part[c & 1], e);
        part_r[c & 1] = __fadd2_rn(part_r[c & 1], bf162_to_f2(pk[c]));
      }
      tc_st32(trow + (j & 1) * 64, pk);
      tc_st_wait();
      if ((entry & 1) && s.len < c0 + AM_COLS) {
        if (!mbar_wait(smem_u32(&vfull[j % NS]), j / NS & 1, abort_flag, p.status)) { ok = false; break; }
        clear_rows<DP>(Vs + (j % NS) * Sh::KV_BYTES, s.len - c0, threadIdx.x - 64);
        fence_proxy_async_smem();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&pready[j & 1]));
      exact += (part[0].x + part[0].y) + (part[1].x + part[1].y);
      sum += (part_r[0].x + part_r[0].y) + (part_r[1].x + part_r[1].y);
    }
    if (ok && n > 0) ok = mbar_wait(smem_u32(&oall), 0, abort_flag, p.status);
    if (ok) {
      tc_fence_after();
      const bool empty = r >= s.len || !(sum > 0.f);
      const long long at = b * p.o0.batch + r * p.o0.row + h * p.o0.head;
      store_row<DP>(trow + O_COL, p.o0.p + at, p.rest ? p.rest + at : nullptr, empty ? 0.f : 1.f / sum, empty, n > 0, r < p.m.S, p.D);
      if (p.lse && r < p.m.S)
        p.lse[((long long)b * p.heads + h) * p.m.S + r] = empty ? -INFINITY : (top + log2f(exact)) * LN2;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_free<256>(tmem);
  }
}

// ---- backward ---------------------------------------------------------------------------------------------

// delta_i = dC_i . (C_i + rest_i): eight elements a lane, the lanes of a row side by side
__global__ void __launch_bounds__(256)
masked_delta_tc(const View dc, const View c, const bf16* rest, float* delta, int S, int heads, int D, int log_lanes, long long rows) {
  pdl_begin();
  const int lanes = 1 << log_lanes;
  const long long n = ((long long)blockIdx.x * 256 + threadIdx.x) >> log_lanes;  // head fastest: neighbours in memory
  const int e = (threadIdx.x & (lanes - 1)) * 8;
  float sum = 0.f;
  int h = 0, i = 0;
  long long b = 0;
  if (n < rows) {
    h = (int)(n % heads);
    i = (int)(n / heads % S);
    b = n / heads / S;
    if (e < D) {
      float x[8], y[8];
      VecT<bf16>::load(dc.p + b * dc.batch + i * dc.row + h * dc.head + e, x);
      const long long at = b * c.batch + i * c.row + h * c.head + e;
      VecT<bf16>::load(c.p + at, y);
      if (rest) {
        float z[8];
        VecT<bf16>::load(rest + at, z);
#pragma unroll
        for (int k = 0; k < 8; k++) y[k] += z[k];
      }
#pragma unroll
      for (int k = 0; k < 8; k++) sum = fmaf(x[k], y[k], sum);
    }
  }
  for (int o = lanes >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (n < rows && e == 0) delta[(b * heads + h) * S + i] = sum;
}

// Tensor memory and stages of the two backward kernels.  Heads of up to 64: 256 columns, two blocks an SM.  Wider
// ones need 384 and more, so one block an SM has two buffers of S and dP and its products run ahead of the softmax.
template <int DP, bool kKeys> struct BwdShape {
  static constexpr bool wide = DP == 128;
  static constexpr int SB = wide || !kKeys ? 2 : 1, PB = wide ? 2 : 1;   // buffers of S, of dP
  static constexpr int STAGES = wide ? 4 : 3;
  static constexpr int COLS = wide ? 512 : 256;
  static constexpr int DP_COL = SB * 64, ACC_COL = DP_COL + PB * 64;
  static constexpr int FIX_BYTES = AM_ROWS * DP * 2, LOOP_BYTES = AM_COLS * DP * 2;
  static constexpr int SMEM = 2 * FIX_BYTES + STAGES * 2 * LOOP_BYTES;
};

// kKeys = false: rows are queries (A = q, B = k, C = dctx, D = v; loop over keys), the result is dq.
// kKeys = true: rows are keys (A = k, B = q, C = v, D = dctx; loop over the queries of every head that shares them): dk, dv.
template <int DP, bool kKeys, int kForm>
__global__ void __launch_bounds__(AM_THREADS, DP == 64 ? 2 : 1)
masked_bwd_tc(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
              const __grid_constant__ CUtensorMap tmC, const __grid_constant__ CUtensorMap tmD, const TcParams p) {
  typedef BwdShape<DP, kKeys> Sh;
  constexpr int NS = Sh::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* As = smem;
  uint8_t* Cs = smem + Sh::FIX_BYTES;
  uint8_t* Bs = Cs + Sh::FIX_BYTES;                 // stage: B then D
  uint16_t* list = (uint16_t*)(Bs + NS * 2 * Sh::LOOP_BYTES);
  __shared__ uint64_t fixfull, full[NS], empty[NS], sfull[2], ready[2], dpread, done;
  __shared__ uint32_t tmem_slot;
  __shared__ int red[16];
  __shared__ __align__(16) int docs_of[AM_SOFT][AM_COLS];
  __shared__ __align__(16) float cols_of[kKeys ? AM_SOFT : 1][2][AM_COLS];   // kKeys: lse (log2) and delta of the loop's queries
  __shared__ __align__(8) int flag_mem[4];
  volatile int* abort_flag = flag_mem + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&fixfull), 1);
    for (int i = 0; i < NS; i++) {
      mbar_init(smem_u32(&full[i]), 1);
      mbar_init(smem_u32(&empty[i]), 1);
    }
    for (int i = 0; i < 2; i++) {
      mbar_init(smem_u32(&sfull[i]), 1);
      mbar_init(smem_u32(&ready[i]), AM_SOFT);
    }
    mbar_init(smem_u32(&dpread), AM_SOFT);
    mbar_init(smem_u32(&done), 1);
    *abort_flag = 0;
    *reinterpret_cast<volatile long long*>(abort_flag + 1) = p.wait_limit;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0 && elect_one()) {
    prefetch_map(&tmA);
    prefetch_map(&tmB);
    prefetch_map(&tmC);
    prefetch_map(&tmD);
  }
  if (warp == 1) tmem_alloc<Sh::COLS>(&tmem_slot);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_begin();

  const int row_heads = kKeys ? p.kv_heads : p.heads, group = p.heads / p.kv_heads;
  const int idx = blockIdx.x % p.tiles, hr = blockIdx.x / p.tiles % row_heads, b = blockIdx.x / p.tiles / row_heads;
  const int tile = p.m.causal && !kKeys ? p.tiles - 1 - idx : idx;  // causal: the tiles with the longest loops start first
  const int r0 = tile * AM_ROWS;
  const Seq s = sequence(p.m, b);
  const int n_list = list_blocks<kKeys>(p.m, s, b, r0, list, red);
  const int n = kKeys ? n_list * group : n_list;
  // loop step j: its list entry and head
  auto entry_of = [&](int j) { return (int)list[kKeys ? j % n_list : j]; };
  auto head_of = [&](int j) { return kKeys ? hr * group + j / n_list : hr / group; };

  if (warp == 0 && n > 0 && !p.starve && elect_one()) {
    // ------------------------------- TMA producer -------------------------------
    const uint32_t fb = smem_u32(&fixfull);
    mbar_expect_tx(fb, 2 * Sh::FIX_BYTES);
    load_rows<DP>(smem_u32(As), &tmA, p.a_perm, fb, r0, hr, b, 16384);
    load_rows<DP>(smem_u32(Cs), &tmC, p.c_perm, fb, r0, hr, b, 16384);
    int issued = 0;
    for (int j = 0; j < n; j++) {
      const int st = j % NS, row = (entry_of(j) >> 1) * AM_COLS, hl = head_of(j);
      if (!mbar_wait(smem_u32(&empty[st]), (uint32_t)(j / NS & 1) ^ 1, abort_flag, p.status)) break;
      const uint32_t bar = smem_u32(&full[st]), dst = smem_u32(Bs + st * 2 * Sh::LOOP_BYTES);
      mbar_expect_tx(bar, 2 * Sh::LOOP_BYTES);
      load_rows<DP>(dst, &tmB, p.b_perm, bar, row, hl, b, 8192);
      load_rows<DP>(dst + Sh::LOOP_BYTES, &tmD, p.d_perm, bar, row, hl, b, 8192);
      issued = j + 1;
    }
    if (issued < n || *abort_flag) {
      drain(&fixfull, 0);
      for (int j = max(0, issued - NS); j < issued; j++) drain(&full[j % NS], (j / NS) & 1);
    }
  } else if (warp == 1 && n > 0 && elect_one()) {
    // ------------------------------- products -------------------------------
    constexpr uint32_t id_s = idesc_of(AM_COLS, false), id_acc = idesc_of(DP, true);
    auto stage = [&](int j) { return smem_u32(Bs + (j % NS) * 2 * Sh::LOOP_BYTES); };
    auto landed = [&](int j) {
      if (!mbar_wait(smem_u32(&full[j % NS]), j / NS & 1, abort_flag, p.status)) return false;
      tc_fence_after();
      return true;
    };
    auto scores = [&](int j) { product_ss<DP>(tmem + (j % Sh::SB) * 64, smem_u32(As), 1024, stage(j), 512, id_s); };
    auto dprobs = [&](int j) {
      product_ss<DP>(tmem + Sh::DP_COL + (j % Sh::PB) * 64, smem_u32(Cs), 1024, stage(j) + Sh::LOOP_BYTES, 512, id_s);
    };
    bool ok = mbar_wait(smem_u32(&fixfull), 0, abort_flag, p.status) && landed(0);
    if (ok) {
      scores(0);
      dprobs(0);
      tc_commit(smem_u32(&sfull[0]));
    }
    for (int j = 0; j < n && ok; j++) {
      const bool more = j + 1 < n;
      if (more) {
        if (!landed(j + 1)) { ok = false; break; }
        if (Sh::SB == 2) scores(j + 1);
        if (Sh::PB == 1) {
          if (!mbar_wait(smem_u32(&dpread), j & 1, abort_flag, p.status)) { ok = false; break; }
          tc_fence_after();
        }
        dprobs(j + 1);
        if (Sh::SB == 2) tc_commit(smem_u32(&sfull[(j + 1) & 1]));
      }
      if (!mbar_wait(smem_u32(&ready[j & 1]), j >> 1 & 1, abort_flag, p.status)) { ok = false; break; }
      tc_fence_after();
      const uint32_t at = tmem + (j % Sh::SB) * 64;
      if (kKeys) {
        product_ts(tmem + Sh::ACC_COL, at, stage(j) + Sh::LOOP_BYTES, id_acc, j > 0);        // dV += P^T dC
        product_ts(tmem + Sh::ACC_COL + DP, at + 32, stage(j), id_acc, j > 0);               // dK += dS^T Q
      } else {
        product_ts(tmem + Sh::ACC_COL, at, stage(j), id_acc, j > 0);                         // dQ += dS K
      }
      tc_commit(smem_u32(&empty[j % NS]));
      if (more && Sh::SB == 1) {
        scores(j + 1);
        tc_commit(smem_u32(&sfull[(j + 1) & 1]));
      }
    }
    if (ok) tc_commit(smem_u32(&done));
    if (!ok || *abort_flag) settle(&done);
  } else if (warp >= 2) {
    // ------------------------------- softmax and its backward: a thread owns a row -------------------------------
    const int quarter = warp & 3, row = quarter * 32 + lane, r = r0 + row;
    const uint32_t trow = tmem + ((uint32_t)(quarter * 32) << 16);
    const int* docs = p.m.docs ? p.m.docs + (long long)b * p.m.S : nullptr;
    const int doc = docs && r < s.len ? docs[r] : 0;
    Form f = form_of(p.m, kKeys ? hr * group : hr);
    float lse2 = INFINITY, delta = 0.f;
    if (!kKeys && r < s.len) {
      const long long at = ((long long)b * p.heads + hr) * p.m.S + r;
      lse2 = p.lse[at] * LOG2E;
      delta = p.delta[at];
    }
    bool ok = true;
    for (int j = 0; j < n; j++) {
      const int entry = entry_of(j), c0 = (entry >> 1) * AM_COLS;
      uint64_t see = ~0ull;
      if (kKeys || ((entry & 1) && docs)) {
        __syncwarp();
        if (kKeys) {
          const int hq = head_of(j);
          if (kForm == 2 || kForm == 1) f = form_of(p.m, hq);
          const long long at = ((long long)b * p.heads + hq) * p.m.S + c0;
#pragma unroll
          for (int e = lane; e < 64; e += 32) {
            const bool live = c0 + e < s.len;
            cols_of[warp - 2][0][e] = live ? -p.lse[at + e] * LOG2E : 0.f;
            cols_of[warp - 2][1][e] = live ? -p.delta[at + e] : 0.f;
          }
        }
        if ((entry & 1) && docs) {
          docs_of[warp - 2][lane] = c0 + lane < s.len ? docs[c0 + lane] : 0;
          docs_of[warp - 2][lane + 32] = c0 + lane + 32 < s.len ? docs[c0 + lane + 32] : 0;
        }
        __syncwarp();
      }
      if (entry & 1) see = visible<kKeys>(s, r, c0, docs != nullptr, doc, docs_of[warp - 2]);
      if (!mbar_wait(smem_u32(&sfull[j & 1]), j >> 1 & 1, abort_flag, p.status)) { ok = false; break; }
      tc_fence_after();
      const uint32_t tS = trow + (j % Sh::SB) * 64, tP = trow + Sh::DP_COL + (j % Sh::PB) * 64;
      uint32_t pk[32];  // kKeys: P in the first half, dS in the second, 32 columns at a time
      uint32_t keep[16];
#pragma unroll
      for (int half = 0; half < 2; half++) {
        uint32_t a[32], d[32];
        tc_ld32_issue(tS + half * 32, a);
        tc_ld32_issue(tP + half * 32, d);
        tc_ld32_wait(a);
        tc_ld32_wait(d);
        if (half == 1 && Sh::PB == 1) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&dpread));
        }
        const uint32_t w = (uint32_t)(see >> (32 * half));
        const float off = (float)(c0 + half * 32 - r);
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
          float2 x = make_float2(__uint_as_float(a[c]), __uint_as_float(a[c + 1]));
          float2 t = make_float2(__uint_as_float(d[c]), __uint_as_float(d[c + 1]));
          float2 nl = splat2(-lse2), nd = splat2(-delta), bend = splat2(1.f);
          if (kKeys) {
            nl = *reinterpret_cast<const float2*>(&cols_of[warp - 2][0][half * 32 + c]);
            nd = *reinterpret_cast<const float2*>(&cols_of[warp - 2][1][half * 32 + c]);
          }
          if (kForm == 0) {
            x = __ffma2_rn(x, splat2(f.sl2), nl);
          } else {
            x.x = exponent<kForm>(f, x.x, fabsf(off + (float)c), &bend.x);
            x.y = exponent<kForm>(f, x.y, fabsf(off + (float)(c + 1)), &bend.y);
            x = __fadd2_rn(x, nl);
          }
          x.x = ex2(x.x);
          x.y = ex2(x.y);
          t = __fmul2_rn(__fadd2_rn(t, nd), x);
          if (kForm == 2) t = __fmul2_rn(t, bend);
          if (entry & 1) {
            // A row with a single key has no gradient by its score: dP - delta is the difference of two sums in different
            // orders there, and is zero in truth.  p(dP_j - delta) is at most (1 - p) times the spread of dP, so
            // nothing above 1e-5 of it is dropped; a block without pairs to test has 64 keys a row and no such p alone.
            const bool one0 = x.x > 0.99999f, one1 = x.y > 0.99999f;
            const bool v0 = w >> c & 1, v1 = w >> (c + 1) & 1;
            x.x = v0 ? x.x : 0.f;
            x.y = v1 ? x.y : 0.f;
            t.x = v0 && !one0 ? t.x : 0.f;
            t.y = v1 && !one1 ? t.y : 0.f;
          }
          if (kKeys) {
            const int at = (half * 32 + c) / 2;
            pk[at] = pack2(x.x, x.y);
            if (half == 0) keep[at] = pack2(t.x, t.y);
            else a[c / 2] = pack2(t.x, t.y);
          } else {
            pk[(half * 32 + c) / 2] = pack2(t.x, t.y);
          }
        }
        if (kKeys && half == 1) {
          uint32_t ds[32];
#pragma unroll
          for (int e = 0; e < 16; e++) {
            ds[e] = keep[e];
            ds[16 + e] = a[e];
          }
          tc_st32(tS + 32, ds);
        }
      }
      tc_st32(tS, pk);
      tc_st_wait();
      if ((entry & 1) && s.len < c0 + AM_COLS) {
        // the products' reads of this stage so far are over (S and dP are complete); its rows are an operand once more
        clear_rows<DP>(Bs + (j % NS) * 2 * Sh::LOOP_BYTES, s.len - c0, threadIdx.x - 64);
        if (kKeys) clear_rows<DP>(Bs + (j % NS) * 2 * Sh::LOOP_BYTES + Sh::LOOP_BYTES, s.len - c0, threadIdx.x - 64);
        fence_proxy_async_smem();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ready[j & 1]));
    }
    if (ok && n > 0) ok = mbar_wait(smem_u32(&done), 0, abort_flag, p.status);
    if (ok) {
      tc_fence_after();
      const bool dead = r >= s.len;
      const long long a0 = b * p.o0.batch + r * p.o0.row + hr * p.o0.head;
      if (kKeys) {
        const long long a1 = b * p.o1.batch + r * p.o1.row + hr * p.o1.head;
        store_row<DP>(trow + Sh::ACC_COL, p.o1.p + a1, nullptr, 1.f, dead, n > 0, r < p.m.S, p.D);
        store_row<DP>(trow + Sh::ACC_COL + DP, p.o0.p + a0, nullptr, p.m.scale, dead, n > 0, r < p.m.S, p.D);
      } else {
        store_row<DP>(trow + Sh::ACC_COL, p.o0.p + a0, nullptr, p.m.scale, dead, n > 0, r < p.m.S, p.D);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_free<Sh::COLS>(tmem);
  }
}

// ---- host ---------------------------------------------------------------------------------------------------

constexpr int kMaxDevices = 64;
std::mutex g_am_mu;

template <typename K>
int opt_in(K kernel, bool (&done)[kMaxDevices], size_t smem, char* err) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev < 0 || dev >= kMaxDevices)) e = cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_am_mu);
  if (e == cudaSuccess && !done[dev]) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) {
    snprintf(err, 256, "attention_masked: %s", cudaGetErrorString(e));
    return MSLT_ERR_CUDA;
  }
  done[dev] = true;
  return 0;
}

int map_of(const mslt_heads& h, const mslt_attention_desc& d, int heads, int box_rows, MapVal* m, int (&perm)[3], char* err) {
  const int rc = get_map(h.data, d.S, d.head_dim, h.row, 1, h.batch, h.head, heads, d.B, box_rows, m, err);
  for (int i = 0; i < 3; i++) perm[i] = m->perm[i];
  return rc;
}
View view_of(const mslt_heads& h) { return View{(bf16*)h.data, h.batch, h.row, h.head}; }

TcParams params_of(const mslt_attention_desc& d, int* status, bool starve) {
  TcParams p;
  memset(&p, 0, sizeof(p));
  p.m = AttnMask{d.S, d.causal != 0, d.scale, d.cap, d.slopes, d.prefix, d.docs, d.lens};
  p.heads = d.heads; p.kv_heads = d.kv_heads; p.D = d.head_dim;
  p.tiles = (d.S + AM_ROWS - 1) / AM_ROWS;
  p.rest = (bf16*)d.rest; p.lse = d.lse;
  p.wait_limit = starve ? 40000000ll : WAIT_LIMIT_CYCLES;  // starved: about 20 ms
  p.starve = starve;
  p.status = status;
  return p;
}
int form_index(const mslt_attention_desc& d) { return d.cap > 0.f ? 2 : d.slopes || !(d.scale > 0.f) ? 1 : 0; }
// shared memory beside the tiles: alignment and the list of blocks.  The largest list (S = 131072) is opted in for.
size_t list_bytes(int S) { return 1024 + ((size_t)(S + AM_COLS - 1) / AM_COLS * 2 + 15) / 16 * 16; }
constexpr size_t kMostList = 1024 + 131072 / AM_COLS * 2;

template <int DP, int kForm>
int forward(const mslt_attention_desc& d, TcParams& p, const MapVal* m, cudaStream_t st, char* err) {
  static bool done[kMaxDevices];
  if (opt_in(masked_fwd_tc<DP, kForm>, done, FwdShape<DP>::SMEM + kMostList, err)) return MSLT_ERR_CUDA;
  launch_pdl(masked_fwd_tc<DP, kForm>, d.B * d.heads * p.tiles, AM_THREADS, FwdShape<DP>::SMEM + list_bytes(d.S), st, m[0].map, m[1].map,
             m[2].map, p);
  return 0;
}
template <int DP, bool kKeys, int kForm>
int backward(const mslt_attention_desc& d, TcParams& p, const MapVal* m, cudaStream_t st, char* err) {
  static bool done[kMaxDevices];
  typedef BwdShape<DP, kKeys> Sh;
  if (opt_in(masked_bwd_tc<DP, kKeys, kForm>, done, Sh::SMEM + kMostList, err)) return MSLT_ERR_CUDA;
  launch_pdl(masked_bwd_tc<DP, kKeys, kForm>, d.B * (kKeys ? d.kv_heads : d.heads) * p.tiles, AM_THREADS, Sh::SMEM + list_bytes(d.S), st,
             m[0].map, m[1].map, m[2].map, m[3].map, p);
  return 0;
}
template <bool kKeys>
int backward_of(const mslt_attention_desc& d, TcParams& p, const MapVal* m, cudaStream_t st, char* err) {
  const int form = form_index(d);
  if (d.head_dim <= 64)
    return form == 0 ? backward<64, kKeys, 0>(d, p, m, st, err) : form == 1 ? backward<64, kKeys, 1>(d, p, m, st, err)
                                                                            : backward<64, kKeys, 2>(d, p, m, st, err);
  return form == 0 ? backward<128, kKeys, 0>(d, p, m, st, err) : form == 1 ? backward<128, kKeys, 1>(d, p, m, st, err)
                                                                           : backward<128, kKeys, 2>(d, p, m, st, err);
}

}  // namespace

int attn_masked_tc_fwd(const mslt_attention_desc& d, int* status, cudaStream_t st, char* err) {
  TcParams p = params_of(d, status, attn_take_starve());
  MapVal m[3];
  int rc = map_of(d.q, d, d.heads, AM_ROWS, &m[0], p.a_perm, err);
  if (!rc) rc = map_of(d.k, d, d.kv_heads, AM_COLS, &m[1], p.b_perm, err);
  if (!rc) rc = map_of(d.v, d, d.kv_heads, AM_COLS, &m[2], p.c_perm, err);
  if (rc) return rc;
  p.o0 = view_of(d.ctx);
  const int form = form_index(d);
  if (d.head_dim <= 64)
    return form == 0 ? forward<64, 0>(d, p, m, st, err) : form == 1 ? forward<64, 1>(d, p, m, st, err) : forward<64, 2>(d, p, m, st, err);
  return form == 0 ? forward<128, 0>(d, p, m, st, err) : form == 1 ? forward<128, 1>(d, p, m, st, err) : forward<128, 2>(d, p, m, st, err);
}

int attn_masked_tc_bwd(const mslt_attention_desc& d, float* delta, int* status, cudaStream_t st, char* err) {
  TcParams p = params_of(d, status, attn_take_starve());
  MapVal mq[4], mk[4];
  TcParams pk = p;
  int rc = map_of(d.q, d, d.heads, AM_ROWS, &mq[0], p.a_perm, err);
  if (!rc) rc = map_of(d.k, d, d.kv_heads, AM_COLS, &mq[1], p.b_perm, err);
  if (!rc) rc = map_of(d.dctx, d, d.heads, AM_ROWS, &mq[2], p.c_perm, err);
  if (!rc) rc = map_of(d.v, d, d.kv_heads, AM_COLS, &mq[3], p.d_perm, err);
  if (!rc) rc = map_of(d.k, d, d.kv_heads, AM_ROWS, &mk[0], pk.a_perm, err);
  if (!rc) rc = map_of(d.q, d, d.heads, AM_COLS, &mk[1], pk.b_perm, err);
  if (!rc) rc = map_of(d.v, d, d.kv_heads, AM_ROWS, &mk[2], pk.c_perm, err);
  if (!rc) rc = map_of(d.dctx, d, d.heads, AM_COLS, &mk[3], pk.d_perm, err);
  if (rc) return rc;
  int log_lanes = 0;
  while ((8 << log_lanes) < d.head_dim) log_lanes++;
  const long long rows = (long long)d.B * d.S * d.heads;
  launch_pdl(masked_delta_tc, (unsigned)(((rows << log_lanes) + 255) / 256), 256, 0, st, view_of(d.dctx), view_of(d.ctx), (const bf16*)d.rest,
             delta, d.S, d.heads, d.head_dim, log_lanes, rows);
  p.delta = pk.delta = delta;
  p.o0 = view_of(d.dq);
  pk.o0 = view_of(d.dk);
  pk.o1 = view_of(d.dv);
  rc = backward_of<false>(d, p, mq, st, err);
  if (!rc) rc = backward_of<true>(d, pk, mk, st, err);
  return rc;
}

}  // namespace mslt
