// Attention under masks in bf16 on the tensor cores, forward and backward, for head widths up to 128 (formulas: mslt.h).
// The scores never reach memory.  Three kernels: a block owns 128 rows of one head at a time (queries in the forward and for
// dQ, keys for dK and dV), and the loop runs over blocks of 64 or 128 rows of the other side that the mask leaves:
//   forward  S = Q K^T                 P = 2^(S' - m)                               O += P V
//   dQ       S = Q K^T, dP = dC V^T    dS = P (dP - delta) dz/ds                    dQ += dS K
//   dK, dV   S^T = K Q^T, dP^T = V dC^T, the same transposed                        dV += P^T dC, dK += dS^T Q
// P and dS are the A operand of the second product and never leave tensor memory: they are written over the scores they
// come from.  dQ and dK, dV are two launches that form S and dP twice (7 products in the place of 5): in return no sum
// crosses blocks, so every run gives the same bits and nothing is added by atomics.
//   warp 0: TMA producer; warp 1: one thread issues the products; the others: softmax, a thread a row (forward: 4 warps) or 32
//   (16) columns of a row (backward, where the rows' sums are known: 16 warps)
// What bounds it.  The exponential unit takes 1024 cycles for 128 x 128 scores, the products 512 in the forward, 768 for dQ and
// 1024 for dK and dV at heads of 64 (twice that at 128).  Around both lies the chain of a step: waits of 150 cycles, reads of
// tensor memory of 100, dependent instructions of three or four warps a scheduler.  So many warps share an SM: heads of 64, four
// forward blocks (128 columns of tensor memory and 80 registers each), sixteen softmax warps of one backward block.
// Measured with 37 tiles a head x 16 heads, all SMs full, cycles of an SM for 128 x 128 scores: forward 1690 (exponential unit
// 59 % busy; without `rest`, which takes 15 % more), dQ 2150 (52 %), dK and dV 2700 (42 %).  Tried on it: two forward blocks of
// double-buffered scores 2240; scores held in registers by three blocks 2330; a quarter to a half of the backward's
// exponentials by polynomial 3 to 12 % slower; eight backward softmax warps of 64 columns 3 % slower; polls with a suspend
// time: level.
//
// Which blocks a row tile visits is worked out once, at its start, from positions, length, prefix and the least and
// greatest document of either side: left out, whole, or with pairs to test.  Documents may be in any order; where they
// are sorted, as in a packed batch, exactly the blocks that hold a common document are visited.  Only blocks with pairs
// to test pay for it: a 32-bit word for 32 columns of a row says which pairs count.
// Rows beyond a sequence may hold anything: those of the row tile give rows that are not stored, those of the other
// side are cleared in shared memory (zero times NaN is NaN) by the softmax warps before the product that contracts over
// them.
#include <math.h>

#include <type_traits>

#include "attn_masked.h"
#include "tc_common.cuh"

namespace mslt {
bool attn_take_starve();  // whether the next attention launch was asked to run out of time (attn_tc.cu)

namespace {

constexpr int AM_ROWS = 128;      // rows of a block
constexpr int AF_COLS = 64;       // rows of a loop block of the forward
constexpr int AF_SOFT = 4, AF_THREADS = 64 + 32 * AF_SOFT;  // forward: softmax warps, threads
constexpr int AB_SOFT = 16, AB_THREADS = 64 + 32 * AB_SOFT;  // backward
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// A row's exponents are relative to a reference: the largest score of the first block in which it sees anything, without its
// bias, rounded up to a whole number (capped scores: none).  Later blocks take no maximum: range is what counts and not
// size, and a row whose probabilities do not add up to something between 2^-64 and 2^64 is the rare exception.  A block with
// such a row goes over its loop again, this time with a running maximum; the reference then moves by whole powers of two,
// so what is there so far is scaled without rounding.  (With a running maximum throughout, a loop block of four
// blocks an SM spent 550 of 2900 cycles on it, and its scores were read a third time; sums tested against the limit block
// by block still cost 450 cycles of a block alone on its SM, 85 of 940 of the SM.)
constexpr float AM_MOST = 1.8446744073709552e19f, AM_LEAST = 5.421010862427522e-20f;  // 2^64, 2^-64

struct View { bf16* p; long long batch, row, head; };
struct TcParams {
  AttnMask m;
  int heads, kv_heads, D, tiles, batch;
  int list_room;        // entries of a list of loop blocks
  View o0, o1;          // ctx | dq | dk, dv
  int wide;             // rows of the outputs allow 32-byte stores
  bf16* rest;
  float* lse;
  const float* delta;
  int* next;            // backward: tiles taken so far beyond the first of every block; zero when the kernel starts
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
__device__ __forceinline__ void tc_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tc_ld16_issue(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tc_ld16_wait(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  tc_ld16_issue(taddr, r);
  tc_ld16_wait(r);
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

// acc += the two bf16 of h, in fp32: one instruction each, where unpacking takes two more
__device__ __forceinline__ void add_bf16(float2& acc, uint32_t h) {
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "mov.b32 {lo, hi}, %2;\n\t"
      "add.f32.bf16 %0, lo, %0;\n\t"
      "add.f32.bf16 %1, hi, %1;\n\t}"
      : "+f"(acc.x), "+f"(acc.y)
      : "r"(h));
}

// ---- which loop blocks a row tile visits (for the forward: attn_masked.h) ------------------------------

// The same by one warp, which runs ahead of the others: blocks of the persistent backward kernels.
template <bool kKeys, int kCols>
__device__ __forceinline__ int list_blocks_warp(const AttnMask& m, const Seq& s, int b, int r0, uint16_t* list) {
  const int lane = threadIdx.x & 31;
  const int* docs = m.docs ? m.docs + (long long)b * m.S : nullptr;
  if (r0 >= s.len) return 0;
  const int r1 = min(r0 + AM_ROWS, s.len) - 1;
  auto range = [&](int c0, int rows, int (&d)[4], int* lo, int* hi) {  // of the documents of rows c0 + 32 e + lane
    int mn = 0x7fffffff, mx = (int)0x80000000;
#pragma unroll
    for (int e = 0; e < 4; e++)
      if (32 * e < rows && c0 + 32 * e + lane < s.len) {
        mn = min(mn, d[e]);
        mx = max(mx, d[e]);
      }
    *lo = __reduce_min_sync(0xffffffffu, mn);
    *hi = __reduce_max_sync(0xffffffffu, mx);
  };
  auto ask = [&](int c0, int rows, int (&d)[4]) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const int c = c0 + 32 * e + lane;
      d[e] = 32 * e < rows && c < s.len ? docs[c] : 0;
    }
  };
  int lo = 0, hi = 0;
  if (docs) {
    int d[4];
    ask(r0, AM_ROWS, d);
    range(r0, AM_ROWS, d, &lo, &hi);
  }
  const int first = kKeys && r0 >= s.prefix ? r0 / kCols : 0;
  const int last = ((kKeys ? s.len : min(s.len, max(r1 + 1, s.prefix))) + kCols - 1) / kCols;
  int n = 0;
  constexpr int kAhead = 4;
  for (int base = first; base < last; base += kAhead) {
    int d[kAhead][4];
    if (docs)
#pragma unroll
      for (int u = 0; u < kAhead; u++) ask((base + u) * kCols, kCols, d[u]);
#pragma unroll
    for (int u = 0; u < kAhead; u++) {
      const int blk = base + u, c0 = blk * kCols;
      if (blk >= last) break;
      bool visit = true;
      bool whole = c0 + kCols <= s.len && (kKeys ? (c0 >= r1 || r1 < s.prefix) : (c0 + kCols - 1 <= r0 || c0 + kCols <= s.prefix));
      if (docs) {
        int mn, mx;
        range(c0, kCols, d[u], &mn, &mx);
        visit = mn <= hi && mx >= lo;
        whole = whole && lo == hi && mn == lo && mx == lo;
      }
      if (visit) {
        if (lane == 0) list[n] = (uint16_t)(blk * 2 + !whole);
        n++;
      }
    }
  }
  return n;
}

// Which of the 32 loop rows from c0 on row r counts a pair with; the whole warp.  The loop rows' documents lie one a lane;
// the warp's own rows seldom hold more than two or three, and each of those takes one ballot for all rows that have it.
// other: the document of loop row c0 + lane, asked for a step ahead.
template <bool kKeys>
__device__ __forceinline__ uint32_t visible(const Seq& s, int r, int c0, bool docs, int doc, int other) {
  const int end = (kKeys ? s.len : min(s.len, max(r + 1, s.prefix))) - c0;
  const int begin = (kKeys && r >= s.prefix ? r : 0) - c0;
  uint32_t w = end >= 32 ? 0xffffffffu : end <= 0 ? 0u : (1u << end) - 1;
  if (begin > 0) w = begin >= 32 ? 0u : w & ~((1u << begin) - 1);
  if (docs) {
    uint32_t same = 0, todo = 0xffffffffu;
    while (todo) {
      const int v = __shfl_sync(0xffffffffu, doc, __ffs(todo) - 1);
      const uint32_t has = __ballot_sync(0xffffffffu, other == v);
      if (doc == v) same = has;
      todo &= ~__ballot_sync(0xffffffffu, doc == v);
    }
    w &= same;
  }
  return w;
}

// ---- scores ---------------------------------------------------------------------------------------------

// How a dot product becomes an exponent of two: 0: s scale log2(e), scale > 0; 1: a bias by distance, or a scale <= 0; 2:
// capped (and perhaps biased).
//
// The cap, cap tanh(z / cap).  The hardware's tanh has an error of 2^-11 of the value: a probability off by 2 % at a score of
// 50.  Where |z| <= 3/8 cap throughout a warp's piece, as nearly always, tanh(u) is u times a polynomial of degree 3 in u^2
// (least greatest error on u^2 <= 9/64, 5.8e-8 of the value), on the multiply-add pipe and with all constants folded in;
// beyond, 1 - 2 / (1 + e^(2u)), two special functions on top of the exponential's one, absolute error 2e-7.  (Degree 5 up
// to 3/4 cap: forward of 2 x 12 x 4096 keys 247 us.)
struct Form { float sl2, slope2, cap2, inv_cap2, z_by, small, b[4]; };
template <int kForm>
__device__ __forceinline__ Form form_of(const AttnMask& m, int h) {
  Form f;
  f.sl2 = m.scale * LOG2E;
  f.slope2 = kForm >= 1 && m.slopes ? m.slopes[h] * LOG2E : 0.f;
  if (kForm == 2) {
    constexpr float kT[4] = {0.999999942f, -0.333319918f, 0.132848227f, -0.0482874447f};
    const float k = m.scale / m.cap;
    f.cap2 = m.cap * LOG2E;
    f.inv_cap2 = 1.f / f.cap2;
    f.z_by = k * (2.f * LOG2E);  // 2^(s z_by) = e^(2 z / cap)
    float by = f.cap2 * k;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      f.b[i] = kT[i] * by;
      by *= k * k;
    }
    f.small = isinf(f.b[3]) ? -1.f : 0.375f / fabsf(k);  // caps far below the scale: no polynomial
  }
  return f;
}
// A warp's piece of 32 (or 16) columns: what is the same for all of it.  side: 0 the distance of pairs needs its absolute value, 1
// all columns lie before all rows of the warp, -1 behind; then the bias is linear in the column.
struct Piece { float off; int side; bool small; };
template <int kForm, int N>
__device__ __forceinline__ Piece piece_of(const Form& f, int r, int c0, const uint32_t (&s)[N]) {
  Piece p;
  p.off = (float)(c0 - r);
  const int r_first = r - (int)(threadIdx.x & 31);
  p.side = c0 + N - 1 <= r_first ? 1 : c0 >= r_first + 31 ? -1 : 0;
  p.small = true;
  if (kForm == 2) {
    float m = 0.f;
#pragma unroll
    for (int c = 0; c < N; c += 2) m = fmaxf(m, fmaxf(fabsf(__uint_as_float(s[c])), fabsf(__uint_as_float(s[c + 1]))));
    p.small = __all_sync(0xffffffffu, m <= f.small);
  }
  return p;
}
// What a piece needs is decided once for all of it: BIAS 0 none, 1 linear in the column, 2 by absolute value; CAP 0 none, 1 the
// polynomial, 2 special functions; TEST: pairs to test.  (Decided pair by pair, the instructions of the other ways are
// issued too, without effect: 710 in the place of 400 for the 64 columns of a row, twice the time with a bias.)
template <int kBias, int kCap, bool kTest> struct Way { static constexpr int BIAS = kBias, CAP = kCap; static constexpr bool TEST = kTest; };
template <int kForm, typename F>
__device__ __forceinline__ void choose_way(const Form& f, const Piece& p, bool test, F&& body) {
  if (kForm == 0) {
    if (test) body(Way<0, 0, true>()); else body(Way<0, 0, false>());
  } else if (kForm == 1) {
    if (test) body(Way<2, 0, true>());
    else if (p.side) body(Way<1, 0, false>());
    else body(Way<2, 0, false>());
  } else if (f.slope2 == 0.f) {
    if (p.small) { if (test) body(Way<0, 1, true>()); else body(Way<0, 1, false>()); }
    else body(Way<0, 2, true>());
  } else {
    if (p.small && !test) body(Way<2, 1, false>());
    else body(Way<2, 2, true>());
  }
}
// exponents of columns c and c + 1 of the piece, plus nb; bend: derivative of the cap
template <typename Wy, bool kBend>
__device__ __forceinline__ float2 exponents(const Form& f, const Piece& p, float2 s, int c, float2 nb, float2* bend) {
  float2 t = nb;
  if (Wy::BIAS == 1) {
    const float by = p.side > 0 ? f.slope2 : -f.slope2, at = by * p.off;
    t = __fadd2_rn(nb, make_float2(fmaf(by, (float)c, at), fmaf(by, (float)(c + 1), at)));
  }
  if (Wy::BIAS == 2) t = make_float2(fmaf(-f.slope2, fabsf(p.off + (float)c), nb.x), fmaf(-f.slope2, fabsf(p.off + (float)(c + 1)), nb.y));
  if (Wy::CAP == 0) return __ffma2_rn(s, splat2(f.sl2), t);
  if (Wy::CAP == 1) {
    const float2 y = __fmul2_rn(s, s);
    float2 q = splat2(f.b[3]);
#pragma unroll
    for (int i = 2; i >= 0; i--) q = __ffma2_rn(q, y, splat2(f.b[i]));
    if (!kBend) return __ffma2_rn(s, q, t);
    const float2 v = __fmul2_rn(s, q), th = __fmul2_rn(v, splat2(f.inv_cap2));
    *bend = __ffma2_rn(make_float2(-th.x, -th.y), th, splat2(1.f));
    return __fadd2_rn(v, t);
  }
  const float2 th = make_float2(fmaf(-2.f, rcp(1.f + ex2(s.x * f.z_by)), 1.f), fmaf(-2.f, rcp(1.f + ex2(s.y * f.z_by)), 1.f));
  if (kBend) *bend = __ffma2_rn(make_float2(-th.x, -th.y), th, splat2(1.f));
  return __ffma2_rn(splat2(f.cap2), th, t);
}

// ---- pieces of the roles ----------------------------------------------------------------------------------

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
// D (+)= A B over kRows rows of B, each of DP contiguous elements.  A lies in tensor memory, 16 kRun of the contraction in
// 8 kRun columns, the next ones `a_step` columns on.
template <int kRows, int kRun>
__device__ __forceinline__ void product_ts(uint32_t d, uint32_t a, uint32_t a_step, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  const uint32_t hi = (uint32_t)(make_smem_desc(0, 16) >> 32), lo = (uint32_t)make_smem_desc(0, kRows * 128);
#pragma unroll
  for (int k = 0; k < kRows / 16; k++)
    tc_mma_ts(d, a + (k / kRun) * a_step + (k % kRun) * 8, ((uint64_t)hi << 32) | (lo + addr16(b) + k * 128), idesc, accumulate | (k > 0));
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

// Rows `from` on of a loop block's tiles of kRows rows become zero; the whole softmax group, thread t of kThreads.
template <int DP, int kRows, int kThreads>
__device__ __forceinline__ void clear_rows(uint8_t* tile, int from, int t) {
#pragma unroll
  for (int kb = 0; kb < DP / 64; kb++)
    for (int v = from * 8 + t; v < kRows * 8; v += kThreads)
      reinterpret_cast<uint4*>(tile + kb * kRows * 128)[v] = make_uint4(0, 0, 0, 0);
}

// 16 elements to memory, or the first 8 of them; wide: 32-byte stores.  A lane's row is its own 128-byte line, and a store takes the
// load/store unit a cycle a line, so half as many stores are half the time (16-byte ones: 1650 cycles a tile of dQ, 3900 of
// dK and dV).
__device__ __forceinline__ void store16(bf16* dst, const uint32_t (&h)[8], bool wide, bool both) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]),
                 "r"(h[4]), "r"(h[5]), "r"(h[6]), "r"(h[7])
                 : "memory");
  } else {
    *reinterpret_cast<uint4*>(dst) = make_uint4(h[0], h[1], h[2], h[3]);
    if (both) *reinterpret_cast<uint4*>(dst + 8) = make_uint4(h[4], h[5], h[6], h[7]);
  }
}
// Columns [c0, c1) of a row of an accumulator, scaled, to bf16 in memory (from dst on), 16 at a time; optionally what the
// rounding took off.  zero: zeros whatever the accumulator holds; have: there is one.
__device__ __forceinline__ void store_row(uint32_t taddr, bf16* dst, bf16* rest, float f, bool zero, bool have, bool write, bool wide, int c0,
                                          int c1, int D) {
#pragma unroll 2
  for (int c = c0; c < c1; c += 16) {
    uint32_t r[16];
    if (have) tc_ld16(taddr + c, r);
    if (zero || !have) {
#pragma unroll
      for (int e = 0; e < 16; e++) r[e] = 0;
    }
    if (!write || c >= D) continue;
    uint32_t hi[8], lo[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float x = __uint_as_float(r[2 * e]) * f, y = __uint_as_float(r[2 * e + 1]) * f;
      hi[e] = pack2(x, y);
      const float2 b = bf162_to_f2(hi[e]);
      lo[e] = pack2(x - b.x, y - b.y);
    }
    store16(dst + c, hi, wide && c + 16 <= D, c + 16 <= D);
    if (rest) store16(rest + c, lo, wide && c + 16 <= D, c + 16 <= D);
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

// Heads of up to 64: 128 columns of tensor memory, four blocks an SM.  Wider ones need 256, so two blocks an SM have two
// buffers of scores each.
template <int DP> struct FwdShape {
  static constexpr int BLOCKS = DP == 64 ? 4 : 2, SB = DP == 64 ? 1 : 2, STAGES = 2;
  static constexpr int COLS = DP == 64 ? 128 : 256, O_COL = SB * 64;
  static constexpr int Q_BYTES = AM_ROWS * DP * 2, KV_BYTES = AF_COLS * DP * 2;
  static constexpr int SMEM = Q_BYTES + 2 * STAGES * KV_BYTES;
};

// x less the two bf16 of h, as bf16
__device__ __forceinline__ uint32_t less_bf16(float2 x, uint32_t h) {
  float lo, hi;
  asm("{\n\t.reg .b16 l, h;\n\t"
      "mov.b32 {l, h}, %2;\n\t"
      "sub.f32.bf16 %0, l, %3;\n\t"
      "sub.f32.bf16 %1, h, %4;\n\t}"
      : "=f"(lo), "=f"(hi)
      : "r"(h), "f"(x.x), "f"(x.y));
  return pack2(-lo, -hi);
}

// Probabilities of 32 columns: 2^(exponent - base), rounded to bf16; sums of the rounded and of the unrounded ones.  see: the
// columns that count, all of them where there is nothing to test.  kRest: what the rounding took off follows the rounded ones
// (and their sum is not needed).
template <int kForm, bool kRest>
__device__ __forceinline__ void probabilities(const Form& f, const Piece& pc, const uint32_t (&s)[32], bool test, uint32_t see,
                                              float base, uint32_t (&pk)[16], uint32_t (&rest)[16], float2& sum, float2& exact) {
  choose_way<kForm>(f, pc, test, [&](auto way) {
    typedef decltype(way) Wy;
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
      float2 e = exponents<Wy, false>(f, pc, make_float2(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), c, splat2(-base), nullptr);
      if (Wy::TEST) {
        e.x = see >> c & 1 ? e.x : -INFINITY;
        e.y = see >> (c + 1) & 1 ? e.y : -INFINITY;
      }
      e.x = ex2(e.x);
      e.y = ex2(e.y);
      pk[c / 2] = pack2(e.x, e.y);
      exact = __fadd2_rn(exact, e);
      if (kRest) rest[c / 2] = less_bf16(e, pk[c / 2]);
      else add_bf16(sum, pk[c / 2]);
    }
  });
}
// Upper bound of the exponents of 32 columns that a row sees (-infinity: none), near enough to the largest to be the
// reference of the row's exponents: without a bias it is the largest, with one it is above by at most 31 slopes, which
// costs nothing but range while a slope is at most one power of two (a larger one is taken element by element).  unbiased:
// as if the pairs were at distance 0, which bounds blocks to come too.
template <int kForm>
__device__ __forceinline__ float largest(const Form& f, const Piece& pc, const uint32_t (&s)[32], bool test, uint32_t see, bool unbiased) {
  float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  if (kForm == 0 || (kForm == 1 && f.sl2 > 0.f && f.slope2 >= 0.f && (unbiased || f.slope2 <= 1.f))) {
    if (test) {
#pragma unroll
      for (int c = 0; c < 32; c += 2) {
        const float x = see >> c & 1 ? __uint_as_float(s[c]) : -INFINITY, y = see >> (c + 1) & 1 ? __uint_as_float(s[c + 1]) : -INFINITY;
        m[c >> 1 & 3] = fmaxf(m[c >> 1 & 3], fmaxf(x, y));
      }
    } else {
#pragma unroll
      for (int c = 0; c < 32; c += 2) m[c >> 1 & 3] = fmaxf(m[c >> 1 & 3], fmaxf(__uint_as_float(s[c]), __uint_as_float(s[c + 1])));
    }
    const float big = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])) * f.sl2;
    if (kForm == 0 || unbiased) return big;
    return big - f.slope2 * (pc.off > 0.f ? pc.off : fmaxf(0.f, -31.f - pc.off));
  }
  choose_way<kForm>(f, pc, test, [&](auto way) {
    typedef decltype(way) Wy;
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
      float2 e = exponents<Wy, false>(f, pc, make_float2(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), c, splat2(0.f), nullptr);
      if (Wy::TEST) {
        e.x = see >> c & 1 ? e.x : -INFINITY;
        e.y = see >> (c + 1) & 1 ? e.y : -INFINITY;
      }
      m[c >> 1 & 3] = fmaxf(m[c >> 1 & 3], fmaxf(e.x, e.y));
    }
  });
  return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}

template <int DP, int kForm>
__global__ void __launch_bounds__(AF_THREADS, FwdShape<DP>::BLOCKS)
masked_fwd_tc(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
              const __grid_constant__ CUtensorMap tmV, const TcParams p) {
  typedef FwdShape<DP> Sh;
  constexpr int NS = Sh::STAGES, SB = Sh::SB;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* Ks = smem + Sh::Q_BYTES;
  uint8_t* Vs = Ks + NS * Sh::KV_BYTES;
  uint16_t* list = (uint16_t*)(Vs + NS * Sh::KV_BYTES);
  __shared__ uint64_t qfull, kfull[NS], kempty[NS], vfull[NS], vempty[NS], sfull[2], pready[2], odone[2], oall;
  __shared__ uint32_t tmem_slot;
  __shared__ int red[16];
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
      mbar_init(smem_u32(&pready[i]), AF_SOFT);
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
  if (warp == 1) tmem_alloc<Sh::COLS>(&tmem_slot);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_begin();

  // causal: the tiles with the most keys start first; else the tiles of a head side by side, which read the same rows
  const int per = p.heads * p.batch, other = p.m.causal ? (int)blockIdx.x % per : (int)blockIdx.x / p.tiles;
  const int h = other % p.heads, b = other / p.heads;
  const int tile = p.m.causal ? p.tiles - 1 - (int)blockIdx.x / per : (int)blockIdx.x % p.tiles;
  const int hk = h / (p.heads / p.kv_heads), r0 = tile * AM_ROWS;
  const Seq s = sequence(p.m, b);
  const int n = list_blocks<false, AF_THREADS / 32, AM_ROWS, AF_COLS>(p.m, s, b, r0, list, red);

  // state of a softmax thread, which owns a query
  const int quarter = warp & 3, r = r0 + quarter * 32 + lane;
  const uint32_t trow = tmem + ((uint32_t)(quarter * 32) << 16);
  const Form f = form_of<kForm>(p.m, h);
  const int* docs = p.m.docs ? p.m.docs + (long long)b * p.m.S : nullptr;
  const int doc = docs && r < s.len ? docs[r] : 0;
  // Capped scores lie in [-cap, cap]: a cap of up to 30 (2^44, and 2^17 keys) needs no reference.
  const bool fixed = kForm == 2 && f.cap2 <= 44.f && f.slope2 >= 0.f;
  float top = 0.f;                                                      // reference of the row's exponents, a whole number
  float2 sum = make_float2(0.f, 0.f), exact = make_float2(0.f, 0.f);   // of the rounded probabilities, and of the unrounded ones
  bool ok = true;

  // Steps are counted on through both goes over the loop, so that the barriers' phases go on too.
  for (int go = 0; go < 2 && n > 0; go++) {
    const int j0 = go * n, j1 = j0 + n;
    bool again = false;
    if (warp == 0 && !p.starve && elect_one()) {
      // ------------------------------- TMA producer -------------------------------
      if (go == 0) {
        mbar_expect_tx(smem_u32(&qfull), Sh::Q_BYTES);
        load_rows<DP>(smem_u32(smem), &tmQ, p.a_perm, smem_u32(&qfull), r0, h, b, 16384);
      }
      int k_issued = j0, v_issued = j0;
      for (int j = j0; j < j1; j++) {
        const int st = j % NS, row = (list[j - j0] >> 1) * AF_COLS;
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
      if (v_issued < j1 || *abort_flag) {
        drain(&qfull, 0);
        for (int j = max(0, k_issued - NS); j < k_issued; j++) drain(&kfull[j % NS], (j / NS) & 1);
        for (int j = max(0, v_issued - NS); j < v_issued; j++) drain(&vfull[j % NS], (j / NS) & 1);
      }
    } else if (warp == 1 && elect_one()) {
      // ------------------------------- products -------------------------------
      constexpr uint32_t id_s = idesc_of(AF_COLS, false), id_o = idesc_of(DP, true);
      auto landed = [&](uint64_t* bar, int j) { return mbar_wait(smem_u32(&bar[j % NS]), j / NS & 1, abort_flag, p.status); };
      auto scores = [&](int j) {
        const int st = j % NS;
        product_ss<DP>(tmem + (j % SB) * 64, smem_u32(smem), 1024, smem_u32(Ks + st * Sh::KV_BYTES), 512, id_s);
        tc_commit(smem_u32(&sfull[j & 1]));
        tc_commit(smem_u32(&kempty[st]));
      };
      // What is not the probabilities is waited for ahead of them: from their arrival to the next scores there is one wait.
      bool fine = mbar_wait(smem_u32(&qfull), 0, abort_flag, p.status) && landed(kfull, j0);
      if (fine) {
        tc_fence_after();
        scores(j0);
      }
      for (int j = j0; j < j1 && fine; j++) {
        const int st = j % NS;
        if (j + 1 < j1) {
          if (!landed(kfull, j + 1)) { fine = false; break; }
          if (SB == 2) {
            tc_fence_after();
            scores(j + 1);
          }
        }
        fine = landed(vfull, j) && mbar_wait(smem_u32(&pready[j & 1]), j >> 1 & 1, abort_flag, p.status);
        if (!fine) break;
        tc_fence_after();
        product_ts<AF_COLS, 2>(tmem + Sh::O_COL, tmem + (j % SB) * 64, 32, smem_u32(Vs + st * Sh::KV_BYTES), id_o, j > j0);
        if (p.rest) product_ts<AF_COLS, 2>(tmem + Sh::O_COL, tmem + (j % SB) * 64 + 16, 32, smem_u32(Vs + st * Sh::KV_BYTES), id_o, 1);
        if (SB == 2) tc_commit(smem_u32(&odone[j & 1]));
        // one buffer: the probabilities lie in it until the product with V, issued before, has read them
        if (SB == 1 && j + 1 < j1) scores(j + 1);
        tc_commit(smem_u32(&vempty[st]));
      }
      if (fine) tc_commit(smem_u32(&oall));
      if (!fine || *abort_flag) settle(&oall);
    } else if (warp >= 2) {
      // ------------------------------- softmax -------------------------------
      bool settled = fixed && go == 0;  // every row of the warp has its reference
      top = settled || r >= s.len ? 0.f : -INFINITY;
      sum = exact = make_float2(0.f, 0.f);
      uint32_t seen = 0;
      int others[2] = {0, 0};  // documents of the next step's keys
      auto ask = [&](int entry) {
        if (!docs || !(entry & 1)) return;
        const int c = (entry >> 1) * AF_COLS + lane;
        others[0] = c < s.len ? docs[c] : 0;
        others[1] = c + 32 < s.len ? docs[c + 32] : 0;
      };
      ask(list[0]);
      for (int j = j0; j < j1; j++) {
        const int entry = list[j - j0], c0 = (entry >> 1) * AF_COLS;
        const bool test = entry & 1;
        uint32_t see[2] = {~0u, ~0u};
        if (test) {
          see[0] = visible<false>(s, r, c0, docs != nullptr, doc, others[0]);
          see[1] = visible<false>(s, r, c0 + 32, docs != nullptr, doc, others[1]);
        }
        if (j + 1 < j1) ask(list[j + 1 - j0]);
        seen |= see[0] | see[1];
        if (!mbar_wait(smem_u32(&sfull[j & 1]), j >> 1 & 1, abort_flag, p.status)) { ok = false; break; }
        tc_fence_after();
        const uint32_t tS = trow + (j % SB) * 64;
        uint32_t a[32];
        if (!settled) {
          float big = -INFINITY;
#pragma unroll
          for (int half = 0; half < 2; half++) {
            tc_ld32_issue(tS + 32 * half, a);
            tc_ld32_wait(a);
            big = fmaxf(big, largest<kForm>(f, piece_of<kForm>(f, r, c0 + 32 * half, a), a, test, see[half], go == 0));
          }
          float up = 0.f;
          if (top == -INFINITY) top = ceilf(big);   // has seen nothing yet: sums and accumulator are zero
          else if (go == 1 && big > top) up = ceilf(big - top);
          if (go == 1 && __any_sync(0xffffffffu, up > 0.f)) {
            const float by = ex2(-up);
            top += up;
            sum = __fmul2_rn(sum, splat2(by));
            exact = __fmul2_rn(exact, splat2(by));
            if (j > j0) {
              // The accumulator of the blocks so far.  One buffer of scores: they were issued behind the last product with V.
              // Two: the scores at hand only say that the product before the last is complete, hence two barriers, so that
              // neither can be a phase ahead.
              if (SB == 2 && !mbar_wait(smem_u32(&odone[(j - 1) & 1]), (j - 1) >> 1 & 1, abort_flag, p.status)) { ok = false; break; }
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < DP; c += 16) {
                uint32_t o[16];
                tc_ld16(trow + Sh::O_COL + c, o);
#pragma unroll
                for (int e = 0; e < 16; e++) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
                tc_st16(trow + Sh::O_COL + c, o);
              }
            }
          }
          settled = go == 0 && __all_sync(0xffffffffu, top != -INFINITY);
        }
        const float base = top == -INFINITY ? 0.f : top;
        // The probabilities of a half take 16 of the 32 columns of scores that were read for it.  A training step's context is
        // formed from more than bf16 holds of them: what their rounding takes off goes to the other 16 columns and
        // through a second product.  The backward's delta = dC . C follows the probabilities to 2^-16 then, and rows of the
        // scores' gradient sum to zero; with the rounded ones alone dQ was off by 2.6e-3 of its norm where the roundings of
        // dS and dQ themselves make 2.4e-3.
#pragma unroll
        for (int half = 0; half < 2; half++) {
          tc_ld32_issue(tS + 32 * half, a);
          tc_ld32_wait(a);
          uint32_t pk[16], rest[16];
          const Piece pc = piece_of<kForm>(f, r, c0 + 32 * half, a);
          if (p.rest) {
            probabilities<kForm, true>(f, pc, a, test, see[half], base, pk, rest, sum, exact);
            tc_st16(tS + 32 * half + 16, rest);
          } else {
            probabilities<kForm, false>(f, pc, a, test, see[half], base, pk, rest, sum, exact);
          }
          tc_st16(tS + 32 * half, pk);
        }
        tc_st_wait();
        if (test && s.len < c0 + AF_COLS) {
          if (!mbar_wait(smem_u32(&vfull[j % NS]), j / NS & 1, abort_flag, p.status)) { ok = false; break; }
          clear_rows<DP, AF_COLS, 32 * AF_SOFT>(Vs + (j % NS) * Sh::KV_BYTES, s.len - c0, threadIdx.x - 64);
          fence_proxy_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&pready[j & 1]));
      }
      if (ok) ok = mbar_wait(smem_u32(&oall), go, abort_flag, p.status);
      const float total = exact.x + exact.y;
      again = ok && seen && r < s.len && !(total >= AM_LEAST && total <= AM_MOST);
    }
    if (!__syncthreads_or(again) || *abort_flag) break;
  }

  if (warp >= 2 && ok) {
    tc_fence_after();
    const float total = p.rest ? exact.x + exact.y : sum.x + sum.y;
    const bool empty = r >= s.len || total == 0.f;  // NaN is not
    const long long at = b * p.o0.batch + r * p.o0.row + h * p.o0.head;
    store_row(trow + Sh::O_COL, p.o0.p + at, p.rest ? p.rest + at : nullptr, empty ? 0.f : 1.f / total, empty, n > 0, r < p.m.S, p.wide, 0, DP,
              p.D);
    if (p.lse && r < p.m.S)
      p.lse[((long long)b * p.heads + h) * p.m.S + r] = empty ? -INFINITY : (top + log2f(exact.x + exact.y)) * LN2;
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_free<Sh::COLS>(tmem);
  }
}

// ---- backward ---------------------------------------------------------------------------------------------

// delta_i = dC_i . (C_i + rest_i), and the counters of the kernels behind it: eight elements a lane, the lanes of a row side by side
__global__ void __launch_bounds__(256)
masked_delta_tc(const View dc, const View c, const bf16* rest, float* delta, int* next, int S, int heads, int D, int log_lanes, long long rows) {
  pdl_begin();
  if (blockIdx.x == 0 && threadIdx.x < 2) next[threadIdx.x] = 0;
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

// Tensor memory, loop blocks and stages of the two backward kernels.  Heads of 64: S 2 x 128 columns (the next block's
// products run under this block's softmax), dP 128 (read at once, so the next one follows soon), the accumulators 64 or
// 128.  Wider heads, dQ: the same with an accumulator of 128.  Wider heads, dK and dV: 256 columns of accumulators leave
// 256, two blocks of 64 x (S, dP).  (One of 128 x (S, dP): products and softmax take turns, 2 x 12 x 4096 x 128 in 877 us.)
template <int DP, bool kKeys> struct BwdShape {
  static constexpr int LOOP = DP == 128 && kKeys ? 64 : 128;      // rows of a loop block
  static constexpr int SB = 2, PB = DP == 128 && kKeys ? 2 : 1;   // buffers of S, of dP
  static constexpr int FB = DP == 64 ? 2 : 1;                     // buffers of the row tiles
  static constexpr int STAGES = DP == 128 && !kKeys ? 2 : 4;
  static constexpr int COLS = 512;
  static constexpr int DP_COL = SB * LOOP, ACC_COL = DP_COL + PB * LOOP;
  static constexpr int PART = LOOP / 4;                           // columns of a softmax thread
  static constexpr int FIX_BYTES = AM_ROWS * DP * 2, LOOP_BYTES = LOOP * DP * 2;
  static constexpr int SMEM = FB * 2 * FIX_BYTES + STAGES * 2 * LOOP_BYTES;
};
static_assert(BwdShape<64, true>::ACC_COL + 2 * 64 <= 512 && BwdShape<128, false>::ACC_COL + 128 <= 512 &&
              BwdShape<128, true>::ACC_COL + 2 * 128 <= 512, "tensor memory");

// kKeys = false: rows are queries (A = q, B = k, C = dctx, D = v; loop over keys), the result is dq.
// kKeys = true: rows are keys (A = k, B = q, C = v, D = dctx; loop over the queries of every head that shares them): dk, dv.
// Persistent, a block an SM: row tiles as they come (from a counter: which block takes a tile changes no sum), steps counted on
// from tile to tile so that the barriers' phases go on.  The producer warp works out a tile's list and asks for its rows while
// the tile before is under way; only the reading of the accumulators lies between two tiles.  (8 x 12 x 2048 in 6 documents: a
// block a tile 344 us, persistent blocks with tiles in turn 300, so 276.)
template <int DP, bool kKeys, int kForm>
__global__ void __launch_bounds__(AB_THREADS, 1)
masked_bwd_tc(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
              const __grid_constant__ CUtensorMap tmC, const __grid_constant__ CUtensorMap tmD, const TcParams p) {
  enum { I_LIST, I_LEN, I_PREFIX, I_ROW, I_HEAD, I_BATCH };  // entries of its list (-1: no tile), length, prefix, first row, head, sequence
  typedef BwdShape<DP, kKeys> Sh;
  constexpr int NS = Sh::STAGES, FB = Sh::FB, SB = Sh::SB, PB = Sh::PB, LOOP = Sh::LOOP, PART = Sh::PART;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);  // row tiles: A then C
  uint8_t* Bs = smem + FB * 2 * Sh::FIX_BYTES;                                  // stage: B then D
  uint16_t* lists = (uint16_t*)(Bs + NS * 2 * Sh::LOOP_BYTES);                  // two
  __shared__ uint64_t fixfull[FB], fixempty[FB], full[NS], empty[NS], sfull[2], ready[2], dpread, done, accfree, listfull[2], listempty[2];
  __shared__ uint32_t tmem_slot;
  __shared__ int info[2][8];                                                    // of a tile: see I_*
  __shared__ __align__(16) float cols_of[kKeys ? AB_SOFT : 1][2][32];           // kKeys: -lse (log2) and -delta of a warp's queries
  __shared__ __align__(8) int flag_mem[4];
  volatile int* abort_flag = flag_mem + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < FB; i++) {
      mbar_init(smem_u32(&fixfull[i]), 1);
      mbar_init(smem_u32(&fixempty[i]), 1);
    }
    for (int i = 0; i < NS; i++) {
      mbar_init(smem_u32(&full[i]), 1);
      mbar_init(smem_u32(&empty[i]), 1);
    }
    for (int i = 0; i < 2; i++) {
      mbar_init(smem_u32(&sfull[i]), 1);
      mbar_init(smem_u32(&ready[i]), AB_SOFT);
      mbar_init(smem_u32(&listfull[i]), 1);
      mbar_init(smem_u32(&listempty[i]), AB_SOFT + 1);
    }
    mbar_init(smem_u32(&dpread), AB_SOFT);
    mbar_init(smem_u32(&done), 1);
    mbar_init(smem_u32(&accfree), AB_SOFT);
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

  const int row_heads = kKeys ? p.kv_heads : p.heads, group = p.heads / p.kv_heads, spans = kKeys ? group : 1;
  const int items = p.tiles * row_heads * p.batch;
  struct Item { int r0, hr, b; };
  auto item_at = [&](int w) {
    Item it;
    if (p.m.causal) {  // the tiles with the longest loops first
      const int per = row_heads * p.batch, t = w / per, x = w - t * per;
      it.b = x / row_heads;
      it.hr = x - it.b * row_heads;
      it.r0 = (kKeys ? t : p.tiles - 1 - t) * AM_ROWS;
    } else {           // tiles of a head side by side: they read the same rows
      const int x = w / p.tiles;
      it.r0 = (w - x * p.tiles) * AM_ROWS;
      it.b = x / row_heads;
      it.hr = x - it.b * row_heads;
    }
    return it;
  };

  if (warp == 0 && !p.starve) {
    // ------------------------------- producer -------------------------------
    int g = 0, tiles_done = 0, i = 0;  // steps and tiles so far
    bool ok = true;
    int taken = 0;
    for (int w = blockIdx.x;; w = (int)gridDim.x + __shfl_sync(0xffffffffu, taken, 0), i++) {
      const Item it = item_at(min(w, items - 1));
      const int slot = i & 1;
      if (lane == 0 && w < items) taken = atomicAdd(p.next, 1);  // asked for a tile ahead
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&listempty[slot]), (uint32_t)(i >> 1 & 1) ^ 1, abort_flag, p.status));
      int n_list = 0;
      uint16_t* list = lists + slot * p.list_room;
      if (ok && w >= items) {
        if (lane == 0) {
          info[slot][I_LIST] = -1;  // no more tiles
          mbar_arrive(smem_u32(&listfull[slot]));
        }
        break;
      }
      if (ok) {
        const Seq s = sequence(p.m, it.b);
        n_list = list_blocks_warp<kKeys, LOOP>(p.m, s, it.b, it.r0, list);
        if (lane == 0) {
          info[slot][I_LIST] = n_list;
          info[slot][I_LEN] = s.len;
          info[slot][I_PREFIX] = s.prefix;
          info[slot][I_ROW] = it.r0;
          info[slot][I_HEAD] = it.hr;
          info[slot][I_BATCH] = it.b;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&listfull[slot]));
      }
      const int n = n_list * spans;
      if (ok && n == 0) continue;
      if (elect_one()) {
        const int f = tiles_done % FB;
        int issued = g, fixed = tiles_done;  // steps and row tiles asked for
        const uint32_t fb = smem_u32(&fixfull[f]), fix = smem_u32(smem + f * 2 * Sh::FIX_BYTES);
        ok = ok && mbar_wait(smem_u32(&fixempty[f]), (uint32_t)(tiles_done / FB & 1) ^ 1, abort_flag, p.status);
        if (ok) {
          mbar_expect_tx(fb, 2 * Sh::FIX_BYTES);
          load_rows<DP>(fix, &tmA, p.a_perm, fb, it.r0, it.hr, it.b, 16384);
          load_rows<DP>(fix + Sh::FIX_BYTES, &tmC, p.c_perm, fb, it.r0, it.hr, it.b, 16384);
          fixed = tiles_done + 1;
        }
        int at_list = 0, hl = kKeys ? it.hr * group : it.hr / group;
        for (int j = g; j < g + n && ok; j++) {
          const int st = j % NS, row = (list[at_list] >> 1) * LOOP;
          ok = mbar_wait(smem_u32(&empty[st]), (uint32_t)(j / NS & 1) ^ 1, abort_flag, p.status);
          if (!ok) break;
          const uint32_t bar = smem_u32(&full[st]), dst = smem_u32(Bs + st * 2 * Sh::LOOP_BYTES);
          mbar_expect_tx(bar, 2 * Sh::LOOP_BYTES);
          load_rows<DP>(dst, &tmB, p.b_perm, bar, row, hl, it.b, LOOP * 128);
          load_rows<DP>(dst + Sh::LOOP_BYTES, &tmD, p.d_perm, bar, row, hl, it.b, LOOP * 128);
          issued = j + 1;
          if (++at_list == n_list) {
            at_list = 0;
            hl++;
          }
        }
        if (!ok || *abort_flag) {
          // what has been asked for must have landed before the block leaves
          for (int t = max(0, fixed - FB); t < fixed; t++) drain(&fixfull[t % FB], (t / FB) & 1);
          for (int j = max(0, issued - NS); j < issued; j++) drain(&full[j % NS], (j / NS) & 1);
          ok = false;
        }
      }
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      g += n;
      tiles_done++;
    }
  } else if (warp == 1 && elect_one()) {
    // ------------------------------- products -------------------------------
    constexpr uint32_t id_s = idesc_of(LOOP, false), id_acc = idesc_of(DP, true);
    auto stage = [&](int j) { return smem_u32(Bs + (j % NS) * 2 * Sh::LOOP_BYTES); };
    auto landed = [&](int j) { return mbar_wait(smem_u32(&full[j % NS]), j / NS & 1, abort_flag, p.status); };
    int g = 0, tiles_done = 0, i = 0;
    bool ok = true;
    for (; ok; i++) {
      const int slot = i & 1;
      if (!mbar_wait(smem_u32(&listfull[slot]), i >> 1 & 1, abort_flag, p.status)) { ok = false; break; }
      const int n = info[slot][I_LIST] * spans;
      if (n < 0) break;
      mbar_arrive(smem_u32(&listempty[slot]));
      if (n == 0) continue;
      const int f = tiles_done % FB;
      const uint32_t fix = smem_u32(smem + f * 2 * Sh::FIX_BYTES);
      auto scores = [&](int j) { product_ss<DP>(tmem + (j % SB) * LOOP, fix, 1024, stage(j), LOOP * 8, id_s); };
      auto dprobs = [&](int j) {
        product_ss<DP>(tmem + Sh::DP_COL + (j % PB) * LOOP, fix + Sh::FIX_BYTES, 1024, stage(j) + Sh::LOOP_BYTES, LOOP * 8, id_s);
      };
      // S and dP of step j.  Their buffers: what lay in the scores' was last read by a product issued before; dP, where it has
      // one, by the softmax of the step before.
      auto next = [&](int j) {
        if (!landed(j)) return false;
        tc_fence_after();
        scores(j);
        if (PB == 1 && j > 0) {
          if (!mbar_wait(smem_u32(&dpread), (j - 1) & 1, abort_flag, p.status)) return false;
          tc_fence_after();
        }
        dprobs(j);
        tc_commit(smem_u32(&sfull[j & 1]));
        return true;
      };
      ok = mbar_wait(smem_u32(&fixfull[f]), tiles_done / FB & 1, abort_flag, p.status) && next(g);
      for (int j = g; j < g + n && ok; j++) {
        if (j + 1 < g + n) {
          if (!next(j + 1)) { ok = false; break; }
        } else {
          tc_commit(smem_u32(&fixempty[f]));
        }
        if (!mbar_wait(smem_u32(&ready[j & 1]), j >> 1 & 1, abort_flag, p.status)) { ok = false; break; }
        if (j == g && tiles_done > 0 && !mbar_wait(smem_u32(&accfree), (tiles_done - 1) & 1, abort_flag, p.status)) { ok = false; break; }
        tc_fence_after();
        const uint32_t at = tmem + (j % SB) * LOOP;
        if (kKeys) {
          product_ts<LOOP, 1>(tmem + Sh::ACC_COL, at, 16, stage(j) + Sh::LOOP_BYTES, id_acc, j > g);    // dV += P^T dC
          product_ts<LOOP, 1>(tmem + Sh::ACC_COL + DP, at + 8, 16, stage(j), id_acc, j > g);            // dK += dS^T Q
        } else {
          product_ts<LOOP, 1>(tmem + Sh::ACC_COL, at, 16, stage(j), id_acc, j > g);                     // dQ += dS K
        }
        tc_commit(smem_u32(&empty[j % NS]));
      }
      if (!ok) break;
      tc_commit(smem_u32(&done));
      g += n;
      tiles_done++;
    }
    if (!ok || *abort_flag) settle(&done);
  } else if (warp >= 2) {
    // ------------------ softmax and its backward: a thread owns PART columns of a row ------------------
    const int quarter = warp & 3, part = (warp - 2) >> 2;
    const uint32_t trow = tmem + ((uint32_t)(quarter * 32) << 16) + part * PART;
    int g = 0, tiles_done = 0, i = 0;
    bool ok = true;
    // What the common step does not need stays in shared memory: registers are short.
    const volatile int* it = info[0];
    // lse and delta of the row (queries), or of the lane's column of the next step (keys), and documents of the row and of the
    // next step's columns.  They are asked for ahead and not touched before they are needed (multiplied where they were asked
    // for, they cost 1000 of 2700 cycles a step): a step ahead, and a tile's first ones before the tile before is stored.
    float lse = 0.f, delta = 0.f;
    int doc = 0, other = 0;
    auto ask = [&](int h, int c) {
      const long long at = ((long long)it[I_BATCH] * p.heads + h) * p.m.S + c;
      lse = delta = 0.f;
      if (c < it[I_LEN]) {
        lse = p.lse[at];
        delta = p.delta[at];
      }
    };
    auto ask_step = [&](int head, int entry) {
      const int c = (entry >> 1) * LOOP + part * PART + lane;
      if (kKeys && lane < PART) ask(head, c);
      if ((entry & 1) && p.m.docs) other = c < it[I_LEN] ? p.m.docs[(long long)it[I_BATCH] * p.m.S + c] : 0;
    };
    auto enter = [&](int tile) {  // the block's tile-th tile
      if (!mbar_wait(smem_u32(&listfull[tile & 1]), tile >> 1 & 1, abort_flag, p.status)) return false;
      it = info[tile & 1];
      if (it[I_LIST] < 0) return true;
      const int r = it[I_ROW] + quarter * 32 + lane;
      if (!kKeys) ask(it[I_HEAD], r);
      if (p.m.docs) doc = r < it[I_LEN] ? p.m.docs[(long long)it[I_BATCH] * p.m.S + r] : 0;
      if (it[I_LIST] > 0) ask_step(kKeys ? it[I_HEAD] * group : 0, lists[(tile & 1) * p.list_room]);
      return true;
    };
    ok = enter(0);
    for (; ok && it[I_LIST] >= 0; i++) {
      const int slot = i & 1;
      const int n_list = it[I_LIST], n = n_list * spans, r = it[I_ROW] + quarter * 32 + lane;
      const uint16_t* list = lists + slot * p.list_room;
      Form f = form_of<kForm>(p.m, it[I_HEAD] * spans);
      int at_list = 0, head = kKeys ? it[I_HEAD] * group : it[I_HEAD] / group;  // of step j
      const float lse2 = lse * LOG2E;
      for (int j = g; j < g + n; j++) {
        const int entry = list[at_list], first = (entry >> 1) * LOOP, c0 = first + part * PART;
        const bool test = entry & 1;
        if (kKeys) {
          __syncwarp();
          cols_of[warp - 2][0][lane] = -lse * LOG2E;
          cols_of[warp - 2][1][lane] = -delta;
          __syncwarp();
          if (kForm == 1 || kForm == 2) f.slope2 = p.m.slopes ? p.m.slopes[head] * LOG2E : 0.f;
        }
        uint32_t see = ~0u;
        if (test) {
          Seq s;
          s.len = it[I_LEN];
          s.prefix = it[I_PREFIX];
          see = visible<kKeys>(s, r, c0, p.m.docs != nullptr, doc, other);
        }
        if (++at_list == n_list) {
          at_list = 0;
          head++;
        }
        if (j + 1 < g + n) ask_step(head, list[at_list]);
        if (!mbar_wait(smem_u32(&sfull[j & 1]), j >> 1 & 1, abort_flag, p.status)) { ok = false; break; }
        tc_fence_after();
        const uint32_t tS = trow + (j % SB) * LOOP, tP = trow + Sh::DP_COL + (j % PB) * LOOP;
        // The step by itself, for blocks without and with pairs to test, 16 columns at a time: 32 need more than the 96
        // registers that 576 threads have.
        auto step = [&](auto testing) {
          constexpr bool kTest = decltype(testing)::value;
          const bool tail = kTest && it[I_LEN] < first + LOOP;
#pragma unroll
          for (int q = 0; q < PART; q += 16) {
            uint32_t out[kKeys ? 16 : 8];  // keys: P, then dS; queries: dS
            uint32_t a[16], d[16];
            auto load = [&] {
              tc_ld16_issue(tS + q, a);
              tc_ld16_issue(tP + q, d);
              tc_ld16_wait(a);
              tc_ld16_wait(d);
            };
            auto read = [&] {
              if (PB == 1 && q + 16 == PART) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&dpread));
              }
            };
            load();
            if (!kTest) read();
            const Piece pc = piece_of<kForm>(f, r, c0 + q, a);
            const uint32_t seen = see >> q;
            float most = 0.f;
            auto gradients = [&](auto careful) {
              choose_way<kForm>(f, pc, kTest, [&](auto way) {
                typedef decltype(way) Wy;
                float4 nl4, nd4;
#pragma unroll
                for (int c = 0; c < 16; c += 2) {
                  float2 x = make_float2(__uint_as_float(a[c]), __uint_as_float(a[c + 1]));
                  float2 t = make_float2(__uint_as_float(d[c]), __uint_as_float(d[c + 1]));
                  float2 nl = splat2(-lse2), nd = splat2(-delta), bend = splat2(1.f);
                  if (kKeys) {
                    if (c % 4 == 0) {
                      nl4 = *reinterpret_cast<const float4*>(&cols_of[warp - 2][0][q + c]);
                      nd4 = *reinterpret_cast<const float4*>(&cols_of[warp - 2][1][q + c]);
                    }
                    nl = c % 4 ? make_float2(nl4.z, nl4.w) : make_float2(nl4.x, nl4.y);
                    nd = c % 4 ? make_float2(nd4.z, nd4.w) : make_float2(nd4.x, nd4.y);
                  }
                  x = exponents<Wy, true>(f, pc, x, c, nl, &bend);
                  const bool v0 = !kTest || (seen >> c & 1), v1 = !kTest || (seen >> (c + 1) & 1);
                  x.x = ex2(v0 ? x.x : -INFINITY);
                  x.y = ex2(v1 ? x.y : -INFINITY);
                  t = __fmul2_rn(__fadd2_rn(t, nd), x);
                  if (Wy::CAP) t = __fmul2_rn(t, bend);
                  if (kTest && !decltype(careful)::value) most = fmaxf(most, fmaxf(x.x, x.y));
                  if (decltype(careful)::value) {
                    t.x = v0 && !(x.x > 0.99999f) ? t.x : 0.f;
                    t.y = v1 && !(x.y > 0.99999f) ? t.y : 0.f;
                  }
                  if (kKeys) out[c / 2] = pack2(x.x, x.y);
                  out[(kKeys ? 8 : 0) + c / 2] = pack2(t.x, t.y);
                }
              });
            };
            if (!kTest) {
              gradients(std::false_type());
            } else {
              // Two rare cases are looked at pair by pair.  Columns beyond the sequence, whose dP may be anything.  And a row with
              // a single key, which has no gradient by its score: dP - delta is the difference of two sums in different
              // orders there, and is zero in truth.  p(dP_j - delta) is at most (1 - p) times the spread of dP, so
              // nothing above 1e-5 of it is dropped; a block without pairs to test has as many keys a row as columns, and
              // no such p alone.
              if (!tail) gradients(std::false_type());
              if (tail || __any_sync(0xffffffffu, most > 0.99999f)) {
                if (!tail) load();  // the first time used them up
                gradients(std::true_type());
              }
              read();
            }
            // over the scores that were just read
            if constexpr (kKeys) tc_st16(tS + q, out);
            else tc_st8(tS + q, out);
          }
        };
        if (test) step(std::true_type());
        else step(std::false_type());
        tc_st_wait();
        if (test && it[I_LEN] < first + LOOP) {
          // the products' reads of this stage so far are over (S and dP are complete); its rows are an operand once more
          uint8_t* tiles = Bs + (j % NS) * 2 * Sh::LOOP_BYTES;
          clear_rows<DP, LOOP, 32 * AB_SOFT>(tiles, it[I_LEN] - first, threadIdx.x - 64);
          if (kKeys) clear_rows<DP, LOOP, 32 * AB_SOFT>(tiles + Sh::LOOP_BYTES, it[I_LEN] - first, threadIdx.x - 64);
          fence_proxy_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ready[j & 1]));
      }
      if (!ok) break;
      const int b = it[I_BATCH], hr = it[I_HEAD];
      const bool dead = r >= it[I_LEN], write = r < p.m.S;
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&listempty[slot]));
      if (!enter(i + 1)) { ok = false; break; }
      if (n > 0) {
        if (!mbar_wait(smem_u32(&done), tiles_done & 1, abort_flag, p.status)) { ok = false; break; }
        tc_fence_after();
      }
      const uint32_t acc = tmem + ((uint32_t)(quarter * 32) << 16) + Sh::ACC_COL;
      if (kKeys) {
        const int which = part >> 1;  // 0: dV, 1: dK
        const View& o = which ? p.o0 : p.o1;
        store_row(acc + which * DP, o.p + (b * o.batch + r * o.row + hr * o.head), nullptr, which ? p.m.scale : 1.f, dead, n > 0, write,
                  p.wide, (part & 1) * (DP / 2), ((part & 1) + 1) * (DP / 2), p.D);
      } else {
        store_row(acc, p.o0.p + (b * p.o0.batch + r * p.o0.row + hr * p.o0.head), nullptr, p.m.scale, dead, n > 0, write, p.wide,
                  part * (DP / 4), (part + 1) * (DP / 4), p.D);
      }
      if (n > 0) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&accfree));
        g += n;
        tiles_done++;
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
// whether every head's row starts on 32 bytes
bool aligned32(const mslt_heads& h) { return ((uintptr_t)h.data & 31) == 0 && h.batch % 16 == 0 && h.row % 16 == 0 && h.head % 16 == 0; }
View view_of(const mslt_heads& h) { return View{(bf16*)h.data, h.batch, h.row, h.head}; }

TcParams params_of(const mslt_attention_desc& d, int* status, bool starve) {
  TcParams p;
  memset(&p, 0, sizeof(p));
  p.m = AttnMask{d.S, d.causal != 0, d.scale, d.cap, d.slopes, d.prefix, d.docs, d.lens};
  p.heads = d.heads; p.kv_heads = d.kv_heads; p.D = d.head_dim;
  p.tiles = (d.S + AM_ROWS - 1) / AM_ROWS;
  p.batch = d.B;
  p.list_room = (d.S + AF_COLS - 1) / AF_COLS;
  p.rest = (bf16*)d.rest; p.lse = d.lse;
  p.wait_limit = starve ? 40000000ll : WAIT_LIMIT_CYCLES;  // starved: about 20 ms
  p.starve = starve;
  p.status = status;
  return p;
}
int form_index(const mslt_attention_desc& d) { return d.cap > 0.f ? 2 : d.slopes || !(d.scale > 0.f) ? 1 : 0; }
// shared memory beside the tiles: alignment and the list of blocks.  The largest list (S = 131072) is opted in for.
size_t list_bytes(int S) { return 1024 + ((size_t)(S + AF_COLS - 1) / AF_COLS * 2 + 15) / 16 * 16; }
constexpr size_t kMostList = 1024 + 131072 / AF_COLS * 2;

template <int DP, int kForm>
int forward(const mslt_attention_desc& d, TcParams& p, const MapVal* m, cudaStream_t st, char* err) {
  static bool done[kMaxDevices];
  if (opt_in(masked_fwd_tc<DP, kForm>, done, FwdShape<DP>::SMEM + kMostList, err)) return MSLT_ERR_CUDA;
  launch_pdl(masked_fwd_tc<DP, kForm>, d.B * d.heads * p.tiles, AF_THREADS, FwdShape<DP>::SMEM + list_bytes(d.S), st, m[0].map, m[1].map,
             m[2].map, p);
  return 0;
}
template <int DP, bool kKeys, int kForm>
int backward(const mslt_attention_desc& d, TcParams& p, const MapVal* m, int sms, cudaStream_t st, char* err) {
  static bool done[kMaxDevices];
  typedef BwdShape<DP, kKeys> Sh;
  if (opt_in(masked_bwd_tc<DP, kKeys, kForm>, done, Sh::SMEM + 2 * kMostList, err)) return MSLT_ERR_CUDA;
  const int items = d.B * (kKeys ? d.kv_heads : d.heads) * p.tiles;
  launch_pdl(masked_bwd_tc<DP, kKeys, kForm>, items < sms ? items : sms, AB_THREADS, Sh::SMEM + 2 * list_bytes(d.S), st,
             m[0].map, m[1].map, m[2].map, m[3].map, p);
  return 0;
}
template <bool kKeys>
int backward_of(const mslt_attention_desc& d, TcParams& p, const MapVal* m, int sms, cudaStream_t st, char* err) {
  const int form = form_index(d);
  if (d.head_dim <= 64)
    return form == 0 ? backward<64, kKeys, 0>(d, p, m, sms, st, err) : form == 1 ? backward<64, kKeys, 1>(d, p, m, sms, st, err)
                                                                            : backward<64, kKeys, 2>(d, p, m, sms, st, err);
  return form == 0 ? backward<128, kKeys, 0>(d, p, m, sms, st, err) : form == 1 ? backward<128, kKeys, 1>(d, p, m, sms, st, err)
                                                                           : backward<128, kKeys, 2>(d, p, m, sms, st, err);
}

}  // namespace

int attn_masked_tc_fwd(const mslt_attention_desc& d, int* status, cudaStream_t st, char* err) {
  TcParams p = params_of(d, status, attn_take_starve());
  MapVal m[3];
  int rc = map_of(d.q, d, d.heads, AM_ROWS, &m[0], p.a_perm, err);
  if (!rc) rc = map_of(d.k, d, d.kv_heads, AF_COLS, &m[1], p.b_perm, err);
  if (!rc) rc = map_of(d.v, d, d.kv_heads, AF_COLS, &m[2], p.c_perm, err);
  if (rc) return rc;
  p.o0 = view_of(d.ctx);
  p.wide = aligned32(d.ctx) && ((uintptr_t)d.rest & 31) == 0;
  const int form = form_index(d);
  if (d.head_dim <= 64)
    return form == 0 ? forward<64, 0>(d, p, m, st, err) : form == 1 ? forward<64, 1>(d, p, m, st, err) : forward<64, 2>(d, p, m, st, err);
  return form == 0 ? forward<128, 0>(d, p, m, st, err) : form == 1 ? forward<128, 1>(d, p, m, st, err) : forward<128, 2>(d, p, m, st, err);
}

int attn_masked_tc_bwd(const mslt_attention_desc& d, float* delta, int* next, int* status, cudaStream_t st, char* err) {
  TcParams p = params_of(d, status, attn_take_starve());
  MapVal mq[4], mk[4];
  const int loop_k = d.head_dim <= 64 ? BwdShape<64, true>::LOOP : BwdShape<128, true>::LOOP;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
    snprintf(err, 256, "attention_masked: no CUDA device");
    return MSLT_ERR_CUDA;
  }
  TcParams pk = p;
  int rc = map_of(d.q, d, d.heads, AM_ROWS, &mq[0], p.a_perm, err);
  if (!rc) rc = map_of(d.k, d, d.kv_heads, BwdShape<64, false>::LOOP, &mq[1], p.b_perm, err);
  if (!rc) rc = map_of(d.dctx, d, d.heads, AM_ROWS, &mq[2], p.c_perm, err);
  if (!rc) rc = map_of(d.v, d, d.kv_heads, BwdShape<64, false>::LOOP, &mq[3], p.d_perm, err);
  if (!rc) rc = map_of(d.k, d, d.kv_heads, AM_ROWS, &mk[0], pk.a_perm, err);
  if (!rc) rc = map_of(d.q, d, d.heads, loop_k, &mk[1], pk.b_perm, err);
  if (!rc) rc = map_of(d.v, d, d.kv_heads, AM_ROWS, &mk[2], pk.c_perm, err);
  if (!rc) rc = map_of(d.dctx, d, d.heads, loop_k, &mk[3], pk.d_perm, err);
  if (rc) return rc;
  int log_lanes = 0;
  while ((8 << log_lanes) < d.head_dim) log_lanes++;
  const long long rows = (long long)d.B * d.S * d.heads;
  launch_pdl(masked_delta_tc, (unsigned)(((rows << log_lanes) + 255) / 256), 256, 0, st, view_of(d.dctx), view_of(d.ctx), (const bf16*)d.rest,
             delta, next, d.S, d.heads, d.head_dim, log_lanes, rows);
  p.delta = pk.delta = delta;
  p.next = next;
  pk.next = next + 1;
  p.o0 = view_of(d.dq);
  p.wide = aligned32(d.dq);
  pk.o0 = view_of(d.dk);
  pk.o1 = view_of(d.dv);
  pk.wide = aligned32(d.dk) && aligned32(d.dv);
  rc = backward_of<false>(d, p, mq, sms, st, err);
  if (!rc) rc = backward_of<true>(d, pk, mk, sms, st, err);
  return rc;
}

}  // namespace mslt
