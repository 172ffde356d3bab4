// Softmax attention over packed sequences as a member of the stack (ET_LAYER_MASKED_ATTENTION).  Rows are
// [q of `heads` | k of `kv` | v of `kv`] blocks of `dim` columns; query head h reads key / value head h / (heads / kv).
//
//   s_ij = c tanh(scale q_i.k_j / c) - slope |i - j|      (no cap: scale q_i.k_j;  no bias: slope 0)
//   o_i  = sum_j p_ij v_j,  p_ij = exp(s_ij - lse_i),      j in [lo_i, hi_i)
//   D_i  = dO_i . o_i ;  ds_ij = p_ij (dO_i . v_j - D_i) (1 - tanh^2)
//   dq_i = scale sum_j ds_ij k_j ;  dk_j = scale sum_i ds_ij q_i ;  dv_j = sum_i p_ij dO_i
//
// Every mask that the layer knows (sequence bounds, causal, prefix) leaves a row ONE interval of keys, and a key one interval of
// rows: a thread owns a row (or key), keeps the two ends of its interval, and a tile is walked only where some interval meets it.
// A row of no sequence has an empty interval: its output and gradient are 0.  Rows of no sequence may hold anything, NaN
// included: they are overwritten with 0 in the tiles that a product reads as weights' other factor (0 * NaN is NaN).
//
// Forward: a block owns 256 (or 128) query rows of one head, two halves of 128.  Scores of a half against 128 keys
// (tcgen05, operands by TMA) lie in tensor memory, one accumulator row a thread; the thread takes the running maximum, writes
// exp(s - m) as bf16 over the scores, and P v reads P from tensor memory.  While one half's scores are worked on the tensor core
// serves the other half.  The output is rescaled only where a row's maximum has grown by more than 2^8: until then sums and
// output are relative to the older maximum, which fp32 holds as well.
// Backward: two passes of one kernel, dq (block = 128 query rows, keys stream by) and dk, dv (block = 128 keys of a key head, the
// rows of its group's heads stream by).  Both form S = X1 Y1^T and dP = X2 Y2^T against 128 streamed rows in tensor memory,
// write P and dS as bf16 over them, and accumulate dS Y1 (and P Y2) with P and dS read from tensor memory.  Nothing is added with
// atomics: a shared head's gradient is the sum that one block forms in order, or the blocks of a cluster, joined in their order.  The price is that S and dP are formed
// twice, 7 products where 5 would do.
//
// Rounding: P and dS are bf16 (half a step 2^-8 of each term); scores, maxima, sums, D and all accumulators are fp32.  For rows
// of fewer than 64 keys D is taken from the output as it was before its rounding, what that left being kept as a second bf16: the fewer the
// keys the larger the output beside v, and with the rounded output's D the error of dq and dk on 5 rows was 1.6 times that of their own
// rounding, so it is 1.4 times, as on long sequences.  (Kept for every row it cost the forward pass 5 %.  64: the same roundings in numpy on random
// rows of width 64 give dq an error larger by 20 % on 3 keys, 15 % on 5, 7 % on 16, 3 % on 32, 2 % on 64 and 1 % on 128 and 256 without it.)
#pragma once

#include "attn.cuh"
#include "seq_attn.h"

namespace et {
namespace seqattn {

using namespace et::tc;

constexpr uint32_t kTimeoutSeqAttn = 8;
constexpr int kRestKeys = 64;                   // rows of fewer keys keep what the rounding of their output left
constexpr int THREADS = 320;                    // warps 0-3, 4-7: row threads; warp 8: MMA issue, TMEM; warp 9: TMA
// The forward pass starts two idle warps more, a whole third warpgroup: it launches with 384 x 168 registers, the third group goes down to 40
// each and the row threads, which hold 128 scores, up to 232 (256 x 232 + 128 x 40 = 384 x 168).  At 168 they spilled: 472 -> 424 us with a cap, 314 -> 287 with
// a distance bias, 256 -> 252 without (16 heads of 128, 8192 causal rows).  The backward pass does not spill and gained nothing.
constexpr int FWD_THREADS = 384, FWD_REGS = 168, ROW_REGS = 232, REST_REGS = 40;
static_assert(256 * ROW_REGS + 128 * REST_REGS <= FWD_THREADS * FWD_REGS, "the row threads would wait for registers for ever");
constexpr uint32_t CHUNK = 16384;               // 128 rows x 64 columns of bf16
constexpr float LOG2E = 1.4426950408889634f;

// ---- intervals ---------------------------------------------------------------------------------
// Largest q with begin[q] <= row, -1 if there is none; the whole warp asks for one row, 32 probes at a time.  Ends for any contents.
__device__ __forceinline__ int find_seq(const int32_t* begin, int n, int row, int lane) {
  int lo = -1, hi = n + 1;
  while (hi - lo > 1) {
    const int step = (hi - lo - 1 + 31) / 32;
    const int at = lo + 1 + lane * step;
    const bool le = at < hi && begin[at] <= row;
    const unsigned ones = __ballot_sync(0xffffffffu, le);
    const int k = ones == 0xffffffffu ? 32 : __ffs(~ones) - 1;         // leading run of probes that are <= row
    if (k == 0) hi = lo + 1;
    else {
      const int base = lo + 1;
      lo = base + (k - 1) * step;
      if (k < 32) hi = min(hi, base + k * step);
    }
  }
  return lo;
}
// Interval of row `row` (lane's own; the warp's rows are consecutive, lane 0 first): its keys, or with KEYS the rows that see key `row`.
template <bool KEYS>
__device__ __forceinline__ int2 interval(const Mask& m, int row, int lane) {
  int b, e, q = 0;
  if (m.begin == nullptr) {
    if (row >= m.M) return make_int2(0, 0);
    b = row / m.len * m.len;
    e = min(b + m.len, m.M);
  } else {
    int lo = find_seq(m.begin, m.n, row - lane, lane);                 // of the warp's first row, and mostly of all its rows
    if (lo >= m.n || m.begin[lo + 1] <= row - lane + 31) {
      int hi = find_seq(m.begin, m.n, row - lane + 31, lane);
      while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (m.begin[mid] <= row) lo = mid; else hi = mid - 1;
      }
    }
    q = lo;
    if (q < 0 || q >= m.n || row >= m.M) return make_int2(0, 0);
    b = min(max(m.begin[q], 0), m.M);
    e = min(max(m.begin[q + 1], 0), m.M);
  }
  if (m.causal) {
    const int pre = m.prefix != nullptr ? min(max(m.prefix[q], 0), max(e - b, 0)) : 0;
    if (KEYS) { if (row - b >= pre) b = row; }
    else e = min(e, max(row + 1, b + pre));
  }
  return e > b ? make_int2(b, e) : make_int2(0, 0);
}
// Rows outside [x, y) are of no sequence.  (Rows from M on need no care: they arrive as 0.)
__device__ __forceinline__ int2 used_rows(const Mask& m) {
  if (m.begin == nullptr) return make_int2(0, 0x7fffffff);
  const int e = min(max(m.begin[m.n], 0), m.M);
  return make_int2(min(max(m.begin[0], 0), m.M), e == m.M ? 0x7fffffff : e);
}

// ---- tensor memory -----------------------------------------------------------------------------
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(db), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void group_sync(int id) { asm volatile("bar.sync %0, 128;" ::"r"(id) : "memory"); }
// The warp that issues products runs its loop as a whole on values that the compiler can see to be the same in every lane, and one
// elected lane issues: descriptors then stay in uniform registers.  (Issued from a branch of lane 0 a product cost 50 to 60 cycles of that lane's time,
// whatever its size, and the issuing warp was what bounded both passes.)  In the forward pass the warp also comes together after each such
// block: 244 -> 220 us for 16 heads of 128 over 8192 causal rows, 408 -> 370 for 16 of 64 without a mask.
__device__ __forceinline__ bool elect() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(ROW_REGS)); }
__device__ __forceinline__ void leave_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REST_REGS)); }
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* status) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, status, kTimeoutSeqAttn));
}

// Descriptors of a tile's first step; a step moves the address field (16-byte units) by a constant, so that a product costs the issuing
// thread little more than the instruction itself (its instructions, not the tensor core, bounded the first version).
// K-major, pieces of 64 columns `CHUNK_B` bytes apart: 16 columns = 32 bytes along the swizzled row.  MN-major: 16 rows = 2048 bytes.
__device__ __forceinline__ uint64_t k_desc(uint32_t tile) { return make_desc(tile, 16, 1024); }
__device__ __forceinline__ uint64_t mn_desc(uint32_t tile, uint32_t chunk) { return make_desc(tile, chunk, 1024); }
template <uint32_t CHUNK_B> __device__ __forceinline__ constexpr uint64_t k_step(int ks) { return ((ks >> 2) * CHUNK_B + (ks & 3) * 32u) >> 4; }
__device__ __forceinline__ constexpr uint64_t mn_step(int ks) { return (uint64_t)ks * (2048u >> 4); }
// D = A B^T over K columns, both K-major
template <int K, uint32_t CHUNK_A, uint32_t CHUNK_B>
__device__ __forceinline__ void product_ss(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc) {
  tc_mma(d, da, db, idesc, 0u);
#pragma unroll
  for (int ks = 1; ks < K / UK; ++ks) tc_mma(d, da + k_step<CHUNK_A>(ks), db + k_step<CHUNK_B>(ks), idesc, 1u);
}

// Pairs of fp32 values in one instruction
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpair(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t both(float a) { return pair(a, a); }
__device__ __forceinline__ float max_nan(float a, float b) {                   // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// 2^x of two values on the FMA pipes.  The exponential unit takes 8 cycles for a warp's 32 values, twice what the tensor core takes
// for the products that these values belong to; part of them is formed here instead.  x = n + f with n whole, |f| <= 1/2 (adding and
// taking off 1.5 2^23 rounds); 2^f by a polynomial of degree 4 with value 1 at 0, fitted here to the least largest relative error (2.9e-6,
// 1/1400 of the bf16 step that follows); n goes into the exponent.  x below -127 gives 0, as -127 does exactly; NaN is not kept.
__device__ __forceinline__ float2 ex2_pair(uint64_t x2) {
  const float2 v = unpair(x2);
  const uint64_t x = pair(fmaxf(v.x, -127.0f), fmaxf(v.y, -127.0f));
  const uint64_t t = add2(x, both(12582912.0f));
  const uint64_t f = fma2(add2(t, both(-12582912.0f)), both(-1.0f), x);
  uint64_t p = fma2(f, both(0.009582852944731712f), both(0.055906426161527634f));
  p = fma2(p, f, both(0.24024099111557007f));
  p = fma2(p, f, both(0.6931241750717163f));
  p = fma2(p, f, both(1.0f));
  const float2 q = unpair(p), n = unpair(t);
  return make_float2(__uint_as_float(__float_as_uint(q.x) + (__float_as_uint(n.x) << 23)),
                     __uint_as_float(__float_as_uint(q.y) + (__float_as_uint(n.y) << 23)));
}
// Pairs k of every eight with bit k of SHARE set take that way.  Measured over 8192 causal rows and 16 heads: one of eight in the forward pass (222 ->
// 213 us at head width 64, 257 -> 254 at 128), three in the backward pass (579 -> 537, 846 -> 840); more gives the time back in instructions.
constexpr int kFwdShare = 0x01, kBwdShare = 0x29;
template <int SHARE>
__device__ __forceinline__ float2 ex2_of(uint64_t x, int k) {
  if ((SHARE >> (k & 7)) & 1) return ex2_pair(x);
  const float2 v = unpair(x);
  return make_float2(attn::ex2(v.x), attn::ex2(v.y));
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
  return r;
}
__device__ __forceinline__ float ld_peer(uint32_t addr, uint32_t cta) {       // the same place in another block's shared memory
  float v;
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}" : "=f"(v) : "r"(addr), "r"(cta));
  return v;
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}

// tanh with an error relative to it of at most 2^-20, of roundings, for the smallest x, too (2^-21 seen, 2^-23 in the mean): the cap multiplies it, so
// that 1 - 2 / (1 + e^2x), whose error is absolute, would lose scores far below the cap.  NaN stays.
// On |x| <= 1, two values: x (1 + x^2 p(x^2)), p of degree 5 fitted here to the least largest relative error (2^-24.1).
__device__ __forceinline__ uint64_t tanh_small(uint64_t x) {
  const uint64_t y = mul2(x, x);
  uint64_t p = fma2(y, both(0.0010582641698420048f), both(-0.0062593379989266396f));
  p = fma2(p, y, both(0.020359758287668228f));
  p = fma2(p, y, both(-0.053498707711696625f));
  p = fma2(p, y, both(0.13326409459114075f));
  p = fma2(p, y, both(-0.33332985639572144f));
  return mul2(x, fma2(p, y, both(1.0f)));
}
// Any x, four values: x P(x^2) / Q(x^2), P and Q of degree 4 fitted in the same way on |x| <= 9 (2^-25.5), where x is held; the four quotients from
// one reciprocal of the Qs' product (at most 1e11), so that a NaN is one for all four.  A warp takes this form where one of its 32 keys' scores is
// beyond the cap.  8192 causal rows, 16 heads of 128, forward: 391 us where none is, 546 where most are.
__device__ __forceinline__ uint64_t held(uint64_t x) {
  const float2 v = unpair(x);
  return pair(max_nan(min_nan(v.x, 9.0f), -9.0f), max_nan(min_nan(v.y, 9.0f), -9.0f));
}
__device__ __forceinline__ void tanh4(uint64_t x01, uint64_t x23, uint64_t* t01, uint64_t* t23) {
  auto top = [](uint64_t y) {
    uint64_t p = fma2(y, both(1.3354624961436912e-08f), both(2.0609053535736166e-05f));
    p = fma2(p, y, both(0.0034955863375216722f));
    p = fma2(p, y, both(0.13381023705005646f));
    return fma2(p, y, both(1.0f));
  };
  auto below = [](uint64_t y) {
    uint64_t q = fma2(y, both(7.776542929605057e-07f), both(0.0003285632119514048f));
    q = fma2(q, y, both(0.025876974686980247f));
    q = fma2(q, y, both(0.46714338660240173f));
    return fma2(q, y, both(1.0f));
  };
  const uint64_t a = held(x01), b = held(x23), ya = mul2(a, a), yb = mul2(b, b), qa = below(ya), qb = below(yb);
  const float2 p = unpair(mul2(qa, qb));
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(p.x * p.y));
  const uint64_t q = pair(r * p.y, r * p.x);
  *t01 = mul2(mul2(a, top(ya)), mul2(q, qb));
  *t23 = mul2(mul2(b, top(yb)), mul2(q, qa));
}
// Scores of 32 keys in powers of 2, in place of the products s.  SLOPES: 1 - tanh^2 to `slope`.
// Off the diagonal (LINEAR) the distance |row - key| is linear in the key: bias = ss (j - d0), d0 = row - first key, ss = +-slope.
// To every score `own` and, with EACH, each(j) of its pair is added (the backward pass: less the log-sum-exp).
template <bool CAP, bool BIAS, bool SLOPES, bool LINEAR, bool EACH, typename F>
__device__ __forceinline__ void scores(float (&s)[32], float (&slope)[SLOPES ? 32 : 1], float c2, float u, float top, float ss, int d0,
                                       float own, F&& each) {
  const uint64_t ss2 = both(ss), base = both(LINEAR && BIAS ? fmaf(-ss, (float)d0, own) : own);
  auto all = [&](auto small) {
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
      uint64_t a = pair(s[j], s[j + 1]), b = pair(s[j + 2], s[j + 3]);
      if (CAP) {
        a = mul2(a, both(u));
        b = mul2(b, both(u));
        if (decltype(small)::value) {
          a = tanh_small(a);
          b = tanh_small(b);
        } else {
          tanh4(a, b, &a, &b);
        }
        if (SLOPES) {
          const float2 x = unpair(fma2(mul2(a, both(-1.0f)), a, both(1.0f))), y = unpair(fma2(mul2(b, both(-1.0f)), b, both(1.0f)));
          slope[j] = x.x; slope[j + 1] = x.y; slope[j + 2] = y.x; slope[j + 3] = y.y;
        }
      }
      const uint64_t f = both(CAP ? top : c2);
      uint64_t ra = base, rb = base;
      if constexpr (EACH) {
        ra = LINEAR && BIAS ? add2(base, each(j)) : each(j);
        rb = LINEAR && BIAS ? add2(base, each(j + 2)) : each(j + 2);
      }
      if (BIAS && LINEAR) {
        ra = fma2(ss2, pair((float)j, (float)(j + 1)), ra);
        rb = fma2(ss2, pair((float)(j + 2), (float)(j + 3)), rb);
      }
      a = fma2(a, f, ra);
      b = fma2(b, f, rb);
      if (BIAS && !LINEAR) {
        const float2 x = unpair(a), y = unpair(b);
        const float d = (float)(d0 - j);
        a = pair(fmaf(-ss, fabsf(d), x.x), fmaf(-ss, fabsf(d - 1.0f), x.y));
        b = pair(fmaf(-ss, fabsf(d - 2.0f), y.x), fmaf(-ss, fabsf(d - 3.0f), y.y));
      }
      const float2 x = unpair(a), y = unpair(b);
      s[j] = x.x; s[j + 1] = x.y; s[j + 2] = y.x; s[j + 3] = y.y;
    }
  };
  if (!CAP) {
    all(std::false_type());
    return;
  }
  float most = max_nan(fabsf(s[0]), fabsf(s[1]));
#pragma unroll
  for (int j = 2; j < 32; j += 2) most = max3_nan(most, fabsf(s[j]), fabsf(s[j + 1]));
  if (__all_sync(0xffffffffu, most * u <= 1.0f)) all(std::true_type());     // no score of the warp's beyond the cap
  else all(std::false_type());
}

// Rows of a 128-byte-swizzled tile that belong to no sequence become 0 (whole warp; the caller orders it before the products).
__device__ __forceinline__ void scrub(uint8_t* tile, int rows, int chunks, uint32_t chunk, int row0, int2 used, int lane) {
  for (int r = 0; r < rows; ++r) {
    if (row0 + r >= used.x && row0 + r < used.y) continue;
    for (int c = 0; c < chunks; ++c) *reinterpret_cast<uint32_t*>(tile + c * chunk + r * 128 + lane * 4) = 0;
  }
}

// Extent of the union of a warp's intervals: {first, last} over the non-empty ones, {large, 0} without any.
__device__ __forceinline__ void note_extent(int* at, int2 iv) {
  const int l = __reduce_min_sync(0xffffffffu, iv.y > iv.x ? iv.x : 0x7fffffff);
  const int h = __reduce_max_sync(0xffffffffu, iv.y > iv.x ? iv.y : 0);
  if ((threadIdx.x & 31) == 0) { at[0] = l; at[1] = h; }
}
__device__ __forceinline__ int2 extent_of(const int* at) {            // of four warps
  return make_int2(uniform(min(min(at[0], at[2]), min(at[4], at[6]))), uniform(max(max(at[1], at[3]), max(at[5], at[7]))));
}

// ---- forward -----------------------------------------------------------------------------------
template <int DHP>
struct FwdCfg {
  static constexpr int CH = DHP / 64;                            // 64-column pieces of a tile
  static constexpr uint32_t TILE = CH * CHUNK;
  static constexpr int ST = DHP == 128 ? 4 : 6;                  // key and value tiles in flight
  static constexpr uint32_t SMEM = (2 + ST) * TILE + 1024 + 256;
};

// P of a tile's first 96 keys is handed over by itself, so that its product runs under the exponentials of the last 32.
template <int DHP, bool CAP, bool BIAS>
__global__ void __launch_bounds__(FWD_THREADS, 1)
forward_kernel(const __grid_constant__ CUtensorMap map_qkv, const __grid_constant__ CUtensorMap map_out, const Args a) {
  using C = FwdCfg<DHP>;
  constexpr int ST = C::ST;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t ring = base + 2 * C::TILE, bars = base + (2 + ST) * C::TILE;
  const uint32_t bar_q = bars;
  auto bar_s = [&](int h) { return bars + 8u + 8u * h; };         // scores of half h complete (and every product before)
  auto bar_p = [&](int h, int k) { return bars + 24u + 16u * h + 8u * k; };    // P of half h, keys 0-95 and 96-127, in tensor memory
  auto full = [&](int s) { return bars + 56u + 8u * s; };
  auto empty = [&](int s) { return bars + 56u + 8u * (ST + s); };
  int* shared = reinterpret_cast<int*>(gen + (2 + ST) * C::TILE + 160);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(shared);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  int* extent = shared + 2;                                       // lo, hi of each row warp

  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int tiles = (a.mask.M + 128 * a.halves - 1) / (128 * a.halves);
  const int h = blockIdx.x % a.heads;
  // causal rows see the more keys the later they come: the longest blocks start first
  const int tile = a.mask.causal ? tiles - 1 - (int)(blockIdx.x / a.heads) : (int)(blockIdx.x / a.heads);
  const int row0 = tile * 128 * a.halves;
  const int kvh = h / (a.heads / a.kv);

  // (A block's start is a chain of latencies, a third of a block of four tiles: barriers, Q's copy, tensor memory and intervals go side by side.)
  chain_begin();
  if (warp == 9 && lane == 0) {
    mbar_init(bar_q, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_s(i), 1);
      for (int k = 0; k < 2; ++k) mbar_init(bar_p(i, k), 4);
    }
    for (int s = 0; s < ST; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    *abort_flag = 0;
    fence_async_smem();
    mbar_expect_tx(bar_q, (uint32_t)a.halves * C::TILE);
    for (int hf = 0; hf < a.halves; ++hf)
      for (int c = 0; c < C::CH; ++c) tma_load_3d(base + hf * C::TILE + c * CHUNK, &map_qkv, bar_q, c * 64, h, row0 + hf * 128);
    prefetch_tmap(&map_out);
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)tmem_slot)), "r"(TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const int my_half = warp >> 2, trow = threadIdx.x & 127, row = row0 + my_half * 128 + trow;
  int2 iv = make_int2(0, 0);
  if (warp < 8) {
    if (my_half < a.halves) iv = interval<false>(a.mask, row, lane);
    note_extent(extent + 2 * warp, iv);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)uniform((int)*tmem_slot);
  // tiles of 128 keys that each half walks; the stream covers both
  int first[2], last[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int2 e = extent_of(extent + 8 * i);
    first[i] = e.y > e.x ? e.x / 128 : 0;
    last[i] = e.y > e.x ? (e.y + 127) / 128 : 0;
  }
  const bool any0 = last[0] > first[0], any1 = last[1] > first[1];
  const int T0 = any0 && any1 ? min(first[0], first[1]) : any0 ? first[0] : first[1];
  const int T1 = max(last[0], last[1]);
  const int n_tiles = max(T1 - T0, 0);

  if (warp >= 8) {
    leave_registers();
    if (warp == 9) {
      if (lane == 0) {
        bool ok = true;
        int fills = 0;
        for (int i = 0; i < 2 * n_tiles && ok; ++i) {               // K and V of the first tile, of the second, ...
          const int s = i % ST;
          ok = mbar_wait(empty(s), ((uint32_t)(i / ST) & 1u) ^ 1u, abort_flag, a.status, kTimeoutSeqAttn);
          if (!ok) break;
          mbar_expect_tx(full(s), C::TILE);
          const int block = a.heads + (i & 1 ? a.kv : 0) + kvh;
          for (int c = 0; c < C::CH; ++c) tma_load_3d(ring + s * C::TILE + c * CHUNK, &map_qkv, full(s), c * 64, block, (T0 + (i >> 1)) * 128);
          ++fills;
        }
        if (!ok) {                                                  // let the copies in flight land before shared memory goes away
          for (int i = max(0, fills - ST); i < fills; ++i)
            for (uint32_t it = 0; it < (1u << 20) && !mbar_try_wait(full(i % ST), (uint32_t)(i / ST) & 1u); ++it) {}
        }
        // Q must have landed, too, whoever waits for it
        for (uint32_t it = 0; it < (1u << 20) && !mbar_try_wait(bar_q, 0); ++it) {}
      }
    } else if (warp == 8) {
      const uint32_t id_s = attn::idesc128(128, false, false), id_o = attn::idesc128(DHP, false, true);
      const uint64_t dq0 = k_desc(base), dk0 = k_desc(ring), dv0 = mn_desc(ring, CHUNK);
      const int2 used = used_rows(a.mask);
      bool ok = n_tiles == 0 || warp_wait(bar_q, 0, abort_flag, a.status);
      uint32_t np[2] = {0, 0};                                      // tiles of each half whose P v has been issued
      int ik = 0;                                                   // stream position of K of tile t + 1; V of tile t is the one before
      for (int t = T0 - 1; t < T1 && n_tiles > 0 && ok; ++t, ik += 2) {
        const int sk = ik % ST, sv = ik == 0 ? 0 : (ik - 1) % ST;
        const bool has_k = t + 1 < T1, has_v = t >= T0;
        if (has_v) {
          ok = warp_wait(full(sv), (uint32_t)((ik - 1) / ST) & 1u, abort_flag, a.status);
          if (!ok) break;
          if (t * 128 < used.x || (t + 1) * 128 > used.y) {
            scrub(gen + (2 + sv) * C::TILE, 128, C::CH, CHUNK, t * 128, used, lane);
            fence_async_smem();
            __syncwarp();
          }
        }
        if (has_k) ok = warp_wait(full(sk), (uint32_t)(ik / ST) & 1u, abort_flag, a.status);
        if (!ok) break;
        if (CAP && has_k && ((t + 1) * 128 < used.x || (t + 2) * 128 > used.y)) {     // four keys share a reciprocal: NaN would reach the others
          scrub(gen + (2 + sk) * C::TILE, 128, C::CH, CHUNK, (t + 1) * 128, used, lane);
          fence_async_smem();
          __syncwarp();
        }
  #pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const bool pv = t >= first[hf] && t < last[hf], nx = t + 1 >= first[hf] && t + 1 < last[hf];
          if (!ok || (!pv && !nx)) continue;
          const uint32_t S = tmem + hf * 128, O = tmem + 256 + hf * DHP;
          const uint64_t dv = dv0 + (uint32_t)sv * (C::TILE >> 4), dk = dk0 + (uint32_t)sk * (C::TILE >> 4);
          const uint32_t add = np[hf] > 0 ? 1u : 0u;
          if (pv) {
            ok = warp_wait(bar_p(hf, 0), np[hf] & 1u, abort_flag, a.status);
            if (!ok) continue;
            tc_fence_after();
            if (elect()) {
              mma_ts(O, S, dv, id_o, add);
  #pragma unroll
              for (int ks = 1; ks < 6; ++ks) mma_ts(O, S + ks * 8, dv + mn_step(ks), id_o, 1u);
            }
            __syncwarp();
            ok = warp_wait(bar_p(hf, 1), np[hf] & 1u, abort_flag, a.status);
            if (!ok) continue;
            tc_fence_after();
            ++np[hf];
          }
          if (elect()) {
            if (pv) {
  #pragma unroll
              for (int ks = 6; ks < 8; ++ks) mma_ts(O, S + ks * 8, dv + mn_step(ks), id_o, 1u);
            }
            if (nx) product_ss<DHP, CHUNK, CHUNK>(S, dq0 + (uint32_t)hf * (C::TILE >> 4), dk, id_s);
            tc_commit(bar_s(hf));                                   // next scores, or after the last tile the output
          }
          __syncwarp();
        }
        if (ok && elect()) {
          if (has_k) tc_commit(empty(sk));
          if (has_v) tc_commit(empty(sv));
        }
        __syncwarp();
      }
      __syncwarp();
    }
  } else if (my_half < a.halves) {
    take_registers();
    const int hf = my_half;
    const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t S = tmem + lane_addr + hf * 128, O = tmem + lane_addr + 256 + hf * DHP;
    const float c2 = a.scale * LOG2E;
    const float slope2 = BIAS ? a.slopes[h] * LOG2E : 0.0f;
    float m = -INFINITY;
    uint64_t sum2 = 0;
    bool ok = true;
    const int n_own = last[hf] - first[hf];
    for (int i = 0; i < n_own && ok; ++i) {
      ok = warp_wait(bar_s(hf), (uint32_t)i & 1u, abort_flag, a.status);
      if (!ok) break;
      tc_fence_after();
      const int k0 = (first[hf] + i) * 128;
      float v[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32_issue(S + c * 32, v[c]);
      tmem_ld_wait(v[0], v[1]);
      tmem_ld_wait(v[2], v[3]);
      if (CAP || BIAS) {
        const float u = CAP ? a.scale / a.cap : 0.0f, top = a.cap * LOG2E;
        const int d0 = row - k0;
        const bool above = __all_sync(0xffffffffu, d0 >= 127), below = __all_sync(0xffffffffu, d0 <= 0);
        float none[1];
        if (!BIAS || above || below) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            scores<CAP, BIAS, false, true, false>(v[c], none, c2, u, top, above ? slope2 : -slope2, d0 - c * 32, 0.0f, 0);
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c) scores<CAP, BIAS, false, false, false>(v[c], none, c2, u, top, slope2, d0 - c * 32, 0.0f, 0);
        }
      }
      if (!__all_sync(0xffffffffu, iv.x <= k0 && iv.y >= k0 + 128)) {
        const int lo = iv.x - k0;
        const unsigned len = (unsigned)(iv.y - iv.x);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if ((unsigned)(c * 32 + j - lo) >= len) v[c][j] = -INFINITY;
      }
      float mx[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        mx[c] = max_nan(v[c][0], v[c][1]);
#pragma unroll
        for (int j = 2; j < 32; j += 2) mx[c] = max3_nan(mx[c], v[c][j], v[c][j + 1]);
      }
      float top = max_nan(max_nan(mx[0], mx[1]), max_nan(mx[2], mx[3]));
      if (!(CAP || BIAS)) top *= c2;                              // scale > 0: the largest score stays the largest
      if (__any_sync(0xffffffffu, !(top <= m + 8.0f))) {           // (NaN counts as grown, too, and stays)
        const float m_new = max_nan(m, top);
        const float f = m == -INFINITY ? 0.0f : attn::ex2(m - m_new);
        sum2 = mul2(sum2, both(f));
        m = m_new;
        if (i > 0) {                                              // the output so far is complete: bar_s follows it
#pragma unroll 1
          for (int c = 0; c < DHP; c += 32) {
            float o[32];
            tmem_ld32(O + c, o);
            uint32_t r[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(o[j] * f);
            tmem_st32(O + c, r);
          }
        }
      }
      const float mm = m == -INFINITY ? 0.0f : m;
      const uint64_t neg_m = both(-mm), factor = both(c2);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t r[16];
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
          const uint64_t x = pair(v[c][j], v[c][j + 1]);
          const float2 e = ex2_of<kFwdShare>(CAP || BIAS ? add2(x, neg_m) : fma2(x, factor, neg_m), j / 2);
          sum2 = add2(sum2, pair(e.x, e.y));
          r[j / 2] = pack_bf16x2(e.x, e.y);
        }
        tmem_st16(S + c * 16, r);
        if (c >= 2) {
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_p(hf, c - 2));
        }
      }
    }
    if (ok && n_own > 0) ok = warp_wait(bar_s(hf), (uint32_t)n_own & 1u, abort_flag, a.status);
    if (ok) ok = warp_wait(bar_q, 0, abort_flag, a.status);       // Q's tile takes the output
    if (ok) {
      tc_fence_after();
      const float2 halves = unpair(sum2);
      const float sum = halves.x + halves.y;
      // (+inf scores have no softmax)
      const float inv = !(m < INFINITY) ? NAN : sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
      uint8_t* out = gen + hf * C::TILE;
#pragma unroll 1
      for (int c = 0; c < DHP / 32; ++c) {
        float o[32];
        if (n_own > 0) tmem_ld32(O + c * 32, o);
#pragma unroll
        for (int j = 0; j < 32; ++j) o[j] = n_own > 0 ? o[j] * inv : 0.0f;
        sts_row32(out + (c >> 1) * CHUNK, trow, c & 1, o);
        if (row < a.mask.M && iv.y - iv.x < kRestKeys) {
          bf16* rest = (bf16*)a.rest + ((size_t)row * a.heads + h) * a.dim + c * 32;
#pragma unroll
          for (int j = 0; j < 32; j += 8) {
            if (c * 32 + j >= a.dim) break;
            float d[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) d[e] = o[j + e] - __bfloat162float(__float2bfloat16_rn(o[j + e]));
            *reinterpret_cast<uint4*>(rest + j) = make_uint4(pack_bf16x2(d[0], d[1]), pack_bf16x2(d[2], d[3]), pack_bf16x2(d[4], d[5]), pack_bf16x2(d[6], d[7]));
          }
        }
      }
      if (h == 0 && row < a.mask.M) a.keys[row] = iv.y - iv.x;
      if (row < a.mask.M) a.lse[(size_t)h * a.ld + row] = sum > 0.0f || sum != sum ? m + log2f(sum) : INFINITY;
      fence_async_smem();
    }
    group_sync(1 + hf);                                           // a thread whose wait gave up comes here, too
    if (ok && trow == 0) {
      for (int c = 0; c < C::CH; ++c)
        if (c * 64 < a.dim && row < a.mask.M) tma_store_3d(&map_out, base + hf * C::TILE + c * CHUNK, c * 64, h, row);
      tma_store_commit();
      tma_store_wait_all();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
  }
}

// ---- backward ----------------------------------------------------------------------------------
// D_i = dO_i . o_i per head: 16 lanes a row and head, 8 columns a lane.
static __global__ void __launch_bounds__(256)
dot_kernel(const bf16* __restrict__ out, const bf16* __restrict__ rest, const int* __restrict__ keys, const bf16* __restrict__ dout,
           float* __restrict__ D, int M, int heads, int dim, int ld) {
  chain_begin();
  const long long item = ((long long)blockIdx.x * 256 + threadIdx.x) / 16;
  const int sub = threadIdx.x & 15;
  const bool on = item < (long long)M * heads;
  float s = 0.0f;
  if (on && sub * 8 < dim) {
    const size_t at = (size_t)item * dim + sub * 8;               // rows hold the heads side by side: item = row * heads + head
    float o[8], d[8] = {}, g[8];
    load_seg<8>(out + at, 8, o);
    load_seg<8>(dout + at, 8, g);
    if (keys[item / heads] < kRestKeys) load_seg<8>(rest + at, 8, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(o[i] + d[i], g[i], s);
  }
#pragma unroll
  for (int k = 8; k > 0; k >>= 1) s += __shfl_xor_sync(0xffffffffu, s, k);
  if (on && sub == 0) D[(size_t)(item % heads) * ld + item / heads] = s;
}

// The same by one thread, for blocks that are a launch short of time rather than of reads.
struct Dots { const bf16 *out, *dout; };
__device__ __forceinline__ float dot_row(const Dots& t, const Args& a, int row, int h, int n_keys) {
  const size_t at = ((size_t)row * a.heads + h) * a.dim;
  float s = 0.0f;
  for (int c = 0; c < a.dim; c += 8) {
    float o[8], d[8] = {}, g[8];
    load_seg<8>(t.out + at + c, 8, o);
    if (n_keys < kRestKeys) load_seg<8>((const bf16*)a.rest + at + c, 8, d);
    load_seg<8>(t.dout + at + c, 8, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(o[i] + d[i], g[i], s);
  }
  return s;
}

template <int DHP>
struct BwdCfg {
  static constexpr int CH = DHP / 64;
  static constexpr uint32_t TILE = CH * CHUNK;                   // 128 rows, resident or streamed
  static constexpr uint32_t STAGE = 2 * TILE + 1024;             // two tiles, the rows' lse and D
  static constexpr int ST = DHP == 128 ? 2 : 4;
  static constexpr uint32_t SMEM = 2 * TILE + ST * STAGE + 1024 + 256;
};

// DKV = false: X1 = q, X2 = dO (rows of head h), Y1 = k, Y2 = v;  acc1 = dq.
// DKV = true:  X1 = k, X2 = v (keys of a key head), Y1 = q, Y2 = dO of every head of its group;  acc1 = dk, acc2 = dv.
// Tensor memory: acc1, acc2, S (P over it), dP (dS over it).  One product's accumulator is worked on while the tensor core forms the
// others: per tile   P(i) | dK(i-1), dP(i)    then    dS(i) | dV(i), S(i+1).  The first half of P is handed over by itself, so that its share of dV runs
// under the exponentials of the second; where P is not needed as a factor (dq) the next S is formed as soon as this one has been read.
// The products are 128 wide: narrower ones take the tensor core as long (measured 57 to 75 cycles an instruction at 64 and 128 columns).
template <int DHP, bool DKV, bool CAP, bool BIAS>
__global__ void __launch_bounds__(THREADS, 1)
backward_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_g,
                const __grid_constant__ CUtensorMap map_out, bf16* __restrict__ dqkv, const Dots dots, const Args a) {
  using C = BwdCfg<DHP>;
  constexpr int ST = C::ST;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t ring = base + 2 * C::TILE, bars = ring + ST * C::STAGE;
  const uint32_t bar_x = bars, bar_done = bars + 8;
  const uint32_t bar_s = bars + 16, bar_dp = bars + 24;           // S, dP of a tile complete
  const uint32_t bar_p = bars + 32, bar_p2 = bars + 40;           // S read, and half of P in its place (dk, dv); all of it
  const uint32_t bar_ds = bars + 48;                              // dS in dP's place
  auto full = [&](int s) { return bars + 56u + 8u * s; };
  auto empty = [&](int s) { return bars + 56u + 8u * (ST + s); };
  int* shared = reinterpret_cast<int*>(gen + 2 * C::TILE + ST * C::STAGE + 160);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(shared);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  int* extent = shared + 2;

  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int blocks_h = DKV ? a.kv : a.heads, group = a.heads / a.kv;
  const int tiles = (a.mask.M + 127) / 128;
  const int parts = (int)cluster_size(), part = (int)cluster_ctarank();       // blocks of a cluster share an item's tiles
  const int item = blockIdx.x / parts;
  const int h = item % blocks_h;                                  // head, or key head
  const int tile = a.mask.causal && !DKV ? tiles - 1 - item / blocks_h : item / blocks_h;
  const int row0 = tile * 128;

  chain_begin();
  if (warp == 9 && lane == 0) {
    for (int i = 0; i < 4; ++i) mbar_init(bars + 8 * i, 1);
    mbar_init(bar_p, 8);
    mbar_init(bar_p2, 8);
    mbar_init(bar_ds, 8);
    for (int s = 0; s < ST; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    *abort_flag = 0;
    fence_async_smem();
    mbar_expect_tx(bar_x, 2 * C::TILE);
    for (int c = 0; c < C::CH; ++c) {
      tma_load_3d(base + c * CHUNK, &map_x, bar_x, c * 64, DKV ? a.heads + h : h, row0);
      if (DKV) tma_load_3d(base + C::TILE + c * CHUNK, &map_x, bar_x, c * 64, a.heads + a.kv + h, row0);
      else tma_load_3d(base + C::TILE + c * CHUNK, &map_g, bar_x, c * 64, h, row0);
    }
    prefetch_tmap(&map_g);
    prefetch_tmap(&map_out);
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)tmem_slot)), "r"(TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  int2 iv = make_int2(0, 0);
  if (warp < 8) {
    iv = interval<DKV>(a.mask, row0 + (int)(threadIdx.x & 127), lane);
    if (warp < 4) note_extent(extent + 2 * warp, iv);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)uniform((int)*tmem_slot);
  constexpr uint32_t ACC2 = DHP, CS = 256, CDP = 384;
  const int2 e = extent_of(extent);
  const int T0 = e.y > e.x ? e.x / 128 : 0;
  const int n_tiles = e.y > e.x ? (e.y + 127) / 128 - T0 : 0;
  const int all = DKV ? n_tiles * group : n_tiles;
  const int total = (all - part + parts - 1) / parts;             // this block's: every parts-th, from its own number on
  struct Place {                                                  // head of the group and tile of the block's i-th
    int g, t;
    __device__ void settle(int n) { while (t >= n) { t -= n; ++g; } }
  };

  if (warp == 9) {
    if (lane == 0) {
      bool ok = true;
      int fills = 0;
      Place p{0, part};
      for (int i = 0; i < total && ok; ++i, p.t += parts) {
        p.settle(n_tiles);
        const int s = i % ST;
        ok = mbar_wait(empty(s), ((uint32_t)(i / ST) & 1u) ^ 1u, abort_flag, a.status, kTimeoutSeqAttn);
        if (!ok) break;
        const uint32_t dst = ring + s * C::STAGE;
        const int r = (T0 + p.t) * 128, hq = h * group + p.g;
        mbar_expect_tx(full(s), 2 * C::TILE + (DKV ? 1024u : 0u));
        for (int c = 0; c < C::CH; ++c) tma_load_3d(dst + c * CHUNK, &map_x, full(s), c * 64, DKV ? hq : a.heads + h / group, r);
        for (int c = 0; c < C::CH; ++c) {
          if (DKV) tma_load_3d(dst + C::TILE + c * CHUNK, &map_g, full(s), c * 64, hq, r);
          else tma_load_3d(dst + C::TILE + c * CHUNK, &map_x, full(s), c * 64, a.heads + a.kv + h / group, r);
        }
        if (DKV) {
          const size_t at = (size_t)hq * a.ld + r;                // ld is a multiple of 128: whole tiles
          bulk_load(dst + 2 * C::TILE, a.lse + at, 512, full(s));
          bulk_load(dst + 2 * C::TILE + 512, a.D + at, 512, full(s));
        }
        ++fills;
      }
      if (!ok) {
        for (int i = max(0, fills - ST); i < fills; ++i)
          for (uint32_t it = 0; it < (1u << 20) && !mbar_try_wait(full(i % ST), (uint32_t)(i / ST) & 1u); ++it) {}
      }
      for (uint32_t it = 0; it < (1u << 20) && !mbar_try_wait(bar_x, 0); ++it) {}
    }
  } else if (warp == 8) {
    const uint32_t id_s = attn::idesc128(128, false, false), id_a = attn::idesc128(DHP, false, true);
    const uint64_t dx1 = k_desc(base), dx2 = k_desc(base + C::TILE), dy1 = k_desc(ring), dy2 = k_desc(ring + C::TILE),
                   dt1 = mn_desc(ring, CHUNK), dt2 = mn_desc(ring + C::TILE, CHUNK);
    const int2 used = used_rows(a.mask);
    bool ok = true;
    Place p{0, part};
    auto landed = [&](int i) {
      const int s = i % ST;
      if (!warp_wait(full(s), (uint32_t)(i / ST) & 1u, abort_flag, a.status)) return false;
      p.settle(n_tiles);
      const int r = (T0 + p.t) * 128;
      if (r < used.x || r + 128 > used.y) {
        scrub(gen + 2 * C::TILE + s * C::STAGE, 128, 2 * C::CH, CHUNK, r, used, lane);
        fence_async_smem();
        __syncwarp();
      }
      p.t += parts;
      return true;
    };
    auto at = [&](int i) { return (uint64_t)((uint32_t)(i % ST) * (C::STAGE >> 4)); };
    if (total > 0) ok = warp_wait(bar_x, 0, abort_flag, a.status) && landed(0);
    if (total > 0 && ok && elect()) {
      product_ss<DHP, CHUNK, CHUNK>(tmem + CS, dx1, dy1, id_s);
      tc_commit(bar_s);
      product_ss<DHP, CHUNK, CHUNK>(tmem + CDP, dx2, dy2, id_s);
      tc_commit(bar_dp);
    }
    for (int i = 0; i < total && ok; ++i) {
      const bool next = i + 1 < total;
      const uint32_t add = i > 0 ? 1u : 0u;
      const uint64_t b1 = dt1 + at(i), b2 = dt2 + at(i), n1 = dy1 + at(i + 1), n2 = dy2 + at(i + 1);
      if (next) ok = landed(i + 1);
      if (ok) ok = warp_wait(bar_p, (uint32_t)i & 1u, abort_flag, a.status);
      if (!ok) break;
      tc_fence_after();
      if (DKV) {
        // each group's half of P lies in the first half of its scores' columns; steps 0, 1, 4, 5 first, then 2, 3, 6, 7
        auto pv = [&](int ks, uint32_t keep) { mma_ts(tmem + ACC2, tmem + CS + (ks >> 2) * 64 + (ks & 3) * 8, b2 + mn_step(ks), id_a, keep); };
        if (elect()) { pv(0, add); pv(1, 1u); pv(4, 1u); pv(5, 1u); }
        ok = warp_wait(bar_p2, (uint32_t)i & 1u, abort_flag, a.status);
        if (!ok) break;
        tc_fence_after();
        if (elect()) { pv(2, 1u); pv(3, 1u); pv(6, 1u); pv(7, 1u); }
      }
      if (elect()) {
        if (next) {
          product_ss<DHP, CHUNK, CHUNK>(tmem + CS, dx1, n1, id_s);
          tc_commit(bar_s);
        }
      }
      ok = warp_wait(bar_ds, (uint32_t)i & 1u, abort_flag, a.status);
      if (!ok) break;
      tc_fence_after();
      if (elect()) {
        mma_ts(tmem, tmem + CDP, b1, id_a, add);
#pragma unroll
        for (int ks = 1; ks < 8; ++ks) mma_ts(tmem, tmem + CDP + (ks >> 2) * 64 + (ks & 3) * 8, b1 + mn_step(ks), id_a, 1u);
        tc_commit(empty(i % ST));
        if (next) {
          product_ss<DHP, CHUNK, CHUNK>(tmem + CDP, dx2, n2, id_s);
          tc_commit(bar_dp);
        }
      }
    }
    if (ok && total > 0 && elect()) tc_commit(bar_done);
    __syncwarp();
  } else {
    const int w = warp >> 2;
    const int trow = threadIdx.x & 127, row = row0 + trow;
    const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t S = tmem + lane_addr + CS + w * 64, DP = tmem + lane_addr + CDP + w * 64;     // 64 of a tile's 128 columns
    const float c2 = a.scale * LOG2E;
    const float u = CAP ? a.scale / a.cap : 0.0f, top = a.cap * LOG2E;
    float own_lse = INFINITY, own_D = 0.0f, slope2 = 0.0f;
    if (!DKV) {
      if (row < a.mask.M) {
        const size_t at = (size_t)h * a.ld + row;
        own_lse = a.lse[at];
        if (a.dot) {                                              // D_i here, and left for the pass that follows
          own_D = dot_row(dots, a, row, h, iv.y - iv.x);
          if (part == 0 && w == 0) a.D[at] = own_D;
        } else {
          own_D = a.D[at];
        }
      }
      if (BIAS) slope2 = a.slopes[h] * LOG2E;
    }
    const uint64_t c22 = pair(c2, c2), neg_lse2 = pair(-own_lse, -own_lse), neg_D2 = pair(-own_D, -own_D);
    bool ok = true;
    Place pl{0, part};
    for (int i = 0; i < total && ok; ++i, pl.t += parts) {
      pl.settle(n_tiles);
      const int k0 = (T0 + pl.t) * 128 + w * 64;
      if (DKV && BIAS) slope2 = a.slopes[h * group + pl.g] * LOG2E;
      ok = warp_wait(bar_s, (uint32_t)i & 1u, abort_flag, a.status);
      if (!ok) break;
      if (DKV) {                                                  // the rows' lse and D came with the tile
        ok = warp_wait(full(i % ST), (uint32_t)(i / ST) & 1u, abort_flag, a.status);
        if (!ok) break;
      }
      tc_fence_after();
      const float* col = reinterpret_cast<const float*>(gen + 2 * C::TILE + (i % ST) * C::STAGE + 2 * C::TILE) + w * 64;
      const bool whole = __all_sync(0xffffffffu, iv.x <= k0 && iv.y >= k0 + 64);
      const int lo = iv.x - k0;
      const unsigned len = (unsigned)(iv.y - iv.x);
      float s[2][32];                                             // p, in the end p (1 - tanh^2)
      tmem_ld32_issue(S, s[0]);
      tmem_ld32_issue(S + 32, s[1]);
      tmem_ld_wait(s[0], s[1]);
      auto hand_over = [&](uint32_t bar) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
      };
      if (!DKV) hand_over(bar_p);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t r[16];
        if (!CAP && !BIAS) {
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            float4 L4;
            if (DKV) L4 = *reinterpret_cast<const float4*>(col + c * 32 + j);
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              const uint64_t nl = DKV ? (e == 0 ? pair(-L4.x, -L4.y) : pair(-L4.z, -L4.w)) : neg_lse2;
              const float2 x = ex2_of<kBwdShare>(fma2(pair(s[c][j + e], s[c][j + e + 1]), c22, nl), (j + e) / 2);
              s[c][j + e] = x.x;
              s[c][j + e + 1] = x.y;
            }
          }
          if (!whole) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if ((unsigned)(c * 32 + j - lo) >= len) s[c][j] = 0.0f;
          }
          if (DKV) {
#pragma unroll
            for (int j = 0; j < 32; j += 2) r[j / 2] = pack_bf16x2(s[c][j], s[c][j + 1]);
          }
        } else {
          float slope[CAP ? 32 : 1];
          const int d0 = row - k0 - c * 32;
          const bool above = __all_sync(0xffffffffu, d0 >= 31), below = __all_sync(0xffffffffu, d0 <= 0);
          auto less = [&](int j) {
            const float2 L = *reinterpret_cast<const float2*>(col + c * 32 + j);
            return pair(-L.x, -L.y);
          };
          const float own = DKV ? 0.0f : -own_lse;
          if (!BIAS || above || below)
            scores<CAP, BIAS, CAP, true, DKV>(s[c], slope, c2, u, top, above ? slope2 : -slope2, d0, own, less);
          else scores<CAP, BIAS, CAP, false, DKV>(s[c], slope, c2, u, top, slope2, d0, own, less);
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            float2 p = ex2_of<kBwdShare>(pair(s[c][j], s[c][j + 1]), j / 2);
            if (!whole) {
              if ((unsigned)(c * 32 + j - lo) >= len) p.x = 0.0f;
              if ((unsigned)(c * 32 + j + 1 - lo) >= len) p.y = 0.0f;
            }
            if (DKV) r[j / 2] = pack_bf16x2(p.x, p.y);
            s[c][j] = CAP ? p.x * slope[j] : p.x;
            s[c][j + 1] = CAP ? p.y * slope[j + 1] : p.y;
          }
        }
        if (DKV) {
          tmem_st16(S + c * 16, r);
          tmem_st_wait();
          hand_over(c == 0 ? bar_p : bar_p2);
        }
      }
      ok = warp_wait(bar_dp, (uint32_t)i & 1u, abort_flag, a.status);
      if (!ok) break;
      tc_fence_after();
      float dp[2][32];
      tmem_ld32_issue(DP, dp[0]);
      tmem_ld32_issue(DP + 32, dp[1]);
      tmem_ld_wait(dp[0], dp[1]);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t r[16];
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          float4 D4;
          if (DKV) D4 = *reinterpret_cast<const float4*>(col + 128 + c * 32 + j);
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const uint64_t nd = DKV ? (e == 0 ? pair(-D4.x, -D4.y) : pair(-D4.z, -D4.w)) : neg_D2;
            const float2 d = unpair(mul2(pair(s[c][j + e], s[c][j + e + 1]), add2(pair(dp[c][j + e], dp[c][j + e + 1]), nd)));
            dp[c][j + e] = d.x;
            dp[c][j + e + 1] = d.y;
          }
        }
        if (!whole) {                                             // 0 times whatever stands in a masked place
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if ((unsigned)(c * 32 + j - lo) >= len) dp[c][j] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 32; j += 2) r[j / 2] = pack_bf16x2(dp[c][j], dp[c][j + 1]);
        tmem_st16(DP + c * 16, r);
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_ds);
    }
    if (ok && total > 0) ok = warp_wait(bar_done, 0, abort_flag, a.status);
    if (ok) ok = warp_wait(bar_x, 0, abort_flag, a.status);
    // dk and dq are staged in X1's tile, dv in X2's.  dk, dv: a group each; dq: the groups share its 64-column pieces
    const bool second = DKV && w == 1;
    const int c0 = DKV ? 0 : w, c1 = DKV ? C::CH : min(w + 1, C::CH);
    if (ok) {
      tc_fence_after();
      if (parts == 1) {
        const float f = second ? 1.0f : a.scale;
        uint8_t* out = gen + (second ? C::TILE : 0);
#pragma unroll 1
        for (int c = c0 * 2; c < c1 * 2; ++c) {
          float o[32];
          if (total > 0) tmem_ld32(tmem + lane_addr + (second ? DHP : 0) + c * 32, o);
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = total > 0 ? o[j] * f : 0.0f;
          sts_row32(out + (c >> 1) * CHUNK, trow, c & 1, o);
        }
        fence_async_smem();
      } else {
        // each block leaves its sums in its own shared memory, [accumulator][column][row]; every tile has been read by now
        float* mine = reinterpret_cast<float*>(gen) + (second ? DHP * 128 : 0) + trow;
        const int g0 = DKV ? 0 : w * (DHP / 64), g1 = DKV ? DHP / 32 : (w + 1) * (DHP / 64);
#pragma unroll 1
        for (int c = g0; c < g1; ++c) {
          float o[32];
          if (total > 0) tmem_ld32(tmem + lane_addr + (second ? DHP : 0) + c * 32, o);
#pragma unroll
          for (int j = 0; j < 32; ++j) mine[(c * 32 + j) * 128] = total > 0 ? o[j] : 0.0f;
        }
      }
    }
    if (parts == 1) {
      group_sync(1 + w);                                          // a thread whose wait gave up comes here, too
      if (ok && trow == 0) {
        const int block = DKV ? a.heads + (w == 1 ? a.kv : 0) + h : h;
        for (int c = c0; c < c1; ++c)
          if (c * 64 < a.dim) tma_store_3d(&map_out, base + (second ? C::TILE : 0) + c * CHUNK, c * 64, block, row0);
        tma_store_commit();
        tma_store_wait_all();
      }
    }
  }
  if (parts > 1) {                                                // join: a block adds up its share of the columns, in the blocks' order
    cluster_sync_all();
    if (warp < 8) {
      const int w = warp >> 2, trow = threadIdx.x & 127, row = row0 + trow;
      const bool second = DKV && w == 1;
      const int n = DKV ? DHP / parts : DHP / parts / 2;            // columns a thread: at least 4
      const int first = part * (DHP / parts) + (DKV ? 0 : w * n);
      const uint32_t at = base + ((second ? DHP * 128 : 0) + first * 128 + trow) * 4;
      const float f = second ? 1.0f : a.scale;
      const int block = DKV ? a.heads + (second ? a.kv : 0) + h : h;
      bf16* out = dqkv + ((size_t)row * (a.heads + 2 * a.kv) + block) * a.dim + first;
      for (int j = 0; j < n && first + j < a.dim; j += 4) {
        float o[4] = {};
        for (int c = 0; c < parts; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] += ld_peer(at + (j + e) * 512, c);
        if (row < a.mask.M) {
          uint2 q;
          q.x = pack_bf16x2(o[0] * f, o[1] * f);
          q.y = pack_bf16x2(o[2] * f, o[3] * f);
          *reinterpret_cast<uint2*>(out + j) = q;
        }
      }
    }
    cluster_sync_all();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
  }
}

}  // namespace seqattn
}  // namespace et
