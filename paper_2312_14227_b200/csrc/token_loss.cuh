// Losses on token logits: log probabilities of given tokens, the clipped policy loss with a KL term and the
// paired log-ratio (preference) loss, each with the gradient of the logits.
//
// A row i of the stack's output holds the logits of one token, z_ij = scale * y_ij for the columns j < vocab.
//   lp_i   = z_it - log sum_j exp z_ij                           t = the token that was taken
//   d lp_i / d y_ij = scale * ([j = t] - p_ij),   p_ij = exp(z_ij) / sum_j exp z_ij
// so every loss here is "one number c_i = d loss / d lp_i per row", and the gradient is c_i times the line above.
// Sums and the log are fp32 (rows) and 64-bit (over rows); the gradient is rounded once, to the storage type.
#pragma once

#include "common.cuh"

namespace et {
namespace tok {

__device__ __forceinline__ float exp2_fast(float x) {      // ex2.approx: 2 ulp, 0 for -inf and underflow
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Two fp32 values in one 64-bit register: one instruction for both (add / mul / fma .f32x2).
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
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
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

enum Mode { kScore = 0, kPolicy = 1 };

struct Args {
  const void* y;              // [rows x width]
  void* dY;                   // same shape, or null; may be y itself
  const int32_t* targets;
  const float* weights;       // null: default_weight everywhere
  const float* advantages;    // kPolicy
  const float* logp_old;      // kPolicy; null: the current log probability (ratio 1)
  const float* logp_ref;      // kPolicy; null: no KL term
  float* logp;                // lp of each row, 0 where the row is left out; may be null
  float2* stats;              // kScore writes, token_grad_kernel reads: (max of the row's y, 1 / sum exp(scale (y - max))), (0, -1) for a
                              // row that is left out; may be null
  float* coef;                // token_grad_kernel: c_i.  kScore sets it to 0 where it is not null
  const int32_t* begin;       // kScore: null, or [n_begin + 1]: rows outside begin[0] .. begin[n_begin] - 1 are left out
  int32_t n_begin;
  double* parts;              // kPolicy: 3 x n_parts: w * (-surrogate), w * kl, w * [clipped], of a row or of a block's rows; may be null
  int32_t n_parts;
  int32_t finish;             // kPolicy: the block that finishes last adds the parts up (else policy_finish_kernel does)
  uint32_t* done;             // kPolicy: blocks that have finished; 0 between calls
  uint32_t* ticket;           // kPolicy: rows handed out beyond the first two of each cluster; 0 between calls
  float* out;                 // kPolicy with parts: {loss, policy part, kl part, clipped share}
  int32_t rows, width, vocab;
  int32_t slices, per;        // blocks (of one cluster) that share a row, 16-byte vectors of each
  float scale;
  float k_hi, k_lo;           // scale * log2(e) as a sum: k_hi rounded towards 0, k_lo > 0 the rest
  float default_weight;
  float clip_low, clip_high, kl_coef;
};
// exp(scale d) for differences d <= 0, as 2^(d k_hi + (d k_lo + kExpUp)) with one rounding of the exponent.  What errs the same way in
// every term moves the log of every sum the same way, which sums over rows do not average out, so:
//  - one fp32 constant for scale * log2(e) would be off by up to 2^-23 of it.  The small product goes into the fused one: added
//    to a rounded d k_hi it would vanish below half a step of it
//  - ex2.approx is low by 5.0e-8 on average (measured in every octave of [-22, -1], 2^20 arguments each against 64-bit values:
//    -4.96e-8 .. -5.11e-8; -2.88e-8 on [-1, 0]): kExpUp = 5.0e-8 / ln 2 raises the exponent by that.  It is below half a step
//    of the exponents that count, and rounding to nearest carries it on average.  2^kExpUp itself comes out as 1: the largest term
//    of a row is exact
// k_lo > 0 keeps d = -inf at -inf (a negative or zero k_lo would make it NaN).
constexpr float kExpUp = 7.2e-8f;
__device__ __forceinline__ uint64_t scale2(uint64_t d, uint64_t k_hi, uint64_t k_lo) {
  return fma2(d, k_hi, fma2(d, k_lo, pack2(kExpUp, kExpUp)));
}
__device__ __forceinline__ float exp_diff(float d, const Args& a) { return exp2_fast(fmaf(d, a.k_hi, fmaf(d, a.k_lo, kExpUp))); }

// lp of the target's logit from the row's (max, sum), the log in 64 bits (an fp32 log rounds by more than the sum's own error).
__device__ __forceinline__ float log_prob(float yt, float m, float s, const Args& a) {
  return (float)((double)(yt - m) * (double)a.scale - log((double)s));
}

// (max, sum) over the lanes of a warp.  fmaxf drops NaN; the sum carries it.
__device__ __forceinline__ void join_lanes(float& m, float& s, const Args& a) {
  const float own = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (own != -INFINITY) s *= exp_diff(own - m, a);
  s = warp_sum(s);
}
// (max, sum) over a block: all threads get the pair.  A thread without elements holds (-inf, 0).
__device__ __forceinline__ void block_max_sum(float& m, float& s, const Args& a) {
  __shared__ float sm[32], ss[32];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, nw = (blockDim.x + 31) >> 5;
  join_lanes(m, s, a);
  __syncthreads();
  if (lane == 0) { sm[wid] = m; ss[wid] = s; }
  __syncthreads();
  m = lane < nw ? sm[lane] : -INFINITY;
  s = lane < nw ? ss[lane] : 0.0f;
  join_lanes(m, s, a);
}

// d loss / d lp of a row of the policy loss, and its contributions to the reported sums.
//   r = exp(lp - old),  surrogate = min(r A, clip(r, 1 - lo, 1 + hi) A),  kl = exp(d) - 1 - d with d = ref - lp
// The clipped branch is constant in lp; at a tie the unclipped one counts.
struct RowTerms { float adv, old, ref; };
__device__ __forceinline__ RowTerms row_terms(const Args& a, int row) {
  RowTerms r;
  r.adv = a.advantages[row];
  r.old = a.logp_old != nullptr ? a.logp_old[row] : 0.0f;
  r.ref = a.logp_ref != nullptr ? a.logp_ref[row] : 0.0f;
  return r;
}
// `sums`: the contributions are added here (64-bit arithmetic, so one thread's work, not a block's); may be null.
__device__ __forceinline__ float policy_coef(const Args& a, const RowTerms& t, float lp, float w, double* sums) {
  const float r = a.logp_old != nullptr ? expf(lp - t.old) : 1.0f;
  const float rc = fminf(fmaxf(r, 1.0f - a.clip_low), 1.0f + a.clip_high);
  const bool nothing = t.adv == 0.0f && r == INFINITY;       // no advantage: nothing, however far the ratio has gone
  const float first = nothing ? 0.0f : r * t.adv, second = nothing ? 0.0f : rc * t.adv;
  const bool clipped = first > second;
  float slope = clipped ? 0.0f : -first;
  float kl = 0.0f;
  if (a.logp_ref != nullptr) {
    const float d = t.ref - lp, e = expm1f(d);
    kl = e < INFINITY ? e - d : e;                         // d = inf (a token of probability 0): inf, not inf - inf; NaN stays
    if (a.kl_coef != 0.0f) slope -= a.kl_coef * e;         // a divergence that is reported only may be infinite
  }
  if (sums != nullptr) {
    sums[0] -= (double)w * (double)(clipped ? second : first);
    sums[1] += (double)w * (double)kl;
    if (clipped) sums[2] += (double)w;
  }
  return w * slope;
}

// Whether a row takes part.
template <int MODE>
__device__ __forceinline__ bool takes_part(const Args& a, int row, int t, float w) {
  if (MODE == kScore && a.begin != nullptr && (row < a.begin[0] || row >= a.begin[a.n_begin])) return false;
  return w != 0.0f && t >= 0 && t < a.vocab;
}
__device__ __forceinline__ void put_parts(const Args& a, int at, const double (&s)[3]) {
#pragma unroll
  for (int q = 0; q < 3; ++q) a.parts[(size_t)q * a.n_parts + at] = s[q];
}
// The parts added up by one block, in a fixed order; counters back to 0 for the next call.
__device__ __forceinline__ void policy_total(const Args& a) {
  __shared__ double sh[3][32];
  if (a.out != nullptr) {
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      double s = 0.0;
#pragma unroll 4
      for (int i = threadIdx.x; i < a.n_parts; i += blockDim.x) s += __ldcg(a.parts + (size_t)q * a.n_parts + i);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if ((threadIdx.x & 31) == 0) sh[q][threadIdx.x >> 5] = s;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    if (a.out != nullptr) {
      double r[3];
      for (int q = 0; q < 3; ++q) {
        r[q] = 0.0;
        for (int wq = 0; wq < (int)((blockDim.x + 31) >> 5); ++wq) r[q] += sh[q][wq];
      }
      a.out[0] = (float)(a.kl_coef != 0.0f ? r[0] + (double)a.kl_coef * r[1] : r[0]);
      a.out[1] = (float)r[0]; a.out[2] = (float)r[1]; a.out[3] = (float)r[2];
    }
    *a.done = 0u;
    *a.ticket = 0u;
  }
}
static __global__ void __launch_bounds__(1024) policy_finish_kernel(const __grid_constant__ Args a) {
  chain_begin();
  policy_total(a);
}
// The same by the block that finishes last.
__device__ __forceinline__ void policy_finish(const Args& a) {
  if (a.finish == 0) return;
  __shared__ bool last;
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(a.done, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  policy_total(a);
}

// ---- 16-byte vectors of a row ------------------------------------------------------------------
// y's base is 16-byte aligned; a row of fp32 may begin inside a vector.  Vector v of a row covers its elements
// v * N - mis .. + N - 1, mis = elements of the row's first vector that belong to the row before.  Vectors that lie in the row
// whole are moved whole, the others element by element, so that no element of another row is read or written.
template <typename T> struct VecOf;
template <> struct VecOf<float> {
  static constexpr int N = 4;
  static constexpr uint32_t kNegInf = 0xff800000u;
  static __device__ __forceinline__ float max_of(const uint4& q) {
    return fmaxf(fmaxf(__uint_as_float(q.x), __uint_as_float(q.y)), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w)));
  }
  static __device__ __forceinline__ void pairs(const uint4& q, uint64_t (&p)[2]) {
    p[0] = pack2(__uint_as_float(q.x), __uint_as_float(q.y));
    p[1] = pack2(__uint_as_float(q.z), __uint_as_float(q.w));
  }
  static __device__ __forceinline__ uint4 from_pairs(const uint64_t (&p)[2]) {
    float a, b, c, d;
    unpack2(p[0], a, b);
    unpack2(p[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
  }
};
template <> struct VecOf<bf16> {
  static constexpr int N = 8;
  static constexpr uint32_t kNegInf = 0xff80ff80u;
  static __device__ __forceinline__ float max_of(const uint4& q) {
    auto h = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
    const __nv_bfloat162 m = __hmax2(__hmax2(h(q.x), h(q.y)), __hmax2(h(q.z), h(q.w)));
    return fmaxf(__low2float(m), __high2float(m));
  }
  static __device__ __forceinline__ void pairs(const uint4& q, uint64_t (&p)[4]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  static __device__ __forceinline__ uint4 from_pairs(const uint64_t (&p)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      unpack2(p[i], a, b);
      w[i] = pack_bf16x2(a, b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <typename T, int B>
__device__ __forceinline__ float max_of_all(const uint4 (&q)[B]) {
  if constexpr (VecOf<T>::N == 4) {
    float m = VecOf<T>::max_of(q[0]);
#pragma unroll
    for (int i = 1; i < B; ++i) m = fmaxf(m, VecOf<T>::max_of(q[i]));
    return m;
  } else {                                                  // packed pairs first
    auto h = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
    __nv_bfloat162 m = h(q[0].x);
#pragma unroll
    for (int i = 0; i < B; ++i) m = __hmax2(m, __hmax2(__hmax2(h(q[i].x), h(q[i].y)), __hmax2(h(q[i].z), h(q[i].w))));
    return fmaxf(__low2float(m), __high2float(m));
  }
}
// Loads are read once and stores written once: both with the streaming hint.
template <typename T>
__device__ __forceinline__ uint4 load_vec(const T* row, int e0, int vocab) {
  constexpr int N = VecOf<T>::N;
  if (e0 >= 0 && e0 + N <= vocab) return __ldcs(reinterpret_cast<const uint4*>(row + e0));
  uint4 q = make_uint4(VecOf<T>::kNegInf, VecOf<T>::kNegInf, VecOf<T>::kNegInf, VecOf<T>::kNegInf);
  T* h = reinterpret_cast<T*>(&q);
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (e0 + i >= 0 && e0 + i < vocab) h[i] = row[e0 + i];
  return q;
}
template <typename T>
__device__ __forceinline__ void store_vec(T* row, int e0, int width, int vocab, uint4 q) {
  constexpr int N = VecOf<T>::N;
  if (e0 >= 0 && e0 + N <= vocab) {
    __stcs(reinterpret_cast<uint4*>(row + e0), q);
    return;
  }
  const T* h = reinterpret_cast<const T*>(&q);
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (e0 + i >= 0 && e0 + i < width) row[e0 + i] = e0 + i < vocab ? h[i] : from_f32<T>(0.0f);
}
// g p + [j = t] c, p = exp(scale (y - m)) / sum, g = -c / sum, for one vector.
template <typename T>
__device__ __forceinline__ uint4 grad_vec(const uint4& q, float m, float g, float c, int hit /* t - e0 */, const Args& a) {
  constexpr int P = VecOf<T>::N / 2;
  uint64_t p[P];
  VecOf<T>::pairs(q, p);
  const uint64_t nm = pack2(-m, -m), kh = pack2(a.k_hi, a.k_hi), kl = pack2(a.k_lo, a.k_lo), gg = pack2(g, g);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    float x, y;
    unpack2(scale2(add2(p[i], nm), kh, kl), x, y);
    p[i] = mul2(gg, pack2(exp2_fast(x), exp2_fast(y)));
  }
  if (hit >= 0 && hit < VecOf<T>::N) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (hit == 2 * i) p[i] = add2(p[i], pack2(c, 0.0f));
      if (hit == 2 * i + 1) p[i] = add2(p[i], pack2(0.0f, c));
    }
  }
  return VecOf<T>::from_pairs(p);
}

// Sum of the terms of B vectors over the reference `ref` (finite), added to s.
template <typename T, int B>
__device__ __forceinline__ float add_terms(const uint4 (&x)[B], float ref, float s, const Args& a) {
  constexpr int P = VecOf<T>::N / 2;
  const uint64_t nm = pack2(-ref, -ref), kh = pack2(a.k_hi, a.k_hi), kl = pack2(a.k_lo, a.k_lo);
  uint64_t acc[2] = {pack2(s, 0.0f), pack2(0.0f, 0.0f)};
#pragma unroll
  for (int i = 0; i < B; ++i) {
    uint64_t p[P];
    VecOf<T>::pairs(x[i], p);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      float x0, x1;
      unpack2(scale2(add2(p[j], nm), kh, kl), x0, x1);
      acc[j & 1] = add2(acc[j & 1], pack2(exp2_fast(x0), exp2_fast(x1)));
    }
  }
  float s0, s1;
  unpack2(add2(acc[0], acc[1]), s0, s1);
  return s0 + s1;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float ld_cluster(const float* p, int rank) {
  uint32_t local = (uint32_t)__cvta_generic_to_shared(p), remote;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote) : "memory");
  return v;
}

// A block's view of one row's slice.  Vectors [lo, hi) of the slice lie in the row and under `vocab` whole, the one or two
// others are moved element by element.
template <typename T>
struct Slice {
  static constexpr int N = VecOf<T>::N;
  const T* y;                   // the row
  T* dY;
  const uint4* src;             // vector 0 of the slice
  uint4* dst;
  int e0, lo, hi;               // column of vector 0's first element
  __device__ __forceinline__ Slice(const Args& a, long long row, int v0) {
    const size_t base = (size_t)row * a.width;
    const int mis = (int)(base % N);
    y = (const T*)a.y + base;
    dY = (T*)a.dY + base;
    src = reinterpret_cast<const uint4*>(y - mis) + v0;
    dst = reinterpret_cast<uint4*>(dY - mis) + v0;
    e0 = v0 * N - mis;
    lo = e0 < 0 ? 1 : 0;
    hi = max(lo, min(a.per, (a.vocab + mis) / N - v0));
  }
};

__device__ __forceinline__ void st_cluster(int* p, int rank, int v) {
  uint32_t local = (uint32_t)__cvta_generic_to_shared(p), remote;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(rank));
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(remote), "r"(v) : "memory");
}
// Asks L2 for a slice: one instruction, nothing waits for it.
template <typename T>
__device__ __forceinline__ void prefetch_slice(const Slice<T>& sl) {
  if (sl.hi > sl.lo)
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(sl.src + sl.lo), "r"((sl.hi - sl.lo) * 16) : "memory");
}
// What the second pass over a row needs, from the warp that worked it out.
struct RowResult { float m, g, cs, hit; };       // hit: the target's gradient

// One read of the logits, one write of the gradient: a.slices blocks of one cluster share a row, every thread holds up to
// NV vectors of it in registers from the load to the store.  (max, sum) go through shuffles, shared memory and the cluster's
// distributed shared memory; one warp turns them into the row's coefficient.  kScore stops after the log probability.
//
// What bounds it is issue slots and the exponential unit next to DRAM: at 16 bytes in and out, an SM has 177 issue slots per
// vector and thread at full bandwidth, the arithmetic of bf16 rows takes about 100 of them and the exponentials alone take 128
// cycles of their unit.  So range checks are made for THREADS vectors at a time and what is done once per row is done by one warp.
// For kPolicy the blocks are persistent and take long rows by ticket (rows that are left out cost less than others, so a fixed share
// leaves SMs idle at the end: 100 against 93 us; short ones even out, and one counter would not serve them all); a row is known an
// iteration ahead and its slice is asked into L2 by one instruction while the row before is worked on (without: 98 us).
// Measured, of the copy bandwidth (6558 GB/s): 8192 rows of 131072 bf16 columns 718 us at full clocks (84 %) and 760 us in
// seconds-long runs, whose clocks the power limit lowers (80 %); 4096 rows of 32003, 15 % of them left out, 95 us (78 %) and 98 us, the
// same in fp32 174 us (85 %).
constexpr int kTicketThreads = 128;
template <typename T, int MODE, int THREADS, int NV>
__global__ void __launch_bounds__(THREADS, THREADS < 64 ? 32 : (NV <= 4 ? 1536 : 1024) / THREADS)    // 40 or 64 registers a thread
token_held_kernel(const __grid_constant__ Args a) {
  chain_begin();
  constexpr int N = VecOf<T>::N, W = THREADS / 32;
  constexpr bool TICKETS = MODE == kPolicy && THREADS >= kTicketThreads;      // else every block takes each gridDim.x-th row
  __shared__ float warp_m[W], warp_s[W], pair_m[2], pair_s[2];
  __shared__ RowResult result;
  __shared__ int rows_after[2];
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int C = a.slices, rank = blockIdx.x % C, clusters = gridDim.x / C;
  int row = blockIdx.x / C, next = MODE == kPolicy ? row + clusters : a.rows;
  int t_next = 0;
  float w_next = 0.0f;
  auto head = [&](int r) {
    t_next = a.targets[r];
    w_next = a.weights != nullptr ? a.weights[r] : a.default_weight;
  };
  double sums[3] = {0.0, 0.0, 0.0};                          // without tickets: of all the rows of the block
  if (C > 1) {                                               // every block of the cluster runs before one writes another's shared memory
    cluster_arrive();
    cluster_wait();
  }
  if (row < a.rows) head(row);
  for (int it = 0; row < a.rows; ++it) {                     // `row` is the same in all blocks of a cluster
    const int b = it & 1;
    const Slice<T> sl(a, row, rank * a.per);
    const int t = t_next;
    const float w = w_next;
    const bool live = takes_part<MODE>(a, row, t, w);
    uint4 q[NV];
    // every round but the last is full: the same for the whole block, and so for all but slices that begin inside a vector or
    // reach far beyond `vocab`
    const bool regular = sl.lo == 0 && (NV - 1) * THREADS <= sl.hi;
    if (live) {
      if (regular) {
#pragma unroll
        for (int i = 0; i < NV - 1; ++i) q[i] = __ldcs(sl.src + i * THREADS + tid);
      } else {
#pragma unroll
        for (int i = 0; i < NV - 1; ++i) {
          const int v = i * THREADS + tid;
          q[i] = load_vec<T>(sl.y, sl.e0 + v * N, v < a.per ? a.vocab : 0);   // out of the slice or the row: nothing but -inf
        }
      }
      const int v = (NV - 1) * THREADS + tid;
      q[NV - 1] = load_vec<T>(sl.y, sl.e0 + v * N, v < a.per ? a.vocab : 0);
    }
    if (MODE == kPolicy) {
      if (TICKETS && rank == 0 && tid == 0) {         // the row after the next one
        // a counter that something else has written to must not lead out of the rows (they are left undone then)
        const int after = (int)min(2u * (uint32_t)clusters + min(atomicAdd(a.ticket, 1u), (uint32_t)a.rows), (uint32_t)a.rows);
        if (C == 1) rows_after[b] = after;
        else for (int c = 0; c < C; ++c) st_cluster(&rows_after[b], c, after);
      }
      if (next < a.rows) {
        head(next);
        if (tid == THREADS - 1 && takes_part<MODE>(a, next, t_next, w_next)) prefetch_slice(Slice<T>(a, next, rank * a.per));
      }
    }
    float m = -INFINITY, s = 0.0f, yt = 0.0f;
    RowTerms terms{};
    if (live) {
      if (wid == 0) {                                        // what the row's coefficient needs besides the sums
        yt = to_f32(sl.y[t]);
        if (MODE == kPolicy) terms = row_terms(a, row);
      }
      m = max_of_all<T>(q);
      s = add_terms<T>(q, m == -INFINITY ? 0.0f : m, 0.0f, a);
      join_lanes(m, s, a);
      if (lane == 0) { warp_m[wid] = m; warp_s[wid] = s; }
    }
    __syncthreads();
    if (wid == 0) {
      if (live) {
        m = lane < W ? warp_m[lane] : -INFINITY;
        s = lane < W ? warp_s[lane] : 0.0f;
        join_lanes(m, s, a);
      }
      if (C > 1) {
        if (lane == 0) { pair_m[b] = m; pair_s[b] = s; }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        if (live) {
          m = lane < C ? ld_cluster(&pair_m[b], lane) : -INFINITY;
          s = lane < C ? ld_cluster(&pair_s[b], lane) : 0.0f;
          join_lanes(m, s, a);
        }
      }
      const bool first = rank == 0 && lane == 0;
      if (live) {
        const float lp = MODE == kPolicy || first ? log_prob(yt, m, s, a) : 0.0f;
        const float inv = 1.0f / s;
        if (first) {
          if (a.logp != nullptr) a.logp[row] = lp;
          if (MODE == kScore && a.stats != nullptr) a.stats[row] = make_float2(m, inv);
        }
        if (MODE == kPolicy) {
          double one[3] = {0.0, 0.0, 0.0};
          const float cs = policy_coef(a, terms, lp, w, first && a.parts != nullptr ? (TICKETS ? one : sums) : nullptr) * a.scale, g = -cs * inv;
          if (TICKETS && first && a.parts != nullptr) put_parts(a, row, one);
          if (lane == 0) result = RowResult{m, g, cs, fmaf(g, exp_diff(yt - m, a), cs)};
        }
      } else if (first) {
        if (a.logp != nullptr) a.logp[row] = 0.0f;
        if (MODE == kScore && a.stats != nullptr) a.stats[row] = make_float2(0.0f, -1.0f);
        if (TICKETS && a.parts != nullptr) put_parts(a, row, {0.0, 0.0, 0.0});
      }
      if (MODE == kScore && first && a.coef != nullptr) a.coef[row] = 0.0f;
    } else if (C > 1) {                                      // barriers of the cluster count every thread
      cluster_arrive();
      cluster_wait();
    }
    if (MODE == kScore) break;                               // one row a block
    __syncthreads();
    const int after = TICKETS ? rows_after[b] : next + clusters;
    const RowResult r = result;
    if (a.dY != nullptr && live && r.cs != 0.0f) {           // a clipped row without a KL term has no gradient either
      auto out = [&](const uint4& x) { return grad_vec<T>(x, r.m, r.g, 0.0f, -1, a); };
      auto out_checked = [&](int i) {                        // a vector that is not known to lie in the row
        const int v = i * THREADS + tid, e0 = sl.e0 + v * N;
        if (v < a.per && e0 < a.width) store_vec<T>(sl.dY, e0, a.width, a.vocab, out(q[i]));
      };
      if (regular) {
#pragma unroll
        for (int i = 0; i < NV - 1; ++i) __stcs(sl.dst + i * THREADS + tid, out(q[i]));
        if ((NV - 1) * THREADS + tid < sl.hi) __stcs(sl.dst + (NV - 1) * THREADS + tid, out(q[NV - 1]));
        else out_checked(NV - 1);
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) out_checked(i);
      }
      const int tv = (t - sl.e0) >> (N == 8 ? 3 : 2);        // the target's element, by the thread that wrote its vector
      if (tv >= 0 && tv < a.per && tv % THREADS == tid) sl.dY[t] = from_f32<T>(r.hit);
    } else if (a.dY != nullptr) {
      const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
      for (int v = tid; v < a.per; v += THREADS) {
        if (v >= sl.lo && v < sl.hi) __stcs(sl.dst + v, zero);
        else store_vec<T>(sl.dY, sl.e0 + v * N, a.width, a.width, zero);
      }
    }
    row = next;
    next = after;
  }
  if (MODE == kPolicy && !TICKETS && a.parts != nullptr && rank == 0 && tid == 0) put_parts(a, blockIdx.x / C, sums);
  if (C > 1) {                                               // no block leaves while another reads its shared memory
    cluster_arrive();
    cluster_wait();
  }
  if (MODE == kPolicy) policy_finish(a);
}

// One block per row of any length.  kScore: a stream over the logits (2048 rows of 50257 bf16 columns 40 us, 78 % of the copy
// bandwidth, 42 us in seconds-long runs; the exponential unit is 57 % busy).  kPolicy: rows too long to be held are read twice
// ((max, sum) first, the gradient from the second read, which finds much of the row in L2).
constexpr int kRowThreads = 512;
template <typename T, int MODE>
__global__ void __launch_bounds__(kRowThreads)
token_row_kernel(const __grid_constant__ Args a) {
  chain_begin();
  constexpr int N = VecOf<T>::N, B = 4;
  const int row = blockIdx.x, tid = threadIdx.x;
  const Slice<T> sl(a, row, 0);                             // a.per: the vectors of a row
  const int t = a.targets[row];
  const float w = a.weights != nullptr ? a.weights[row] : a.default_weight;
  const bool live = takes_part<MODE>(a, row, t, w);
  float c = 0.0f, m = -INFINITY, inv = 0.0f;
  if (live) {
    // a gradient will read the logits once more: they are not marked as read for the last time
    const bool last_read = MODE == kScore && a.coef == nullptr;
    float s = 0.0f;
    auto batch = [&](const auto& q) {
      const float cm = fmaxf(max_of_all<T>(q), m);
      if (m != -INFINITY) s *= exp_diff(m - cm, a);
      m = cm;
      s = add_terms<T>(q, m == -INFINITY ? 0.0f : m, s, a);
    };
    int v = tid;
    if (v < sl.lo) {
      const uint4 q[1] = {load_vec<T>(sl.y, sl.e0 + v * N, a.vocab)};
      batch(q);
      v += kRowThreads;
    }
    for (; v + (B - 1) * kRowThreads < sl.hi; v += B * kRowThreads) {
      uint4 q[B];
#pragma unroll
      for (int j = 0; j < B; ++j) q[j] = last_read ? __ldcs(sl.src + v + j * kRowThreads) : sl.src[v + j * kRowThreads];
      batch(q);
    }
    for (; v < a.per; v += kRowThreads) {
      const uint4 q[1] = {load_vec<T>(sl.y, sl.e0 + v * N, a.vocab)};
      batch(q);
    }
    block_max_sum(m, s, a);
    const float yt = to_f32(sl.y[t]);
    const float lp = MODE == kPolicy || tid == 0 ? log_prob(yt, m, s, a) : 0.0f;
    inv = 1.0f / s;
    if (MODE == kPolicy) {
      double sums[3] = {0.0, 0.0, 0.0};
      c = policy_coef(a, row_terms(a, row), lp, w, tid == 0 && a.parts != nullptr ? sums : nullptr);
      if (tid == 0 && a.parts != nullptr) put_parts(a, row, sums);
    }
    if (tid == 0) {
      if (a.logp != nullptr) a.logp[row] = lp;
      if (MODE == kScore && a.stats != nullptr) a.stats[row] = make_float2(m, inv);
      if (MODE == kScore && a.coef != nullptr) a.coef[row] = 0.0f;
    }
    if (MODE == kPolicy && a.dY == a.y) __syncthreads();    // y[t] is read before it is overwritten
  } else if (tid == 0) {
    if (a.logp != nullptr) a.logp[row] = 0.0f;
    if (MODE == kScore && a.stats != nullptr) a.stats[row] = make_float2(0.0f, -1.0f);
    if (MODE == kScore && a.coef != nullptr) a.coef[row] = 0.0f;
    if (MODE == kPolicy && a.parts != nullptr) put_parts(a, row, {0.0, 0.0, 0.0});
  }
  if (MODE == kPolicy && a.dY != nullptr) {
    const float cs = c * a.scale, g = -cs * inv;
    for (int v = tid; v < a.per; v += kRowThreads) {
      const int e0 = sl.e0 + v * N;
      if (!live) store_vec<T>(sl.dY, e0, a.width, a.width, make_uint4(0u, 0u, 0u, 0u));
      else store_vec<T>(sl.dY, e0, a.width, a.vocab, grad_vec<T>(load_vec<T>(sl.y, e0, a.vocab), m, g, cs, t - e0, a));
    }
  }
  if (MODE == kPolicy) policy_finish(a);
}

// The gradient from a row's (max, 1 / sum) and c, block (row, slice): nothing but a stream over the logits.  0.82 GB in
// and out of 8192 rows of 32000 bf16 columns in 124 us: at the copy bandwidth.
constexpr int kGradThreads = 256, kGradVecs = 4;
template <typename T>
__global__ void __launch_bounds__(kGradThreads)
token_grad_kernel(const __grid_constant__ Args a) {
  chain_begin();
  constexpr int N = VecOf<T>::N, STEP = kGradThreads;
  const int row = (int)(blockIdx.x / a.slices);
  const Slice<T> sl(a, row, (blockIdx.x % a.slices) * (kGradThreads * kGradVecs));   // a.per: vectors of a slice
  const int tid = threadIdx.x;
  const float c = a.coef[row];
  const float2 st = a.stats[row];
  const int t = a.targets[row];
  const bool regular = sl.lo == 0 && kGradVecs * STEP <= sl.hi;                       // the same for the whole block
  if (c == 0.0f || st.y < 0.0f) {                           // left out, or of no weight: the logits are not read
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < kGradVecs; ++i) {
      const int v = i * STEP + tid;
      if (regular) __stcs(sl.dst + v, zero);
      else if (sl.e0 + v * N < a.width) store_vec<T>(sl.dY, sl.e0 + v * N, a.width, a.width, zero);
    }
    return;
  }
  const float cs = c * a.scale, g = -cs * st.y;
  uint4 q[kGradVecs];
  if (regular) {
#pragma unroll
    for (int i = 0; i < kGradVecs; ++i) q[i] = __ldcs(sl.src + i * STEP + tid);
#pragma unroll
    for (int i = 0; i < kGradVecs; ++i) __stcs(sl.dst + i * STEP + tid, grad_vec<T>(q[i], st.x, g, 0.0f, -1, a));
    const int tv = (t - sl.e0) >> (N == 8 ? 3 : 2);          // the target's vector once more, by the thread that wrote it
    if (t >= sl.e0 && tv < kGradVecs * STEP && tv % STEP == tid) {
      // its words are in a register that a constant index names
#pragma unroll
      for (int i = 0; i < kGradVecs; ++i)
        if (tv / STEP == i) __stcs(sl.dst + tv, grad_vec<T>(q[i], st.x, g, cs, t - (sl.e0 + tv * N), a));
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kGradVecs; ++i) q[i] = load_vec<T>(sl.y, sl.e0 + (i * STEP + tid) * N, a.vocab);
#pragma unroll
  for (int i = 0; i < kGradVecs; ++i) {
    const int e0 = sl.e0 + (i * STEP + tid) * N;
    if (e0 < a.width) store_vec<T>(sl.dY, e0, a.width, a.vocab, grad_vec<T>(q[i], st.x, g, cs, t - e0, a));
  }
}

// ---- preference loss -----------------------------------------------------------------------
// Sequence q is the rows [begin[q], begin[q + 1]); sequences 2p and 2p + 1 are the chosen and the rejected answer of
// pair p.  S_q = sum of w_i lp_i;  x = beta ((S_c - ref_c) - (S_r - ref_r)).  Bounds outside [0, rows] are clamped and
// an end before its begin is an empty sequence, so that no value in `begin` reads out of range.
constexpr int kPrefSigmoid = 0, kPrefIpo = 1, kPrefHinge = 2;
struct PairArgs {
  const float* logp;          // 0 where a row is left out
  const float* weights;       // null: 1
  const int32_t* targets;
  const int32_t* begin;       // [2 pairs + 1]
  const float* ref;           // [2 pairs] or null (0)
  float* seq_logp;            // [2 pairs] or null
  double* parts;              // pairs x 4: loss, chosen reward, rejected reward, [chosen > rejected]
  uint32_t* done;             // blocks that have finished; 0 between calls
  float* out;                 // their means, or null
  float* coef;                // [rows] c_i, 0 for the rows of no sequence
  int32_t rows, pairs, vocab, kind;
  float beta, smoothing;
};
__device__ __forceinline__ float pair_weight(const PairArgs& a, int row) {
  const int t = a.targets[row];
  return t >= 0 && t < a.vocab ? (a.weights != nullptr ? a.weights[row] : 1.0f) : 0.0f;
}
// One block per pair, half its threads for each sequence: both sums (64 bits, fixed order), the pair's loss, the rows'
// coefficients.  What takes its time is latency: the loads of four rows a thread go out together, one thread does the loss.
constexpr int kPairThreads = 512, kPairHalf = kPairThreads / 2;
static __global__ void __launch_bounds__(kPairThreads)
pair_kernel(const __grid_constant__ PairArgs a) {
  chain_begin();
  __shared__ double sh[kPairThreads / 32];
  __shared__ double slope_sh;
  const int p = blockIdx.x, side = threadIdx.x / kPairHalf, at = threadIdx.x % kPairHalf;
  const int b = min(max(a.begin[2 * p + side], 0), a.rows);
  const int e = max(b, min(max(a.begin[2 * p + side + 1], 0), a.rows));
  double s = 0.0;
  for (int i = b + at; i < e; i += 4 * kPairHalf) {
    float w[4], lp[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = i + k * kPairHalf;
      w[k] = r < e ? pair_weight(a, r) : 0.0f;
      lp[k] = r < e ? a.logp[r] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (w[k] != 0.0f) s += (double)w[k] * (double)lp[k];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double total[2] = {0.0, 0.0};
#pragma unroll
    for (int k = 0; k < kPairThreads / 32; ++k) total[k / (kPairHalf / 32)] += sh[k];
    const double beta = a.beta, eps = a.smoothing;
    const double rc = beta * (total[0] - (a.ref != nullptr ? (double)a.ref[2 * p] : 0.0));
    const double rr = beta * (total[1] - (a.ref != nullptr ? (double)a.ref[2 * p + 1] : 0.0));
    const double x = rc - rr;
    double loss, dx;
    if (a.kind == kPrefSigmoid) {
      // t = exp(-|x|): log(1 + exp(+-x)) = max(0, +-x) + log(1 + t), sigmoid(-|x|) = t / (1 + t)
      const double t = exp(-fabs(x)), l = log1p(t), small = t / (1.0 + t), large = 1.0 / (1.0 + t);
      loss = l + (1.0 - eps) * fmax(-x, 0.0);
      if (eps > 0.0) loss += eps * fmax(x, 0.0);           // x = inf (a rejected token of probability 0) times no smoothing is nothing
      dx = eps * (x < 0.0 ? small : large) - (1.0 - eps) * (x < 0.0 ? large : small);
      if (x != x) loss = dx = x;
    } else if (a.kind == kPrefIpo) {
      const double h = x / beta - 0.5 / beta;
      loss = h * h;
      dx = 2.0 * h / beta;
    } else {
      loss = fmax(0.0, 1.0 - x);
      dx = x < 1.0 ? -1.0 : 0.0;
      if (x != x) loss = dx = x;
    }
    slope_sh = dx * beta / (double)a.pairs;
    if (a.seq_logp != nullptr) { a.seq_logp[2 * p] = (float)total[0]; a.seq_logp[2 * p + 1] = (float)total[1]; }
    double* out = a.parts + (size_t)p * 4;
    out[0] = loss; out[1] = rc; out[2] = rr; out[3] = x > 0.0 ? 1.0 : 0.0;
  }
  __syncthreads();
  const double slope = side == 0 ? slope_sh : -slope_sh;
#pragma unroll 4
  for (int i = b + at; i < e; i += kPairHalf) a.coef[i] = (float)((double)pair_weight(a, i) * slope);
  if (a.out == nullptr) return;
  // the block that finishes last adds the pairs up, in a fixed order
  __shared__ bool last;
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(a.done, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last || threadIdx.x >= 32) return;
  __threadfence();
  double mean[4] = {0.0, 0.0, 0.0, 0.0};
  for (int i = threadIdx.x; i < a.pairs; i += 32)
#pragma unroll
    for (int q = 0; q < 4; ++q) mean[q] += __ldcg(a.parts + (size_t)i * 4 + q);
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mean[q] += __shfl_xor_sync(0xffffffffu, mean[q], o);
  if (threadIdx.x == 0) {
    for (int q = 0; q < 4; ++q) a.out[q] = (float)(mean[q] / (double)a.pairs);
    *a.done = 0u;
  }
}

}  // namespace tok
}  // namespace et
