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

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {      // ex2.approx: 2 ulp, 0 for -inf and underflow
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

enum Mode { kScore = 0, kPolicy = 1, kGrad = 2 };

struct Args {
  const void* y;              // [rows x width]
  void* dY;                   // same shape, or null; may be y itself
  const int32_t* targets;
  const float* weights;       // null: default_weight everywhere
  const float* advantages;    // kPolicy
  const float* logp_old;      // kPolicy; null: the current log probability (ratio 1)
  const float* logp_ref;      // kPolicy; null: no KL term
  float* logp;                // lp of each row, 0 where the row is left out; may be null
  float2* stats;              // kScore writes, kGrad reads: (max of the row's y, 1 / sum exp2((y - max) k))
  const float* coef;          // kGrad: c_i
  double* parts;              // kPolicy: rows x 3: w * (-surrogate), w * kl, w * [clipped]; may be null
  int32_t width, vocab;
  float scale;
  float default_weight;
  float clip_low, clip_high, kl_coef;
};

// (max, sum) of a block's rows: all threads get the pair.  A thread without elements holds (-inf, 0).
__device__ __forceinline__ void block_max_sum(float& m, float& s, float k) {
  __shared__ float sm[32], ss[32];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, nw = (blockDim.x + 31) >> 5;
  float wm = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) wm = fmaxf(wm, __shfl_xor_sync(0xffffffffu, wm, o));
  // fmaxf drops NaN; the sum carries it
  float ws = m == -INFINITY ? s : s * exp2_fast((m - wm) * k);
  ws = warp_sum(ws);
  __syncthreads();
  if (lane == 0) { sm[wid] = wm; ss[wid] = ws; }
  __syncthreads();
  float bm = lane < nw ? sm[lane] : -INFINITY;
  const float own = bm;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) bm = fmaxf(bm, __shfl_xor_sync(0xffffffffu, bm, o));
  float bs = lane < nw ? ss[lane] : 0.0f;
  if (own != -INFINITY) bs *= exp2_fast((own - bm) * k);
  s = warp_sum(bs);
  m = bm;
}

// d loss / d lp of a row of the policy loss, and its contributions to the reported sums.
//   r = exp(lp - old),  surrogate = min(r A, clip(r, 1 - lo, 1 + hi) A),  kl = exp(d) - 1 - d with d = ref - lp
// The clipped branch is constant in lp; at a tie the unclipped one counts.
__device__ __forceinline__ float policy_coef(const Args& a, int row, float lp, float w, double* part) {
  const float adv = a.advantages[row];
  const float r = a.logp_old != nullptr ? expf(lp - a.logp_old[row]) : 1.0f;
  const float rc = fminf(fmaxf(r, 1.0f - a.clip_low), 1.0f + a.clip_high);
  const bool clipped = r * adv > rc * adv;
  float slope = clipped ? 0.0f : -adv * r;
  float kl = 0.0f;
  if (a.logp_ref != nullptr) {
    const float d = a.logp_ref[row] - lp, e = expm1f(d);
    kl = e - d;
    slope -= a.kl_coef * e;
  }
  part[0] = -(double)w * (double)((clipped ? rc : r) * adv);
  part[1] = (double)w * (double)kl;
  part[2] = clipped ? (double)w : 0.0;
  return w * slope;
}

// One block per row, two passes over the row: (max, sum) first, the gradient from a second read.
template <typename T, int MODE>
__global__ void __launch_bounds__(256)
token_row_kernel(const Args a) {
  constexpr int V = 8;
  const int row = blockIdx.x;
  const size_t base = (size_t)row * a.width;
  const T* y = (const T*)a.y + base;
  T* dY = a.dY != nullptr ? (T*)a.dY + base : nullptr;
  const int t = a.targets[row];
  const float w = a.weights != nullptr ? a.weights[row] : a.default_weight;
  const bool live = w != 0.0f && t >= 0 && t < a.vocab && (MODE != kGrad || a.coef[row] != 0.0f);
  const float k = a.scale * kLog2e;
  float c = 0.0f, m = 0.0f, inv = 0.0f;
  if (live) {
    if constexpr (MODE == kGrad) {
      const float2 st = a.stats[row];
      m = st.x; inv = st.y;
      c = a.coef[row];
    } else {
      m = -INFINITY;
      float s = 0.0f;
      for (int j = threadIdx.x * V; j < a.vocab; j += blockDim.x * V) {
        float v[V];
        const int n = min(V, a.vocab - j);
        load_seg<V>(y + j, n, v);
        float cm = m;
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (i < n) cm = fmaxf(cm, v[i]);
        if (cm != m) { s *= m == -INFINITY ? 0.0f : exp2_fast((m - cm) * k); m = cm; }
        const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (i < n) s += exp2_fast((v[i] - ref) * k);
      }
      block_max_sum(m, s, k);
      inv = 1.0f / s;
      const float lp = kLn2 * ((to_f32(y[t]) - m) * k - log2f(s));
      if (MODE == kPolicy) {
        double part[3];
        c = policy_coef(a, row, lp, w, part);
        if (threadIdx.x == 0 && a.parts != nullptr)
          for (int q = 0; q < 3; ++q) a.parts[(size_t)row * 3 + q] = part[q];
      }
      if (threadIdx.x == 0) {
        if (a.logp != nullptr) a.logp[row] = lp;
        if (a.stats != nullptr) a.stats[row] = make_float2(m, inv);
      }
      if (MODE == kPolicy && dY == (T*)y) __syncthreads();     // y[t] is read before it is overwritten
    }
  } else if (threadIdx.x == 0) {
    if (MODE != kGrad && a.logp != nullptr) a.logp[row] = 0.0f;
    if (MODE == kPolicy && a.parts != nullptr)
      for (int q = 0; q < 3; ++q) a.parts[(size_t)row * 3 + q] = 0.0;
  }
  if (MODE == kScore || dY == nullptr) return;
  const float cs = c * a.scale;
  const float g = -cs * inv;
  for (int j = threadIdx.x * V; j < a.width; j += blockDim.x * V) {
    float v[V];
    const int n = min(V, a.width - j);
    if (live) load_seg<V>(y + j, n, v);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float p = exp2_fast((v[i] - m) * k);
      v[i] = live && j + i < a.vocab ? fmaf(g, p, j + i == t ? cs : 0.0f) : 0.0f;
    }
    store_seg<V>(dY + j, n, v);
  }
}

// Sums of the policy loss's row contributions, in a fixed order: out = {loss, policy part, kl part, clipped share}.
static __global__ void __launch_bounds__(1024)
policy_finalize_kernel(const double* __restrict__ parts, int rows, float kl_coef, float* __restrict__ out) {
  __shared__ double sh[3][32];
  double s[3] = {0.0, 0.0, 0.0};
  for (int i = threadIdx.x; i < rows; i += blockDim.x)
#pragma unroll
    for (int q = 0; q < 3; ++q) s[q] += parts[(size_t)i * 3 + q];
#pragma unroll
  for (int q = 0; q < 3; ++q) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s[q] += __shfl_xor_sync(0xffffffffu, s[q], o);
    if ((threadIdx.x & 31) == 0) sh[q][threadIdx.x >> 5] = s[q];
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double r[3];
    for (int q = 0; q < 3; ++q) {
      r[q] = 0.0;
      for (int wq = 0; wq < (int)(blockDim.x >> 5); ++wq) r[q] += sh[q][wq];
    }
    out[0] = (float)(r[0] + (double)kl_coef * r[1]);
    out[1] = (float)r[0]; out[2] = (float)r[1]; out[3] = (float)r[2];
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
  float* coef;                // [rows] c_i
  int32_t rows, pairs, vocab, kind;
  float beta, smoothing;
};
__device__ __forceinline__ float pair_weight(const PairArgs& a, int row) {
  const int t = a.targets[row];
  return t >= 0 && t < a.vocab ? (a.weights != nullptr ? a.weights[row] : 1.0f) : 0.0f;
}
__device__ __forceinline__ double log1pexp(double x) {       // log(1 + exp(x))
  return fmax(x, 0.0) + log1p(exp(-fabs(x)));
}
// One block per pair: both sums (64 bits, fixed order), the pair's loss, the rows' coefficients.
static __global__ void __launch_bounds__(256)
pair_kernel(const PairArgs a) {
  __shared__ double sh[8];
  __shared__ double total[2];
  const int p = blockIdx.x;
  int b[2], e[2];
  for (int q = 0; q < 2; ++q) {
    b[q] = min(max(a.begin[2 * p + q], 0), a.rows);
    e[q] = max(b[q], min(max(a.begin[2 * p + q + 1], 0), a.rows));
    double s = 0.0;
    for (int i = b[q] + (int)threadIdx.x; i < e[q]; i += blockDim.x) {
      const float w = pair_weight(a, i);
      if (w != 0.0f) s += (double)w * (double)a.logp[i];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
      double r = 0.0;
      for (int wq = 0; wq < (int)(blockDim.x >> 5); ++wq) r += sh[wq];
      total[q] = r;
    }
    __syncthreads();
  }
  const double beta = a.beta, eps = a.smoothing;
  const double rc = beta * (total[0] - (a.ref != nullptr ? (double)a.ref[2 * p] : 0.0));
  const double rr = beta * (total[1] - (a.ref != nullptr ? (double)a.ref[2 * p + 1] : 0.0));
  const double x = rc - rr;
  double loss, dx;
  if (a.kind == kPrefSigmoid) {
    loss = (1.0 - eps) * log1pexp(-x) + eps * log1pexp(x);
    dx = eps / (1.0 + exp(-x)) - (1.0 - eps) / (1.0 + exp(x));
  } else if (a.kind == kPrefIpo) {
    const double h = x / beta - 0.5 / beta;
    loss = h * h;
    dx = 2.0 * h / beta;
  } else {
    loss = fmax(0.0, 1.0 - x);
    if (x != x) loss = x;
    dx = x < 1.0 ? -1.0 : (x != x ? x : 0.0);
  }
  const double slope = dx * beta / (double)a.pairs;
  if (threadIdx.x == 0) {
    if (a.seq_logp != nullptr) { a.seq_logp[2 * p] = (float)total[0]; a.seq_logp[2 * p + 1] = (float)total[1]; }
    double* out = a.parts + (size_t)p * 4;
    out[0] = loss; out[1] = rc; out[2] = rr; out[3] = x > 0.0 ? 1.0 : 0.0;
  }
  for (int q = 0; q < 2; ++q)
    for (int i = b[q] + (int)threadIdx.x; i < e[q]; i += blockDim.x)
      a.coef[i] = (float)((double)pair_weight(a, i) * (q == 0 ? slope : -slope));
}
// Means over the pairs, in a fixed order: out = {loss, chosen reward, rejected reward, share chosen > rejected}.
static __global__ void __launch_bounds__(32)
pair_finalize_kernel(const double* __restrict__ parts, int pairs, float* __restrict__ out) {
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  for (int i = threadIdx.x; i < pairs; i += 32)
    for (int q = 0; q < 4; ++q) s[q] += parts[(size_t)i * 4 + q];
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s[q] += __shfl_xor_sync(0xffffffffu, s[q], o);
  if (threadIdx.x == 0)
    for (int q = 0; q < 4; ++q) out[q] = (float)(s[q] / (double)pairs);
}

}  // namespace tok
}  // namespace et
