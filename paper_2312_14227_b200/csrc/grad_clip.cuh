// Global gradient norm over many tensors, clipping, and the masked update on clipped gradients.
//   n = sqrt( sum over all selected tensors of g^2 ),   k = max_norm / n where n > max_norm, else 1
// The squares are formed and added in 64 bits (fp32 squares leave fp32's range both ways: 1e20, 1e-25), in an order
// that depends on the tensors' sizes and the grid alone.  The tensors of a launch are named by a table in the
// kernel's parameters, so nothing is copied to the device and a captured graph replays it as it is.
// Both passes are bound by DRAM; the sum comes before the first product, so gradients beyond L2 are read twice.  Measured: 80 M
// elements clipped 153 us (the squares 51 us, 95 % of the copy bandwidth); Adam on fp32 masters of 101 M elements 555 us (94 %
// of it moved, the second read of the gradients included).
#pragma once

#include "kernels.cuh"

namespace et {

constexpr int kClipThreads = 256;
constexpr int kClipVec = 16;                                // elements per thread and block of work
constexpr int kClipBlock = kClipThreads * kClipVec;         // elements of one block of work
constexpr int kClipBlocksPerSm = 8;

struct ClipEntry {
  const float* g;
  float* out;                // clipped copy (clip) -- or the optimiser's operands (update):
  void* W;
  float* master;
  float* m_state;
  float* v_state;
  unsigned long long count;
  long long block_begin;     // first block of work of this tensor in the launch
};
template <int N>
struct ClipTable {
  long long blocks;          // blocks of work of the launch
  int n;
  ClipEntry e[N];
};

template <int N>
__device__ __forceinline__ int clip_find(const ClipTable<N>& t, long long vb) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {                                         // last entry with block_begin <= vb
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].block_begin <= vb) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// 64-bit block sum, fixed order; result valid in thread 0.
__device__ __forceinline__ double block_sum64(double v) {
  __shared__ double part[32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  double r = 0.0;
  if (threadIdx.x == 0)
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) r += part[w];
  return r;
}

// Four elements, of which `left` exist.  `once`: they will not be read again soon, L2 may let go of them first.
__device__ __forceinline__ void clip_load(const float* p, int left, bool once, float (&v)[4]) {
  if (left == 4 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    const float4* q = reinterpret_cast<const float4*>(p);
    const float4 x = once ? __ldcs(q) : *q;
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
  } else {
    load_seg<4>(p, left, v);
  }
}
// The end of the gradients that the second pass, which walks backwards, still finds in L2 (126 MB, of which the outputs take
// a share): blocks of work that the first pass reads for keeps.  80 million elements: 164 us without the hints, 156 us keeping
// 40 MB, 153 us keeping 64, 154 us keeping 112.
constexpr long long kClipKeep = (64ll << 20) / (kClipBlock * 4);

template <int N>
__global__ void __launch_bounds__(kClipThreads)
sumsq_kernel(const __grid_constant__ ClipTable<N> tab, double* __restrict__ parts) {
  chain_begin();
  double acc = 0.0;
  for (long long vb = blockIdx.x; vb < tab.blocks; vb += gridDim.x) {
    const ClipEntry& e = tab.e[clip_find(tab, vb)];
    const size_t i0 = (size_t)(vb - e.block_begin) * kClipBlock;
    const float* g = e.g;
    float v[kClipVec / 4][4];
#pragma unroll
    for (int q = 0; q < kClipVec / 4; ++q) {
      const size_t i = i0 + ((size_t)q * kClipThreads + threadIdx.x) * 4;
      const long long left = (long long)e.count - (long long)i;
      clip_load(g + i, left < 0 ? 0 : (int)min(left, 4ll), vb < tab.blocks - kClipKeep, v[q]);
    }
#pragma unroll
    for (int q = 0; q < kClipVec / 4; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc = fma((double)v[q][i], (double)v[q][i], acc);
  }
  acc = block_sum64(acc);
  if (threadIdx.x == 0) parts[blockIdx.x] = acc;
}

// Every block sums the partials itself, in the same order.  A clipped gradient is g * pre * factor: pre is 1, but 2^-126 where
// the factor itself is below fp32's normal numbers (a norm of 1e35 clipped to 1e-4; its product with a gradient is an ordinary number
// all the same).  A norm that is not finite gives finite = 0 and factor 0.
struct ClipFactor {
  float norm, factor, pre, reported;
  int finite;
};
__device__ __forceinline__ ClipFactor norm_and_factor(const double* __restrict__ parts, int n, float max_norm) {
  __shared__ ClipFactor sh;
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += blockDim.x) s += parts[i];
  s = block_sum64(s);
  if (threadIdx.x == 0) {
    const double norm = sqrt(s);
    const bool finite = norm <= 1.7976931348623157e308;     // false for NaN too
    const double f = !finite ? 0.0 : norm > (double)max_norm ? (double)max_norm / norm : 1.0;
    const bool small = finite && f < 0x1p-126;
    sh.norm = (float)norm;
    sh.factor = (float)(small ? f * 0x1p126 : f);
    sh.pre = small ? 0x1p-126f : 1.0f;
    sh.reported = finite ? fmaxf((float)f, 0x1p-149f) : 0.0f;            // 0 says that the norm was not finite
    sh.finite = finite;
  }
  __syncthreads();
  return sh;
}
static __global__ void __launch_bounds__(kClipThreads)
norm_finalize_kernel(const double* __restrict__ parts, int n, float max_norm, float* __restrict__ out) {
  chain_begin();
  const ClipFactor c = norm_and_factor(parts, n, max_norm);
  if (threadIdx.x == 0) { out[0] = c.norm; out[1] = c.reported; }
}

template <int N>
__global__ void __launch_bounds__(kClipThreads)
clip_kernel(const __grid_constant__ ClipTable<N> tab, const double* __restrict__ parts, int n_parts, float max_norm,
            float* __restrict__ norm_out) {
  chain_begin();
  const ClipFactor c = norm_and_factor(parts, n_parts, max_norm);
  const float f = c.factor, pre = c.pre;
  if (norm_out != nullptr && blockIdx.x == 0 && threadIdx.x == 0) { norm_out[0] = c.norm; norm_out[1] = c.reported; }
  for (long long vb = tab.blocks - 1 - blockIdx.x; vb >= 0; vb -= gridDim.x) {   // backwards: the end is still in L2
    const ClipEntry& e = tab.e[clip_find(tab, vb)];
    if (f == 1.0f && e.out == e.g) continue;                // in place and nothing to clip: nothing changes
    const size_t i0 = (size_t)(vb - e.block_begin) * kClipBlock;
    float v[kClipVec / 4][4];
    int left[kClipVec / 4];
#pragma unroll
    for (int q = 0; q < kClipVec / 4; ++q) {
      const size_t i = i0 + ((size_t)q * kClipThreads + threadIdx.x) * 4;
      const long long l = (long long)e.count - (long long)i;
      left[q] = l < 0 ? 0 : (int)min(l, 4ll);
      if (c.finite) clip_load(e.g + i, left[q], true, v[q]);
    }
#pragma unroll
    for (int q = 0; q < kClipVec / 4; ++q) {
      const size_t i = i0 + ((size_t)q * kClipThreads + threadIdx.x) * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[q][j] = c.finite ? v[q][j] * pre * f : 0.0f;
      if (left[q] == 4 && (reinterpret_cast<uintptr_t>(e.out + i) & 15) == 0)
        __stcs(reinterpret_cast<float4*>(e.out + i), make_float4(v[q][0], v[q][1], v[q][2], v[q][3]));
      else
        store_seg<4>(e.out + i, left[q], v[q]);
    }
  }
}

// The optimiser step of et_update_masked on g * factor, every tensor in one launch.  A norm that is not finite leaves
// weights and optimiser state as they are.
template <typename T, int N>
__global__ void __launch_bounds__(kClipThreads)
update_clipped_kernel(const __grid_constant__ ClipTable<N> tab, const double* __restrict__ parts, int n_parts, float max_norm,
                      float* __restrict__ norm_out, const OptParams opt) {
  chain_begin();
  const ClipFactor c = norm_and_factor(parts, n_parts, max_norm);
  const float f = c.factor, pre = c.pre;
  if (norm_out != nullptr && blockIdx.x == 0 && threadIdx.x == 0) { norm_out[0] = c.norm; norm_out[1] = c.reported; }
  if (!c.finite) return;
  for (long long vb = tab.blocks - 1 - blockIdx.x; vb >= 0; vb -= gridDim.x) {   // backwards: the end is still in L2
    const ClipEntry& e = tab.e[clip_find(tab, vb)];
#pragma unroll
    for (int q = 0; q < kClipVec / 8; ++q) {
      const size_t i0 = (size_t)(vb - e.block_begin) * kClipBlock + ((size_t)q * kClipThreads + threadIdx.x) * 8;
      if (i0 >= e.count) continue;
      const int n = (int)min((size_t)8, (size_t)e.count - i0);
      float g[8], w[8];
      load_seg<8>(e.g + i0, n, g);
      if (e.master != nullptr) load_seg<8>(e.master + i0, n, w);
      else load_seg<8>((const T*)e.W + i0, n, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = g[i] * pre * f;
      opt_update_seg(w, g, opt, e.m_state, e.v_state, i0, n);
      if (e.master != nullptr) store_seg<8>(e.master + i0, n, w);
      store_seg<8>((T*)e.W + i0, n, w);
    }
  }
}

}  // namespace et
