// fp32 GEMM on the ordinary FMA pipes, used by fp32 stacks (tensor cores would need TF32,
// whose 10-bit mantissa cannot hold a 1e-4 bound).  One kernel covers forward, dgrad and
// wgrad through element strides:
//   C[i, j] = sum_seg sum_kk  A[i*sa_i + kk*sa_k] * B[kk*sb_k + seg*sb_seg + (j mod b_wrap)*sb_j]
#pragma once

#include "common.cuh"
#include "epilogue.cuh"

namespace et {
namespace simt {

constexpr int TK = 16, THREADS = 256;

struct Params {
  int rows, cols;       // output extent
  int kc;               // contraction length per segment
  int segs;             // fold segments
  long long sa_i, sa_k;
  long long sb_k, sb_seg, sb_j;
  int b_wrap;           // 0 = off
};

// Tiles of TILE x TILE outputs, R x R a thread.  STAGES tiles of TK contraction elements are on their way into shared memory (cp.async) while one
// is worked on, and neighbouring threads load along whichever dimension is contiguous in memory.  Small stacks are bound by the
// latency of these loads: 100 x 136 from 688 took 42 us with a load, a barrier and the products in turn, 34 us with one tile ahead, 19 us so.
// Every output is summed in the order of the contraction whatever the tile, so that the choice of tile changes no bit.
template <class Epi, int TILE>
__global__ void __launch_bounds__(THREADS)
gemm_simt_kernel(const float* __restrict__ A, const float* __restrict__ B, const Params p, const Epi epi) {
  constexpr int R = TILE / 16, LOADS = TILE * TK / THREADS, STAGES = 4;
  __shared__ __align__(16) float As[STAGES][TK][TILE + 4];
  __shared__ __align__(16) float Bs[STAGES][TK][TILE + 4];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;   // 16 x 16 threads, R x R outputs each
  const int i0 = row_block() * TILE, j0 = blockIdx.x * TILE;
  const bool a_along_k = p.sa_k == 1, b_along_k = p.sb_k == 1;
  float acc[R][R];
#pragma unroll
  for (int a = 0; a < R; ++a)
#pragma unroll
    for (int b = 0; b < R; ++b) acc[a][b] = 0.0f;

  auto copy = [](uint32_t dst, const float* src, bool there) {      // 4 bytes, or 0 where there is nothing (src is then not read)
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
  };
  // this thread's elements of a tile: where they go, where the first segment's come from, how far along the contraction
  uint32_t at_a[LOADS], at_b[LOADS];
  const float *from_a[LOADS], *from_b[LOADS];
  int k_a[LOADS], k_b[LOADS];
#pragma unroll
  for (int e = 0; e < LOADS; ++e) {
    const int idx = threadIdx.x + e * THREADS;
    const int ka = a_along_k ? idx & (TK - 1) : idx / TILE, ii = a_along_k ? idx / TK : idx & (TILE - 1);
    const int kb = b_along_k ? idx & (TK - 1) : idx / TILE, jj = b_along_k ? idx / TK : idx & (TILE - 1);
    const int gj = j0 + jj, jw = p.b_wrap > 0 ? gj % p.b_wrap : gj;
    at_a[e] = (uint32_t)__cvta_generic_to_shared(&As[0][ka][ii]);
    at_b[e] = (uint32_t)__cvta_generic_to_shared(&Bs[0][kb][jj]);
    k_a[e] = i0 + ii < p.rows ? ka : p.kc;                  // never below the contraction's end: nothing there
    k_b[e] = gj < p.cols ? kb : p.kc;
    from_a[e] = A + (i0 + ii) * p.sa_i + ka * p.sa_k;
    from_b[e] = B + kb * p.sb_k + jw * p.sb_j;
  }
  const int per_seg = (p.kc + TK - 1) / TK, steps = per_seg * p.segs;
  const long long step_a = TK * p.sa_k, step_b = TK * p.sb_k;
  long long off_a = 0, off_b = 0, seg_b = 0;
  int k0 = 0, buf_in = 0;
  auto fetch = [&](int step) {                              // the next tile; always a group, so that waiting counts
    if (step < steps) {
      const uint32_t to = (uint32_t)(buf_in * TK * (TILE + 4) * 4);
#pragma unroll
      for (int e = 0; e < LOADS; ++e) {
        const bool a = k0 + k_a[e] < p.kc, b = k0 + k_b[e] < p.kc;
        copy(at_a[e] + to, a ? from_a[e] + off_a : A, a);
        copy(at_b[e] + to, b ? from_b[e] + off_b : B, b);
      }
      k0 += TK; off_a += step_a; off_b += step_b;
      if (k0 >= p.kc) { k0 = 0; off_a = 0; seg_b += p.sb_seg; off_b = seg_b; }
      if (++buf_in == STAGES) buf_in = 0;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int s = 0; s < STAGES - 1; ++s) fetch(s);
  for (int step = 0; step < steps; ++step) {
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
    __syncthreads();                                        // this tile is there for all, and the one before has been read by all
    fetch(step + STAGES - 1);
    const float (*Ab)[TILE + 4] = As[step % STAGES], (*Bb)[TILE + 4] = Bs[step % STAGES];
#pragma unroll
    for (int kk = 0; kk < TK; ++kk) {
      float a[R], b[R];
      if constexpr (R == 4) {
        const float4 u = *reinterpret_cast<const float4*>(&Ab[kk][ty * 4]), v = *reinterpret_cast<const float4*>(&Bb[kk][tx * 4]);
        a[0] = u.x; a[1] = u.y; a[2] = u.z; a[3] = u.w;
        b[0] = v.x; b[1] = v.y; b[2] = v.z; b[3] = v.w;
      } else {
        const float2 u = *reinterpret_cast<const float2*>(&Ab[kk][ty * 2]), v = *reinterpret_cast<const float2*>(&Bb[kk][tx * 2]);
        a[0] = u.x; a[1] = u.y;
        b[0] = v.x; b[1] = v.y;
      }
#pragma unroll
      for (int q = 0; q < R; ++q)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[q][r] = fmaf(a[q], b[r], acc[q][r]);
    }
  }
  const int col0 = j0 + tx * R;
  const int n = p.cols - col0;
  if (n <= 0) return;
#pragma unroll
  for (int q = 0; q < R; ++q) {
    const int row = i0 + ty * R + q;
    if (row < p.rows) epi.template operator()<R>(row, col0, n, acc[q]);
  }
}

}  // namespace simt
}  // namespace et
