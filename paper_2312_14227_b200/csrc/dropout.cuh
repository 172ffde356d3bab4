// Dropout without a stored mask (ET_LAYER_DROPOUT): element e of the [M x width] matrix stays where word e % 4 of the generator's
// block e / 4 is at least `limit` = p 2^32, and is multiplied by 1 / (1 - limit 2^-32).  The generator is Philox 4x32 with ten rounds
// (Salmon, Moraes, Dror, Shaw, SC 2011): counter (block low, block high, step, layer), key = seed.  The backward pass forms the same
// words again.
//
// Bound by HBM: 4 bytes an element of bf16 (6 with the residual).  Ten rounds are 20 wide products for four elements, about 20
// instructions an element.
#pragma once

#include "common.cuh"

namespace et {

constexpr int kDropThreads = 256;

__device__ __forceinline__ uint4 philox(uint4 c, uint2 k) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k.x, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k.y, (uint32_t)a);
    k.x += 0x9E3779B9u;
    k.y += 0xBB67AE85u;
  }
  return c;
}

struct DropArgs {
  const uint64_t* seed;      // device: seed, step; nullptr: every element stays as it is
  size_t count;
  uint32_t limit, layer;
  float scale;
  int act;                   // backward: activation below
};
// out = kept ? in * scale : 0, + add.  z, dz: also dz = out * act'(z); out may then be nullptr.
template <typename T>
__global__ void __launch_bounds__(kDropThreads)
dropout_kernel(const T* __restrict__ in, const T* __restrict__ add, T* __restrict__ out, const T* __restrict__ z, T* __restrict__ dz,
               const DropArgs a) {
  chain_begin();
  constexpr int V = 8;
  const size_t e0 = ((size_t)blockIdx.x * kDropThreads + threadIdx.x) * V;
  if (e0 >= a.count) return;
  const int n = a.count - e0 < (size_t)V ? (int)(a.count - e0) : V;
  float v[V], t[V];
  load_seg<V>(in + e0, n, v);
  if (add != nullptr) load_seg<V>(add + e0, n, t);
  if (a.seed != nullptr) {
    const uint64_t seed = a.seed[0];
    const uint32_t step = (uint32_t)a.seed[1];
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
      const uint64_t block = e0 / 4 + q;
      const uint4 w = philox(make_uint4((uint32_t)block, (uint32_t)(block >> 32), step, a.layer), make_uint2((uint32_t)seed, (uint32_t)(seed >> 32)));
      const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * q + i] = word[i] >= a.limit ? v[4 * q + i] * a.scale : 0.0f;
    }
  }
  if (add != nullptr) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += t[i];
  }
  if (out != nullptr) store_seg<V>(out + e0, n, v);
  if (dz != nullptr) {
    load_seg<V>(z + e0, n, t);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] *= act_grad(t[i], a.act);
    store_seg<V>(dz + e0, n, v);
  }
}

}  // namespace et
