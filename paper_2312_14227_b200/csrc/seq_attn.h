// Launches of the kernels in seq_attn.cuh, compiled in a unit of their own.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace et {
namespace seqattn {

struct Mask {
  const int32_t* begin;     // [n + 1] or nullptr: sequences of `len` rows
  const int32_t* prefix;    // [n] or nullptr
  int n, len, M;
  bool causal;
};
struct Args {
  Mask mask;
  float* lse;               // [heads][ld]: log2 of the sum of 2^(s log2 e); +inf for a row without keys
  float* D;                 // [heads][ld]
  const float* slopes;      // [heads] or nullptr
  void* rest;               // [M][heads dim] bf16: the output less its rounding to bf16, in rows of few keys
  int* keys;                // [M]: keys that a row sees
  uint32_t* status;
  int heads, kv, dim, ld;   // ld: M rounded up to a multiple of 128
  int halves;               // forward: 1 or 2 halves of 128 rows a block
  bool dot;                 // backward: D is formed in the dq pass
  float scale, cap;
};

// Tensor maps of head blocks (boxes of 64 columns x 128 rows): qkv the input, out the output, g the output's gradient, gqkv (and dqkv, the
// same memory) where the input's gradient goes.
cudaError_t forward(const CUtensorMap& qkv, const CUtensorMap& out, Args a, int sms, cudaStream_t st);
// Launches: D (unless the dq pass forms it: *launches = 2), dq, (dk, dv).
cudaError_t backward(const CUtensorMap& qkv, const CUtensorMap& g, const CUtensorMap& gqkv, const void* out, const void* dout, void* dqkv,
                     Args a, int sms, int* launches, cudaStream_t st);

}  // namespace seqattn
}  // namespace et
