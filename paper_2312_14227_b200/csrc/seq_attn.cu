// Launches of the sequence attention kernels: one instance per padded head width, capped or not, with a distance bias or not.
#include "seq_attn.cuh"

#include <mutex>

namespace et {
namespace seqattn {
namespace {

std::mutex g_mutex;

// Dynamic shared memory above 48 KB has to be allowed once per kernel and device.  A kernel that hands registers over among its warps needs
// that many at its launch: with fewer, those that ask would wait for ever.
template <auto kern>
cudaError_t allow(uint32_t bytes, int registers = 0) {
  static bool done[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_mutex);
  if (done[dev]) return cudaSuccess;
  cudaFuncAttributes has{};
  e = cudaFuncGetAttributes(&has, kern);
  if (e != cudaSuccess) return e;
  if (has.numRegs < registers) return cudaErrorInvalidConfiguration;
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  done[dev] = e == cudaSuccess;
  return e;
}
// The kernels begin with chain_begin(): their launch latency overlaps the stream's previous kernel.
template <typename... P, typename... A>
cudaError_t launch(void (*kern)(P...), unsigned grid, unsigned block, uint32_t smem, cudaStream_t st, unsigned parts, A&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = parts;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = parts > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
}
template <typename F>
cudaError_t by_form(const Args& a, F&& f) {
  auto with = [&](auto wide, auto cap) {
    return a.slopes != nullptr ? f(wide, cap, std::true_type()) : f(wide, cap, std::false_type());
  };
  auto both = [&](auto wide) { return a.cap > 0.0f ? with(wide, std::true_type()) : with(wide, std::false_type()); };
  return a.dim > 64 ? both(std::integral_constant<int, 128>()) : both(std::integral_constant<int, 64>());
}

}  // namespace

cudaError_t forward(const CUtensorMap& qkv, const CUtensorMap& out, Args a, int sms, cudaStream_t st) {
  // two halves a block where that still gives every SM a block: the tensor core then works on one half's products during the
  // other's exponentials; else twice the blocks of one half
  const long long pairs = (long long)((a.mask.M + 255) / 256) * a.heads;
  a.halves = pairs >= sms ? 2 : 1;
  const unsigned grid = (unsigned)((a.mask.M + 128 * a.halves - 1) / (128 * a.halves)) * (unsigned)a.heads;
  return by_form(a, [&](auto wide, auto cap, auto bias) -> cudaError_t {
    constexpr auto kern = forward_kernel<decltype(wide)::value, decltype(cap)::value, decltype(bias)::value>;
    constexpr uint32_t smem = FwdCfg<decltype(wide)::value>::SMEM;
    const cudaError_t e = allow<kern>(smem, FWD_REGS);
    return e != cudaSuccess ? e : launch(kern, grid, FWD_THREADS, smem, st, 1, qkv, out, a);
  });
}

cudaError_t backward(const CUtensorMap& qkv, const CUtensorMap& g, const CUtensorMap& gqkv, const void* out, const void* dout, void* dqkv,
                     Args a, int sms, int* launches, cudaStream_t st) {
  const unsigned tiles = (unsigned)((a.mask.M + 127) / 128);
  // one wave of blocks at most: a launch of its own for D takes longer than the threads' own sums (37 rows, 4 heads, forward and backward: 25.0 -> 24.2 us)
  a.dot = (long long)tiles * a.heads <= sms;
  *launches = a.dot ? 2 : 3;
  if (!a.dot) {
    const long long threads = (long long)a.mask.M * a.heads * 16;
    const cudaError_t e = launch(dot_kernel, (unsigned)((threads + 255) / 256), 256, 0, st, 1, (const bf16*)out, (const bf16*)a.rest,
                                 a.keys, (const bf16*)dout, a.D, a.mask.M, a.heads, a.dim, a.ld);
    if (e != cudaSuccess) return e;
  }
  const Dots dots{(const bf16*)out, (const bf16*)dout};
  return by_form(a, [&](auto wide, auto cap, auto bias) -> cudaError_t {
    constexpr int W = decltype(wide)::value;
    constexpr auto dq = backward_kernel<W, false, decltype(cap)::value, decltype(bias)::value>;
    constexpr auto dkv = backward_kernel<W, true, decltype(cap)::value, decltype(bias)::value>;
    constexpr uint32_t smem = BwdCfg<W>::SMEM;
    cudaError_t r = allow<dq>(smem);
    if (r == cudaSuccess) r = allow<dkv>(smem);
    // Few items, or key heads that many query heads share: a cluster of blocks takes an item's tiles in turn and joins the sums, until
    // there are two blocks an SM (so that causal items, the longest twice the mean, even out) or fewer than two tiles a block.
    auto parts = [&](long long items, long long tiles_each) {
      unsigned n = 1;
      while (n < 8 && items * n < 2 * sms && tiles_each >= 4 * n) n *= 2;
      return n;
    };
    const unsigned pq = parts(tiles * a.heads, tiles), pk = parts(tiles * a.kv, (long long)tiles * (a.heads / a.kv));
    if (r == cudaSuccess) r = launch(dq, tiles * a.heads * pq, THREADS, smem, st, pq, qkv, g, gqkv, (bf16*)dqkv, dots, a);
    if (r == cudaSuccess) r = launch(dkv, tiles * a.kv * pk, THREADS, smem, st, pk, qkv, g, gqkv, (bf16*)dqkv, dots, a);
    return r;
  });
}

}  // namespace seqattn
}  // namespace et
