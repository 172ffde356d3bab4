// Embedding lookup as the first layer of a stack, and the gradient of its table by sorted tokens.
//   a_1[i]  = s * T[id_i]                          rows of zeros for ids outside [0, V)
//   dT[v]   = s * sum over the rows i with id_i = v of G_1[i]
// The rows are sorted by id (stable radix sort: rows of one id stay in order), the sorted positions are cut into
// chunks of kEmbChunk, and a block adds up the rows of one chunk, id by id.  An id whose rows lie within one chunk is
// finished there; an id that crosses chunk borders leaves one fp32 partial row per chunk, which a second kernel adds
// in order.  Work per block is the same whatever the ids' frequencies, and the sums' order depends on the ids alone.
#pragma once

#include "kernels.cuh"

namespace et {

constexpr int kEmbChunk = 32;              // sorted positions per block of the gradient kernel
constexpr int kSortThreads = 256;
constexpr int kSortPerThread = 8;
constexpr int kSortTile = kSortThreads * kSortPerThread;   // ids per block of a sorting pass
constexpr int kSortMaxBits = 9;            // digit bits of one pass

// ---- lookup: one warp per row -----------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256)
embed_forward_kernel(const T* __restrict__ table, const int32_t* __restrict__ ids, T* __restrict__ out, long long rows,
                     int vocab, int d, float scale) {
  constexpr int V = 8;
  const int lane = threadIdx.x & 31;
  for (long long r = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += (long long)gridDim.x * 8) {
    const int id = ids[r];
    const bool ok = id >= 0 && id < vocab;
    const T* src = table + (size_t)(ok ? id : 0) * d;
    T* dst = out + (size_t)r * d;
    for (int c = lane * V; c < d; c += 32 * V) {
      const int n = min(V, d - c);
      float v[V];
      load_seg<V>(src + c, ok ? n : 0, v);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] *= scale;
      store_seg<V>(dst + c, n, v);
    }
  }
}

// ---- stable radix sort of (id, row) --------------------------------------------------------------
// Ids outside [0, vocab) become `vocab` and end up behind all others.
__device__ __forceinline__ uint32_t emb_key(const int32_t* ids, const uint32_t* keys, long long i, int vocab) {
  if (keys != nullptr) return keys[i];
  const int id = ids[i];
  return id >= 0 && id < vocab ? (uint32_t)id : (uint32_t)vocab;
}
// hist[digit * blocks + block] = how many keys of this block's tile have the digit
static __global__ void __launch_bounds__(kSortThreads)
sort_hist_kernel(const int32_t* __restrict__ ids, const uint32_t* __restrict__ keys, int n, int vocab, int shift, int bits,
                 uint32_t* __restrict__ hist) {
  __shared__ uint32_t cnt[1 << kSortMaxBits];
  const int bins = 1 << bits;
  for (int i = threadIdx.x; i < bins; i += kSortThreads) cnt[i] = 0;
  __syncthreads();
  const long long i0 = (long long)blockIdx.x * kSortTile;
  for (int q = 0; q < kSortPerThread; ++q) {
    const long long i = i0 + q * kSortThreads + threadIdx.x;
    if (i < n) atomicAdd(&cnt[(emb_key(ids, keys, i, vocab) >> shift) & (bins - 1)], 1u);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kSortThreads) hist[(size_t)i * gridDim.x + blockIdx.x] = cnt[i];
}
// exclusive scan in place, one block
static __global__ void __launch_bounds__(1024)
sort_scan_kernel(uint32_t* __restrict__ hist, int n) {
  __shared__ uint32_t wsum[32];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  uint32_t carry = 0;
  for (int i0 = 0; i0 < n; i0 += 1024) {
    const int i = i0 + threadIdx.x;
    const uint32_t v = i < n ? hist[i] : 0u;
    uint32_t s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t u = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += u;
    }
    if (lane == 31) wsum[wid] = s;
    __syncthreads();
    uint32_t before = 0, total = 0;
    for (int w = 0; w < 32; ++w) {
      if (w < wid) before += wsum[w];
      total += wsum[w];
    }
    if (i < n) hist[i] = carry + before + s - v;
    carry += total;
    __syncthreads();
  }
}
// Places every key of a tile: where the scan says its digit begins for this block, plus its rank among the tile's keys
// of the same digit.  A warp owns kSortPerThread * 32 consecutive keys and takes them 32 at a time in order.
static __global__ void __launch_bounds__(kSortThreads)
sort_scatter_kernel(const int32_t* __restrict__ ids, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ rows, int n,
                    int vocab, int shift, int bits, const uint32_t* __restrict__ offs, uint32_t* __restrict__ keys_out,
                    uint32_t* __restrict__ rows_out) {
  constexpr int kWarps = kSortThreads / 32;
  __shared__ uint32_t cnt[kWarps][1 << kSortMaxBits];
  const int bins = 1 << bits, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < kWarps * (1 << kSortMaxBits); i += kSortThreads) (&cnt[0][0])[i] = 0;
  __syncthreads();
  const long long i0 = (long long)blockIdx.x * kSortTile + wid * (kSortPerThread * 32);
  uint32_t key[kSortPerThread], rank[kSortPerThread];
#pragma unroll
  for (int q = 0; q < kSortPerThread; ++q) {
    const long long i = i0 + q * 32 + lane;
    const bool in = i < n;
    key[q] = in ? emb_key(ids, keys, i, vocab) : 0u;
    const uint32_t dig = in ? (key[q] >> shift) & (bins - 1) : 0xffffffffu;
    const uint32_t same = __match_any_sync(0xffffffffu, dig);
    rank[q] = in ? cnt[wid][dig] + __popc(same & ((1u << lane) - 1u)) : 0u;
    __syncwarp();
    if (in && lane == 31 - __clz(same)) cnt[wid][dig] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads) {      // per digit: where each warp's keys begin
    uint32_t at = offs[(size_t)b * gridDim.x + blockIdx.x];
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t c = cnt[w][b];
      cnt[w][b] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kSortPerThread; ++q) {
    const long long i = i0 + q * 32 + lane;
    if (i >= n) continue;
    const uint32_t pos = cnt[wid][(key[q] >> shift) & (bins - 1)] + rank[q];
    keys_out[pos] = key[q];
    rows_out[pos] = rows != nullptr ? rows[i] : (uint32_t)i;
  }
}

// ---- gradient ------------------------------------------------------------------------------------
template <typename T>
struct EmbSink {                 // what becomes of a finished gradient row: the tail of wgrad_reduce_elems
  float* grad;
  const T* delta;
  T* W;
  float* master;
  float* m_state;
  float* v_state;
  OptParams opt;
  int do_sgd, delta_is_snapshot;
};
template <typename T>
__device__ __forceinline__ float emb_finish(const EmbSink<T>& k, size_t i0, int n, const float (&g)[kVec]) {
  return consume_grad<T>(i0, n, g, k.grad, k.delta, k.W, k.opt, k.do_sgd, k.delta_is_snapshot, k.master, k.m_state, k.v_state);
}

// Block (chunk, column tile): sums of the chunk's rows, id by id.  part: [chunks][2][d]; slot 0 = the id the chunk
// continues from the one before, slot 1 = the id it hands on to the next.  imp_part: one number per block.
template <typename T>
__global__ void __launch_bounds__(256)
embed_grad_kernel(const T* __restrict__ G, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ rows, int n, int vocab,
                  int d, float scale, float* __restrict__ part, float* __restrict__ imp_part, const EmbSink<T> sink) {
  __shared__ uint32_t sk[kEmbChunk + 2], sr[kEmbChunk];
  const int chunk = blockIdx.x, p0 = chunk * kEmbChunk, len = min(kEmbChunk, n - p0);
  for (int i = threadIdx.x; i < len + 2; i += blockDim.x) {     // sk[0]: the key before, sk[len + 1]: the one behind
    const int p = p0 + i - 1;
    sk[i] = p >= 0 && p < n ? keys[p] : 0xffffffffu;
    if (i < len) sr[i] = rows[p0 + i];
  }
  __syncthreads();
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * kVec;
  const int nc = min(kVec, d - c);
  float dot = 0.0f;
  if (nc > 0) {
    float acc[kVec];
    bool head = sk[1] == sk[0];                                 // the first id began in an earlier chunk
#pragma unroll
    for (int i = 0; i < kVec; ++i) acc[i] = 0.0f;
    for (int q = 0; q < len; ++q) {
      const uint32_t key = sk[q + 1];
      if (key >= (uint32_t)vocab) break;                        // left-out rows: behind all others
      float v[kVec];
      load_seg<kVec>(G + (size_t)sr[q] * d + c, nc, v);
#pragma unroll
      for (int i = 0; i < kVec; ++i) acc[i] += v[i];
      if (q + 1 < len && sk[q + 2] == key) continue;            // more of this id in the chunk
      const bool tail = q + 1 == len && sk[q + 2] == key;       // ... or in the next one
      if (head || tail) {
        store_seg<kVec>(part + ((size_t)chunk * 2 + (head ? 0 : 1)) * d + c, nc, acc);
      } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) acc[i] *= scale;
        dot += emb_finish(sink, (size_t)key * d + c, nc, acc);
      }
      head = false;
#pragma unroll
      for (int i = 0; i < kVec; ++i) acc[i] = 0.0f;
    }
  }
  if (imp_part != nullptr) {
    dot = block_sum(dot);
    if (threadIdx.x == 0) imp_part[blockIdx.y * gridDim.x + blockIdx.x] = dot;
  }
}

// Block (chunk, column tile): the id that begins in this chunk and goes on in the next ones: adds its partial rows.
template <typename T>
__global__ void __launch_bounds__(256)
embed_join_kernel(const uint32_t* __restrict__ keys, int n, int vocab, int d, float scale, const float* __restrict__ part,
                  float* __restrict__ imp_part, const EmbSink<T> sink) {
  const int chunk = blockIdx.x, p0 = chunk * kEmbChunk, p1 = p0 + kEmbChunk;      // p1 <= n - 1 where anything follows
  float dot = 0.0f;
  if (p1 < n) {
    const uint32_t key = keys[p1 - 1];
    const bool spans = key < (uint32_t)vocab && keys[p1] == key;
    const bool begins_here = !(keys[p0] == key && p0 > 0 && keys[p0 - 1] == key);
    const int c = (blockIdx.y * blockDim.x + threadIdx.x) * kVec;
    const int nc = min(kVec, d - c);
    if (spans && begins_here && nc > 0) {
      float acc[kVec], v[kVec];
      load_seg<kVec>(part + ((size_t)chunk * 2 + 1) * d + c, nc, acc);
      for (int q = chunk + 1; q * kEmbChunk < n && keys[q * kEmbChunk] == key; ++q) {
        load_seg<kVec>(part + (size_t)q * 2 * d + c, nc, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) acc[i] += v[i];
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) acc[i] *= scale;
      dot = emb_finish(sink, (size_t)key * d + c, nc, acc);
    }
  }
  if (imp_part != nullptr) {
    dot = block_sum(dot);
    if (threadIdx.x == 0) imp_part[blockIdx.y * gridDim.x + blockIdx.x] = dot;
  }
}

// Table rows that no token names: their gradient is 0.  It is exported, and optimisers whose state or decay moves a
// weight without a gradient get it; the importance sum and plain SGD have nothing to do there.
template <typename T>
__global__ void __launch_bounds__(256)
embed_untouched_kernel(const uint32_t* __restrict__ keys, int n, int vocab, int d, const EmbSink<T> sink) {
  const int v = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (v >= vocab) return;
  int lo = 0, hi = n;                                           // first position with key >= v
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (keys[mid] < (uint32_t)v) lo = mid + 1; else hi = mid;
  }
  if (lo < n && keys[lo] == (uint32_t)v) return;
  for (int c = lane * kVec; c < d; c += 32 * kVec) {
    float g[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) g[i] = 0.0f;
    emb_finish(sink, (size_t)v * d + c, min(kVec, d - c), g);
  }
}

}  // namespace et
