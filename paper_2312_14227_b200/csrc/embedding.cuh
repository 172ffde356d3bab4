// Embedding lookup as the first layer of a stack, and the gradient of its table by sorted tokens.
//   a_1[i]  = s * T[id_i]                          rows of zeros for ids outside [0, V)
//   dT[v]   = s * sum over the rows i with id_i = v of G_1[i]
// The rows are sorted by id (stable radix sort: rows of one id stay in order), the sorted positions are cut into
// chunks of kEmbChunk, and a block adds up the rows of one chunk, id by id.  An id whose rows lie within one chunk is
// finished there; an id that crosses chunk borders leaves one fp32 partial row per chunk, which a second kernel adds
// in order.  The sums' order depends on the ids alone.  Work per block of the gradient kernel is the same whatever the ids'
// frequencies.  Not so in the second kernel: one block per 256 columns adds all partial rows of an id, a 32nd of its tokens, so an id
// with half of the batch shows (plain SGD on a bf16 table of 65536 rows: 32768 tokens x 2048 columns 81 -> 96 us, 65536 x 1024
// 81 -> 121 us, 262144 x 256 105 -> 284 us).
#pragma once

#include "kernels.cuh"

namespace et {

constexpr int kEmbChunk = 32;              // sorted positions per block of the gradient kernel
constexpr int kSortThreads = 512;
constexpr int kSortPerThread = 4;
constexpr int kSortTile = kSortThreads * kSortPerThread;   // ids per block of a sorting pass
constexpr int kSortMaxBits = 9;            // digit bits of one pass
constexpr int kSortOneMax = 4096;          // up to this many ids one block sorts them all
constexpr int kSortOneBits = 8;

// VEC kernels take widths that are multiples of kVec with 16-byte aligned bases: eight elements move as whole vectors without a
// test, so that the compiler can put the loads of several rows on their way together (behind load_seg's tests it cannot: 103
// against 60 us for the gradient kernel of 32768 x 2048).
// Eight elements as they lie in memory: what is held while loads are on their way (four registers for bf16, not eight).
template <typename T, bool VEC> struct EmbRaw;
template <> struct EmbRaw<float, true> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p, int) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
  __device__ __forceinline__ void get(float (&v)[kVec]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};
template <> struct EmbRaw<bf16, true> {
  uint4 q;
  __device__ __forceinline__ void load(const bf16* p, int) { q = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&v)[kVec]) const {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(w[j] << 16);
      v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  }
};
template <typename T> struct EmbRaw<T, false> {
  float f[kVec];
  __device__ __forceinline__ void load(const T* p, int n) { load_seg<kVec>(p, n, f); }
  __device__ __forceinline__ void get(float (&v)[kVec]) const {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = f[i];
  }
};
template <bool VEC, typename T>
__device__ __forceinline__ void emb_load(const T* p, int n, float (&v)[kVec]) {
  EmbRaw<T, VEC> r;
  r.load(p, n);
  r.get(v);
}
// ---- lookup: one warp per row -----------------------------------------------------------------
// A copy with random rows: DRAM.  65536 rows of 1024 bf16 28 us (87 % of the copy bandwidth, each named row counted once).
template <typename T, bool VEC>
__global__ void __launch_bounds__(256)
embed_forward_kernel(const T* __restrict__ table, const int32_t* __restrict__ ids, T* __restrict__ out, long long rows,
                     int vocab, int d, float scale) {
  chain_begin();
  constexpr int U = 4;                                      // loads of a row that are on their way at once
  const int lane = threadIdx.x & 31;
  for (long long r = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += (long long)gridDim.x * 8) {
    const int id = ids[r];
    const bool ok = id >= 0 && id < vocab;
    const T* src = table + (size_t)(ok ? id : 0) * d;
    const float f = ok ? scale : 0.0f;
    T* dst = out + (size_t)r * d;
    int c = lane * kVec;
    if (VEC && ok) {
      for (; c + (U - 1) * 32 * kVec < d; c += U * 32 * kVec) {
        float v[U][kVec];
#pragma unroll
        for (int u = 0; u < U; ++u) emb_load<VEC>(src + c + u * 32 * kVec, kVec, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
          for (int i = 0; i < kVec; ++i) v[u][i] *= f;
          store_seg<kVec>(dst + c + u * 32 * kVec, kVec, v[u]);
        }
      }
    }
    for (; c < d; c += 32 * kVec) {
      float v[kVec];
      load_seg<kVec>(src + c, ok ? min(kVec, d - c) : 0, v);
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[i] *= f;
      store_seg<kVec>(dst + c, min(kVec, d - c), v);
    }
  }
}

// ---- what becomes of a finished gradient row: the tail of wgrad_reduce_elems ----------------------
template <typename T>
struct EmbSink {
  float* grad;
  const T* delta;
  T* W;
  float* master;
  float* m_state;
  float* v_state;
  OptParams opt;
  int do_sgd, delta_is_snapshot;
  size_t wrap;               // not 0: `grad` is a scratch of so many elements (whole rows), written over and over (et_profile_costs)
};
template <typename T>
__device__ __forceinline__ void emb_sgd(const EmbSink<T>& k, size_t i0, float (&w)[kVec], const float (&g)[kVec]) {
#pragma unroll
  for (int i = 0; i < kVec; ++i) w[i] = fmaf(-k.opt.lr, g[i], w[i]);        // opt_update's plain SGD
  if (k.master != nullptr) store_seg<kVec>(k.master + i0, kVec, w);
  store_seg<kVec>(k.W + i0, kVec, w);
}
// Importance, optimisers and ragged widths: called, not inlined.  Eight inlined copies of the optimisers in the gradient kernel's
// unrolled loop cost it more in instruction fetches than a call does (28 against 10 us for 300 rows, caches cold).
struct Eight { float v[kVec]; };
template <typename T>
__device__ __noinline__ float emb_finish_call(const EmbSink<T>& k, size_t i0, int n, Eight e) {
  float g[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) g[i] = e.v[i];
  float* grad = k.wrap == 0 ? k.grad : k.grad + (i0 % k.wrap) - i0;
  return consume_grad<T>(i0, n, g, grad, k.delta, k.W, k.opt, k.do_sgd, k.delta_is_snapshot, k.master, k.m_state, k.v_state);
}
// Ways a finished row is consumed.  Export: it is written and nothing else is wanted.  Sgd, SgdMaster: w <- w - lr g and nothing else,
// on the table or on its fp32 master.  General: all the rest, and ragged widths.
enum EmbWay { kEmbGeneral = 0, kEmbExport = 1, kEmbSgd = 2, kEmbSgdMaster = 3 };
template <int WAY, typename T> struct EmbWeight { using type = T; };          // where the current weight is read
template <typename T> struct EmbWeight<kEmbSgdMaster, T> { using type = float; };
template <int WAY, typename T>
__device__ __forceinline__ const typename EmbWeight<WAY, T>::type* emb_weight(const EmbSink<T>& k) {
  if constexpr (WAY == kEmbSgdMaster) return k.master;
  else return k.W;
}
template <int WAY, typename T>
__device__ __forceinline__ float emb_finish(const EmbSink<T>& k, size_t i0, int n, const float (&g)[kVec]) {
  if constexpr (WAY == kEmbExport) {
    float4* p = reinterpret_cast<float4*>(k.grad + i0);
    __stcs(p, make_float4(g[0], g[1], g[2], g[3]));
    __stcs(p + 1, make_float4(g[4], g[5], g[6], g[7]));
    return 0.0f;
  } else if constexpr (WAY >= kEmbSgd) {
    float w[kVec];
    emb_load<true>(emb_weight<WAY>(k) + i0, kVec, w);
    emb_sgd(k, i0, w, g);
    return 0.0f;
  } else {
    Eight e;
#pragma unroll
    for (int i = 0; i < kVec; ++i) e.v[i] = g[i];
    return emb_finish_call<T>(k, i0, n, e);
  }
}
// Table rows that no token names: their gradient is 0.  It is exported, and optimisers whose state or decay moves a weight without
// a gradient get it; plain SGD and the importance sum have nothing to do there.  `named` has a bit per table row.  The rows
// [v0, v1) are shared by `blocks` blocks; a warp takes a stretch of kFillCols columns of a row at a time.
template <typename T>
struct EmbFill {
  EmbSink<T> sink;
  const uint32_t* named;
  int v0, v1, d;
};
constexpr int kFillCols = 1024;
template <typename T>
__device__ __forceinline__ void embed_fill(const EmbFill<T>& f, int block, int blocks) {
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5, segs = (f.d + kFillCols - 1) / kFillCols;
  const bool zeros = f.sink.do_sgd == 0 && f.d % 4 == 0 && (reinterpret_cast<uintptr_t>(f.sink.grad) & 15) == 0;
  const long long units = (long long)(f.v1 - f.v0) * segs;
  for (long long u = block * warps + (threadIdx.x >> 5); u < units; u += blocks * warps) {
    const int v = f.v0 + (int)(u / segs), c0 = (int)(u % segs) * kFillCols, c1 = min(f.d, c0 + kFillCols);
    if ((f.named[v >> 5] >> (v & 31)) & 1u) continue;
    if (zeros) {                                            // a gradient that is exported and not applied
      size_t at = (size_t)v * f.d;
      if (f.sink.wrap != 0) at %= f.sink.wrap;
      float4* g = reinterpret_cast<float4*>(f.sink.grad + at);
      for (int c = c0 / 4 + lane; c < c1 / 4; c += 32) __stcs(g + c, make_float4(0.0f, 0.0f, 0.0f, 0.0f));
    } else {
      for (int c = c0 + lane * kVec; c < c1; c += 32 * kVec) {
        float g[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) g[i] = 0.0f;
        emb_finish<kEmbGeneral>(f.sink, (size_t)v * f.d + c, min(kVec, c1 - c), g);
      }
    }
  }
}

// ---- stable radix sort of (id, row) --------------------------------------------------------------
// Ids outside [0, vocab) become `vocab` and end up behind all others.
__device__ __forceinline__ uint32_t emb_key(int32_t id, int vocab) { return id >= 0 && id < vocab ? (uint32_t)id : (uint32_t)vocab; }

// Sets an id's bit.  Frequent ids find it set and leave the word alone: 60000 tokens of 300 ids would queue up at ten words.
__device__ __forceinline__ void emb_name(uint32_t* named, uint32_t key) {
  const uint32_t bit = 1u << (key & 31);
  if ((__ldcg(named + (key >> 5)) & bit) == 0) atomicOr(&named[key >> 5], bit);
}
// Ranks a warp's keys, 32 at a time in order: rank = keys of the same digit the warp has met before.  cnt: the warp's counters.
template <int E, typename Cnt>
__device__ __forceinline__ void warp_ranks(const uint32_t (&key)[E], const bool (&in)[E], int shift, int mask, Cnt* cnt,
                                           uint32_t (&rank)[E]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int q = 0; q < E; ++q) {
    const uint32_t dig = in[q] ? (key[q] >> shift) & mask : 0xffffffffu;
    const uint32_t same = __match_any_sync(0xffffffffu, dig);
    rank[q] = in[q] ? cnt[dig] + __popc(same & ((1u << lane) - 1u)) : 0u;
    __syncwarp();
    if (in[q] && lane == 31 - __clz(same)) cnt[dig] += (Cnt)__popc(same);
    __syncwarp();
  }
}
// Exclusive scan over the values of the block's first `n` threads (n a multiple of 32, at most blockDim.x <= 1024); every thread calls.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, int n) {
  __shared__ uint32_t wsum[32];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  uint32_t s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  if (lane == 31) wsum[wid] = s;
  __syncthreads();
  uint32_t w = lane < n / 32 ? wsum[lane] : 0u, before = 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {                        // sum of the warps before this one
    if (o == 16) w = lane < wid ? w : 0u;
    w += __shfl_xor_sync(0xffffffffu, w, o);
  }
  before = w;
  __syncthreads();
  return before + s - v;
}

// Up to kSortOneMax ids: one block, everything in shared memory, 8 bits a pass.  Also the bits of the named table rows.
static __global__ void __launch_bounds__(1024)
sort_one_kernel(const int32_t* __restrict__ ids, int n, int vocab, int bits, uint32_t* __restrict__ keys_out,
                uint32_t* __restrict__ rows_out, uint32_t* __restrict__ named) {
  chain_begin();
  constexpr int E = kSortOneMax / 1024, BINS = 1 << kSortOneBits;
  __shared__ uint16_t cnt[32][BINS];
  __shared__ uint32_t sk[kSortOneMax];
  __shared__ uint16_t sr[kSortOneMax];
  __shared__ uint32_t base[BINS];
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int warps = (n + E * 32 - 1) / (E * 32);            // warps that hold ids
  if (named != nullptr)
    for (int i = tid; i < (vocab + 31) / 32; i += 1024) named[i] = 0;
  // a warp owns E * 32 consecutive positions; few ids: the first warps hold them all
  uint32_t key[E], row[E], rank[E];
  bool in[E];
#pragma unroll
  for (int q = 0; q < E; ++q) {
    const int i = wid * (E * 32) + q * 32 + lane;
    in[q] = i < n;
    key[q] = in[q] ? emb_key(ids[i], vocab) : 0u;
    row[q] = i;
  }
  __syncthreads();
  if (named != nullptr) {
#pragma unroll
    for (int q = 0; q < E; ++q)
      if (in[q] && key[q] < (uint32_t)vocab) emb_name(named, key[q]);
  }
  for (int shift = 0; shift < bits; shift += kSortOneBits) {
    for (int i = tid; i < warps * BINS / 2; i += 1024) reinterpret_cast<uint32_t*>(&cnt[0][0])[i] = 0;
    __syncthreads();
    if (wid < warps) warp_ranks<E>(key, in, shift, BINS - 1, cnt[wid], rank);
    __syncthreads();
    uint32_t total = 0;
    if (tid < BINS)
      for (int w0 = 0; w0 < warps; w0 += 8) {               // eight warps' counts at a time: one shared-memory latency for them
        uint32_t c[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) c[k] = w0 + k < warps ? cnt[w0 + k][tid] : 0u;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (w0 + k < warps) cnt[w0 + k][tid] = (uint16_t)total;
          total += c[k];
        }
      }
    const uint32_t at = block_scan(tid < BINS ? total : 0u, 1024);
    if (tid < BINS) base[tid] = at;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < E; ++q)
      if (in[q]) {
        const uint32_t dig = (key[q] >> shift) & (BINS - 1), pos = base[dig] + cnt[wid][dig] + rank[q];
        sk[pos] = key[q];
        sr[pos] = (uint16_t)row[q];
      }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < E; ++q) {
      const int i = wid * (E * 32) + q * 32 + lane;
      if (in[q]) { key[q] = sk[i]; row[q] = sr[i]; }
    }
  }
#pragma unroll
  for (int q = 0; q < E; ++q) {
    const int i = wid * (E * 32) + q * 32 + lane;
    if (in[q]) { keys_out[i] = key[q]; rows_out[i] = row[q]; }
  }
}

// More ids.  First: digit counts of every tile for the first pass, hist[tile][digit]; the other passes' counts are cleared; the
// bits of the named table rows (cleared before).
static __global__ void __launch_bounds__(kSortThreads)
sort_hist_kernel(const int32_t* __restrict__ ids, int n, int vocab, int bits, uint32_t* __restrict__ hist, int passes,
                 uint32_t* __restrict__ named) {
  chain_begin();
  __shared__ uint32_t cnt[1 << kSortMaxBits];
  const int bins = 1 << bits;
  for (int i = threadIdx.x; i < bins; i += kSortThreads) cnt[i] = 0;
  __syncthreads();
  const long long i0 = (long long)blockIdx.x * kSortTile;
#pragma unroll
  for (int q = 0; q < kSortPerThread; ++q) {
    const long long i = i0 + q * kSortThreads + threadIdx.x;
    if (i >= n) continue;
    const uint32_t key = emb_key(ids[i], vocab);
    atomicAdd(&cnt[key & (bins - 1)], 1u);
    if (named != nullptr && key < (uint32_t)vocab) emb_name(named, key);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kSortThreads) {
    const size_t at = (size_t)blockIdx.x * bins + i, pass = (size_t)gridDim.x * bins;
    hist[at] = cnt[i];
    for (int p = 1; p < passes; ++p) hist[p * pass + at] = 0;
  }
}
// One pass: places every key of a tile where its digit begins for this tile plus its rank among the tile's keys of that digit, and
// counts the next pass's digits by the tile they land in.  Every tile reads all tiles' counts, so a pass reads tiles^2 * bins words
// from L2: nothing at 16 tiles, most of the time beyond a million ids (plain SGD on 64 columns: 65536 ids 44 us, 262144 83, 1 M
// 259, 4 M 1821).  Blocks behind the last tile fill table rows that no token names (the
// passes of few blocks would leave the GPU idle otherwise).
template <typename T>
__global__ void __launch_bounds__(kSortThreads)
sort_pass_kernel(const int32_t* __restrict__ ids, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ rows, int n,
                 int vocab, int shift, int bits, int tiles, const uint32_t* __restrict__ hist, uint32_t* __restrict__ hist_next,
                 uint32_t* __restrict__ keys_out, uint32_t* __restrict__ rows_out, const __grid_constant__ EmbFill<T> fill) {
  chain_begin();
  constexpr int kWarps = kSortThreads / 32, E = kSortPerThread;
  if ((int)blockIdx.x >= tiles) {
    embed_fill(fill, blockIdx.x - tiles, gridDim.x - tiles);
    return;
  }
  __shared__ uint16_t cnt[kWarps][1 << kSortMaxBits];
  __shared__ uint32_t base[1 << kSortMaxBits];
  const int bins = 1 << bits, lane = threadIdx.x & 31, wid = threadIdx.x >> 5, tile = blockIdx.x;
  for (int i = threadIdx.x; i < kWarps * (1 << kSortMaxBits) / 2; i += kSortThreads) reinterpret_cast<uint32_t*>(&cnt[0][0])[i] = 0;
  const long long i0 = (long long)tile * kSortTile + wid * (E * 32) + lane;
  uint32_t key[E], row[E], rank[E];
  bool in[E];
#pragma unroll
  for (int q = 0; q < E; ++q) {
    const long long i = i0 + q * 32;
    in[q] = i < n;
    key[q] = !in[q] ? 0u : keys != nullptr ? keys[i] : emb_key(ids[i], vocab);
    row[q] = in[q] && rows != nullptr ? rows[i] : (uint32_t)i;
  }
  // digit b (thread b): keys of it in the tiles before this one, and in all
  uint32_t before = 0, all = 0;
  if ((int)threadIdx.x < bins) {
#pragma unroll 8
    for (int j = 0; j < tiles; ++j) {
      const uint32_t c = hist[(size_t)j * bins + threadIdx.x];
      all += c;
      if (j < tile) before += c;
    }
  }
  __syncthreads();
  warp_ranks<E>(key, in, shift, bins - 1, cnt[wid], rank);
  const uint32_t at = block_scan(all, kSortThreads);
  if ((int)threadIdx.x < bins) {
    base[threadIdx.x] = at + before;
    uint32_t run = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t c = cnt[w][threadIdx.x];
      cnt[w][threadIdx.x] = (uint16_t)run;
      run += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < E; ++q) {
    if (!in[q]) continue;
    const uint32_t dig = (key[q] >> shift) & (bins - 1);
    const uint32_t pos = base[dig] + cnt[wid][dig] + rank[q];
    keys_out[pos] = key[q];
    rows_out[pos] = row[q];
    if (hist_next != nullptr) atomicAdd(&hist_next[(size_t)(pos / kSortTile) * bins + ((key[q] >> (shift + bits)) & (bins - 1))], 1u);
  }
}

// ---- gradient ------------------------------------------------------------------------------------
// Bound by DRAM and the latency of a chunk's batches of rows: 32768 rows of 2048 bf16, named rows exported, 43 us (238 MB).
// Block (chunk, column tile): sums of the chunk's rows, id by id.  part: [chunks][2][d]; slot 0 = the id the chunk
// continues from the one before, slot 1 = the id it hands on to the next.  imp_part: one number per block.
// Blocks behind the last chunk fill table rows that no token names.
template <typename T, bool VEC, int WAY>
__global__ void __launch_bounds__(256, WAY == kEmbGeneral || sizeof(T) == 4 ? 2 : 3)
embed_grad_kernel(const T* __restrict__ G, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ rows, int n, int vocab,
                  int d, float scale, int chunks, float* __restrict__ part, float* __restrict__ imp_part, const __grid_constant__ EmbSink<T> sink,
                  const __grid_constant__ EmbFill<T> fill) {
  chain_begin();
  constexpr bool SGD = WAY >= kEmbSgd;
  constexpr int U = sizeof(T) == 2 && WAY != kEmbSgdMaster ? 8 : 4;   // rows on their way at once
  if ((int)blockIdx.x >= chunks) {
    embed_fill(fill, (blockIdx.x - chunks) * gridDim.y + blockIdx.y, (gridDim.x - chunks) * gridDim.y);
    return;
  }
  // What happens after a row has been added: nothing (more of its id follows), the id is finished here, or its sum goes to one
  // of the chunk's two slots: 0 for an id that began in an earlier chunk, 1 for one that goes on in the next.
  enum { kMore = 0, kFinish = 1, kSlot0 = 2, kSlot1 = 3 };
  __shared__ uint32_t sk[kEmbChunk], sr[kEmbChunk];
  __shared__ uint8_t then[kEmbChunk];
  __shared__ int count;                                         // rows that take part: left-out ones are behind all others
  const int chunk = blockIdx.x, p0 = chunk * kEmbChunk, len = min(kEmbChunk, n - p0);
  if (threadIdx.x < 32) {                                       // kEmbChunk = 32: one lane per row
    const int i = threadIdx.x, p = p0 + i;
    const uint32_t key = i < len ? keys[p] : 0xffffffffu;
    const uint32_t behind = i < len && p + 1 < n ? keys[p + 1] : 0xffffffffu;
    const uint32_t before = p0 > 0 ? keys[p0 - 1] : 0xffffffffu;
    const bool in = key < (uint32_t)vocab;
    const uint32_t ins = __ballot_sync(0xffffffffu, in);
    sk[i] = key;
    sr[i] = in ? rows[p] : 0u;
    const bool last = i + 1 == len, ends = last || behind != key;
    then[i] = !in || !ends ? kMore : key == before ? kSlot0 : last && behind == key ? kSlot1 : kFinish;
    if (i == 0) count = __popc(ins);
  }
  __syncthreads();
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * kVec;
  const int nc = min(kVec, d - c), rows_in = count;
  float dot = 0.0f;
  if (nc > 0) {
    float acc[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) acc[i] = 0.0f;
    for (int q0 = 0; q0 < rows_in; q0 += U) {
      EmbRaw<T, VEC> raw[U];
      EmbRaw<typename EmbWeight<WAY, T>::type, true> weight[SGD ? U : 1];
#pragma unroll
      for (int u = 0; u < U; ++u) {                             // behind the last row: row 0 again, or nothing; not added
        const int q = min(q0 + u, kEmbChunk - 1);
        raw[u].load(G + (size_t)sr[q] * d + c, q0 + u < rows_in ? nc : 0);
        if constexpr (SGD) {
          if (q0 + u < rows_in && then[q] == kFinish) weight[u].load(emb_weight<WAY>(sink) + (size_t)sk[q] * d + c, kVec);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int q = q0 + u;
        if (q >= rows_in) break;
        float v[kVec];
        raw[u].get(v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) acc[i] += v[i];
        const int what = then[q];
        if (what == kMore) continue;
        if (what == kFinish) {
#pragma unroll
          for (int i = 0; i < kVec; ++i) acc[i] *= scale;
          if constexpr (SGD) {
            weight[u].get(v);
            emb_sgd(sink, (size_t)sk[q] * d + c, v, acc);
          } else dot += emb_finish<WAY>(sink, (size_t)sk[q] * d + c, nc, acc);
        } else {
          store_seg<kVec>(part + ((size_t)chunk * 2 + (what - kSlot0)) * d + c, nc, acc);
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) acc[i] = 0.0f;
      }
    }
  }
  if (imp_part != nullptr) {
    dot = block_sum(dot);
    if (threadIdx.x == 0) imp_part[blockIdx.y * chunks + chunk] = dot;
  }
}
static_assert(kEmbChunk == 32, "the gradient kernel's first warp looks at one row a lane");

// Block (group of kJoinChunks chunks, tile of 256 columns): the ids that begin in one of the chunks and go on in the next ones: adds
// their partial rows.  Warp j takes chunk j's id where it crosses few borders; the others are added by all warps, eight
// lanes of rows side by side, joined in a fixed order.
constexpr int kJoinChunks = 8, kJoinCols = 32 * kVec, kJoinAlone = 4;
template <typename T, bool VEC, int WAY>
__global__ void __launch_bounds__(256)
embed_join_kernel(const uint32_t* __restrict__ keys, int n, int vocab, int d, float scale, int chunks, const float* __restrict__ part,
                  float* __restrict__ imp_part, const __grid_constant__ EmbSink<T> sink) {
  chain_begin();
  __shared__ int count[kJoinChunks];                            // chunks that an id beginning in this one goes on in; 0: none does
  __shared__ float sm[8][kJoinCols];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int c = blockIdx.y * kJoinCols + lane * kVec, nc = min(kVec, d - c);
  {                                                             // a warp a chunk: how many chunks the id goes on in, 32 at a look
    const long long first = (long long)blockIdx.x * kJoinChunks + wid, p0 = first * kEmbChunk, p1 = p0 + kEmbChunk;
    int k = 0;
    if (p1 < n) {
      const uint32_t key = keys[p1 - 1];
      if (key < (uint32_t)vocab && keys[p1] == key && !(p0 > 0 && keys[p0 - 1] == key)) {
        for (;;) {
          const long long p = p1 + (long long)(k + lane) * kEmbChunk;
          const uint32_t same = __ballot_sync(0xffffffffu, p < n && keys[p] == key);
          k += __popc(same);                                    // sorted: the ones come first
          if (same != 0xffffffffu) break;
        }
      }
    }
    if (lane == 0) count[wid] = k;
  }
  __syncthreads();
  float dot = 0.0f;
  {                                                             // few partial rows: a warp adds them by itself, in order
    const int k = count[wid], chunk = blockIdx.x * kJoinChunks + wid;
    if (k > 0 && k < kJoinAlone && nc > 0) {
      float acc[kVec], v[kJoinAlone - 1][kVec];
      const float* p = part + (size_t)chunk * 2 * d + c;
      emb_load<VEC>(p + d, nc, acc);
#pragma unroll
      for (int r = 1; r < kJoinAlone; ++r)
        if (r <= k) emb_load<VEC>(p + (size_t)r * 2 * d, nc, v[r - 1]);
#pragma unroll
      for (int r = 1; r < kJoinAlone; ++r)
        if (r <= k) {
#pragma unroll
          for (int i = 0; i < kVec; ++i) acc[i] += v[r - 1][i];
        }
#pragma unroll
      for (int i = 0; i < kVec; ++i) acc[i] *= scale;
      dot += emb_finish<WAY>(sink, (size_t)keys[(size_t)(chunk + 1) * kEmbChunk] * d + c, nc, acc);
    }
  }
  for (int j = 0; j < kJoinChunks; ++j) {
    const int k = count[j];
    if (k < kJoinAlone) continue;
    const int chunk = blockIdx.x * kJoinChunks + j;
    // partial row r: slot 1 of the first chunk, slot 0 of the r-th one behind it; lane-of-rows `wid` takes r = wid, wid + 8, ...
    float acc[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) acc[i] = 0.0f;
    if (nc > 0) {
#pragma unroll 8
      for (int r = wid; r <= k; r += 8) {
        float v[kVec];
        emb_load<VEC>(part + ((size_t)(chunk + r) * 2 + (r == 0 ? 1 : 0)) * d + c, nc, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) acc[i] += v[i];
      }
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i) sm[wid][lane * kVec + i] = acc[i];
    __syncthreads();
    if (wid == 0 && nc > 0) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += sm[w][lane * kVec + i];
        acc[i] = s * scale;
      }
      const uint32_t key = keys[(size_t)(chunk + 1) * kEmbChunk];
      dot += emb_finish<WAY>(sink, (size_t)key * d + c, nc, acc);
    }
    __syncthreads();
  }
  if (imp_part != nullptr) {
    dot = block_sum(dot);
    if (threadIdx.x == 0) imp_part[blockIdx.y * gridDim.x + blockIdx.x] = dot;
  }
}

}  // namespace et
