// Softmax attention over packed sequences as a member of the stack (ET_LAYER_MASKED_ATTENTION).  Rows are
// [q of `heads` | k of `kv` | v of `kv`] blocks of `dim` columns; query head h reads key / value head h / (heads / kv).
//
//   s_ij = c tanh(scale q_i.k_j / c) - slope |i - j|      (no cap: scale q_i.k_j;  no bias: slope 0)
//   o_i  = sum_j p_ij v_j,  p_ij = exp(s_ij - lse_i),      j in [lo_i, hi_i)
//   D_i  = dO_i . o_i ;  ds_ij = p_ij (dO_i . v_j - D_i) (1 - tanh^2)
//   dq_i = scale sum_j ds_ij k_j ;  dk_j = scale sum_i ds_ij q_i ;  dv_j = sum_i p_ij dO_i
//
// Every mask that the layer knows (sequence bounds, causal, prefix) leaves a row ONE interval of keys, and a key one interval of
// rows: a thread owns a row (or key), keeps the two ends of its interval, and a tile is walked only where some interval meets it.
// A row of no sequence has an empty interval: its output and gradient are 0.  Rows of no sequence may hold anything, NaN
// included: they are overwritten with 0 in the tiles that a product reads as weights' other factor (0 * NaN is NaN).
//
// Forward: a block owns 256 (or 128) query rows of one head, two halves of 128.  Scores of a half against 128 keys
// (tcgen05, operands by TMA) lie in tensor memory, one accumulator row a thread; the thread takes the running maximum, writes
// exp(s - m) as bf16 over the scores, and P v reads P from tensor memory.  While one half's scores are worked on the tensor core
// serves the other half.  The output is rescaled only where a row's maximum has grown by more than 2^8: until then sums and
// output are relative to the older maximum, which fp32 holds as well.
// Backward: two passes of one kernel, dq (block = 128 query rows, keys stream by) and dk, dv (block = 128 keys of a key head, the
// rows of its group's heads stream by).  Both form S = X1 Y1^T and dP = X2 Y2^T against 64 streamed rows in tensor memory,
// write P and dS as bf16 over them, and accumulate dS Y1 (and P Y2) with P and dS read from tensor memory.  Nothing is added with
// atomics: a shared head's gradient is the sum that one block forms in order.  The price is that S and dP are formed
// twice, 7 products where 5 would do.
//
// Rounding: P and dS are bf16 (half a step 2^-9 of each term); scores, maxima, sums, D and all accumulators are fp32.
#pragma once

#include "attn.cuh"
#include "seq_attn.h"

namespace et {
namespace seqattn {

using namespace et::tc;

constexpr uint32_t kTimeoutSeqAttn = 8;
constexpr int THREADS = 320;                    // warps 0-3, 4-7: row threads; warp 8: MMA issue, TMEM; warp 9: TMA
constexpr uint32_t CHUNK = 16384;               // 128 rows x 64 columns of bf16
constexpr uint32_t HCHUNK = 8192;               // 64 rows x 64 columns
constexpr int STREAM = 64;                      // rows of a streamed tile of the backward pass
constexpr float LOG2E = 1.4426950408889634f;

// ---- intervals ---------------------------------------------------------------------------------
// Largest q with begin[q] <= row, -1 if there is none; the whole warp asks for one row, 32 probes at a time.  Ends for any contents.
__device__ __forceinline__ int find_seq(const int32_t* begin, int n, int row, int lane) {
  int lo = -1, hi = n + 1;
  while (hi - lo > 1) {
    const int step = (hi - lo - 1 + 31) / 32;
    const int at = lo + 1 + lane * step;
    const bool le = at < hi && begin[at] <= row;
    const unsigned ones = __ballot_sync(0xffffffffu, le);
    const int k = ones == 0xffffffffu ? 32 : __ffs(~ones) - 1;         // leading run of probes that are <= row
    if (k == 0) hi = lo + 1;
    else {
      const int base = lo + 1;
      lo = base + (k - 1) * step;
      if (k < 32) hi = min(hi, base + k * step);
    }
  }
  return lo;
}
// Interval of row `row` (lane's own; the warp's rows are consecutive, lane 0 first): its keys, or with KEYS the rows that see key `row`.
template <bool KEYS>
__device__ __forceinline__ int2 interval(const Mask& m, int row, int lane) {
  int b, e, q = 0;
  if (m.begin == nullptr) {
    if (row >= m.M) return make_int2(0, 0);
    b = row / m.len * m.len;
    e = min(b + m.len, m.M);
  } else {
    int lo = find_seq(m.begin, m.n, row - lane, lane);                 // of the warp's first and last row
    int hi = find_seq(m.begin, m.n, row - lane + 31, lane);
    while (lo < hi) {
      const int mid = lo + (hi - lo + 1) / 2;
      if (m.begin[mid] <= row) lo = mid; else hi = mid - 1;
    }
    q = lo;
    if (q < 0 || q >= m.n || row >= m.M) return make_int2(0, 0);
    b = min(max(m.begin[q], 0), m.M);
    e = min(max(m.begin[q + 1], 0), m.M);
  }
  if (m.causal) {
    const int pre = m.prefix != nullptr ? min(max(m.prefix[q], 0), max(e - b, 0)) : 0;
    if (KEYS) { if (row - b >= pre) b = row; }
    else e = min(e, max(row + 1, b + pre));
  }
  return e > b ? make_int2(b, e) : make_int2(0, 0);
}
// Rows that belong to some sequence: [first, last).
__device__ __forceinline__ int2 used_rows(const Mask& m) {
  if (m.begin == nullptr) return make_int2(0, m.M);
  return make_int2(min(max(m.begin[0], 0), m.M), min(max(m.begin[m.n], 0), m.M));
}

// ---- tensor memory -----------------------------------------------------------------------------
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(db), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void group_sync(int id) { asm volatile("bar.sync %0, 128;" ::"r"(id) : "memory"); }

// K-major operand of tiles of `chunk` bytes a 64-column piece
__device__ __forceinline__ uint64_t kdesc(uint32_t tile, int ks, uint32_t chunk) {
  return make_desc(tile + (uint32_t)(ks >> 2) * chunk + (uint32_t)(ks & 3) * 32u, 16, 1024);
}
__device__ __forceinline__ uint64_t mndesc(uint32_t tile, int ks, uint32_t chunk) {
  return make_desc(tile + (uint32_t)ks * 2048u, chunk, 1024);
}

// tanh from one exponential and one reciprocal: exp overflow gives 1, underflow -1, absolute error near 2^-23
__device__ __forceinline__ float tanh_of(float x2) {            // x2 = 2 x log2 e
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(attn::ex2(x2) + 1.0f));
  return fmaf(-2.0f, r, 1.0f);
}

// Rows of a 128-byte-swizzled tile that belong to no sequence become 0 (whole warp; the caller orders it before the products).
__device__ __forceinline__ void scrub(uint8_t* tile, int rows, int chunks, uint32_t chunk, int row0, int2 used, int lane) {
  for (int r = 0; r < rows; ++r) {
    if (row0 + r >= used.x && row0 + r < used.y) continue;
    for (int c = 0; c < chunks; ++c) *reinterpret_cast<uint32_t*>(tile + c * chunk + r * 128 + lane * 4) = 0;
  }
}

// Extent of the union of a block's intervals, by shared memory: {first, last} over non-empty ones.
__device__ __forceinline__ void note_extent(int* lo, int* hi, int2 iv) {
  const int l = __reduce_min_sync(0xffffffffu, iv.y > iv.x ? iv.x : 0x7fffffff);
  const int h = __reduce_max_sync(0xffffffffu, iv.y > iv.x ? iv.y : 0);
  if ((threadIdx.x & 31) == 0) { atomicMin(lo, l); atomicMax(hi, h); }
}

// ---- forward -----------------------------------------------------------------------------------
template <int DHP>
struct FwdCfg {
  static constexpr int CH = DHP / 64;                            // 64-column pieces of a tile
  static constexpr uint32_t TILE = CH * CHUNK;
  static constexpr int ST = DHP == 128 ? 4 : 6;                  // key and value tiles in flight
  static constexpr uint32_t SMEM = (2 + ST) * TILE + 1024 + 256;
};

template <int DHP, bool CAP, bool BIAS>
__global__ void __launch_bounds__(THREADS, 1)
forward_kernel(const __grid_constant__ CUtensorMap map_qkv, const __grid_constant__ CUtensorMap map_out, const Args a) {
  using C = FwdCfg<DHP>;
  constexpr int ST = C::ST;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t ring = base + 2 * C::TILE, bars = base + (2 + ST) * C::TILE;
  const uint32_t bar_q = bars;
  auto bar_s = [&](int h) { return bars + 8u + 8u * h; };         // scores of half h complete (and every product before)
  auto bar_p = [&](int h) { return bars + 24u + 8u * h; };        // P of half h is in tensor memory
  auto full = [&](int s) { return bars + 40u + 8u * s; };
  auto empty = [&](int s) { return bars + 40u + 8u * (ST + s); };
  int* shared = reinterpret_cast<int*>(gen + (2 + ST) * C::TILE + 160);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(shared);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  int* extent = shared + 2;                                       // lo, hi of half 0, of half 1

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tiles = (a.mask.M + 128 * a.halves - 1) / (128 * a.halves);
  const int h = blockIdx.x % a.heads;
  // causal rows see the more keys the later they come: the longest blocks start first
  const int tile = a.mask.causal ? tiles - 1 - (int)(blockIdx.x / a.heads) : (int)(blockIdx.x / a.heads);
  const int row0 = tile * 128 * a.halves;
  const int kvh = h / (a.heads / a.kv);

  if (threadIdx.x == 0) {
    prefetch_tmap(&map_qkv);
    prefetch_tmap(&map_out);
    mbar_init(bar_q, 1);
    for (int i = 0; i < 2; ++i) { mbar_init(bar_s(i), 1); mbar_init(bar_p(i), 128); extent[2 * i] = 0x7fffffff; extent[2 * i + 1] = 0; }
    for (int s = 0; s < ST; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    *abort_flag = 0;
    fence_async_smem();
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)tmem_slot)), "r"(TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  chain_begin();
  if (warp == 9 && lane == 0) {
    mbar_expect_tx(bar_q, (uint32_t)a.halves * C::TILE);
    for (int hf = 0; hf < a.halves; ++hf)
      for (int c = 0; c < C::CH; ++c) tma_load_3d(base + hf * C::TILE + c * CHUNK, &map_qkv, bar_q, c * 64, h, row0 + hf * 128);
  }
  int2 iv = make_int2(0, 0);
  if (warp < 8) {
    if ((warp >> 2) < a.halves) iv = interval<false>(a.mask, row0 + (int)threadIdx.x, lane);
    note_extent(extent + 2 * (warp >> 2), extent + 2 * (warp >> 2) + 1, iv);
  }
  __syncthreads();
  // tiles of 128 keys that each half walks; the stream covers both
  int first[2], last[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int lo = extent[2 * i], hi = extent[2 * i + 1];
    first[i] = hi > lo ? lo / 128 : 0;
    last[i] = hi > lo ? (hi + 127) / 128 : 0;
  }
  const bool any0 = last[0] > first[0], any1 = last[1] > first[1];
  const int T0 = any0 && any1 ? min(first[0], first[1]) : any0 ? first[0] : first[1];
  const int T1 = max(last[0], last[1]);
  const int n_tiles = max(T1 - T0, 0);

  if (warp == 9) {
    if (lane == 0) {
      bool ok = true;
      int fills = 0;
      for (int i = 0; i < 2 * n_tiles && ok; ++i) {               // K and V of the first tile, of the second, ...
        const int s = i % ST;
        ok = mbar_wait(empty(s), ((uint32_t)(i / ST) & 1u) ^ 1u, abort_flag, a.status, kTimeoutSeqAttn);
        if (!ok) break;
        mbar_expect_tx(full(s), C::TILE);
        const int block = a.heads + (i & 1 ? a.kv : 0) + kvh;
        for (int c = 0; c < C::CH; ++c) tma_load_3d(ring + s * C::TILE + c * CHUNK, &map_qkv, full(s), c * 64, block, (T0 + (i >> 1)) * 128);
        ++fills;
      }
      if (!ok) {                                                  // let the copies in flight land before shared memory goes away
        for (int i = max(0, fills - ST); i < fills; ++i)
          for (uint32_t it = 0; it < (1u << 20) && !mbar_try_wait(full(i % ST), (uint32_t)(i / ST) & 1u); ++it) {}
      }
      // Q must have landed, too, whoever waits for it
      for (uint32_t it = 0; it < (1u << 20) && !mbar_try_wait(bar_q, 0); ++it) {}
    }
  } else if (warp == 8) {
    const uint32_t id_s = attn::idesc128(128, false, false), id_o = attn::idesc128(DHP, false, true);
    const int2 used = used_rows(a.mask);
    bool ok = n_tiles == 0 || mbar_wait(bar_q, 0, abort_flag, a.status, kTimeoutSeqAttn);
    int np[2] = {0, 0};                                           // products P v issued per half
    for (int t = T0 - 1; t < T1 && ok; ++t) {
      const int ik = 2 * (t + 1 - T0), iv_ = 2 * (t - T0) + 1;    // stream positions of K of tile t + 1 and V of tile t
      const int sk = ik % ST, sv = iv_ < 0 ? 0 : iv_ % ST;
      const bool has_k = t + 1 < T1, has_v = t >= T0;
      if (has_k) ok = mbar_wait(full(sk), (uint32_t)(ik / ST) & 1u, abort_flag, a.status, kTimeoutSeqAttn);
      if (ok && has_v) ok = mbar_wait(full(sv), (uint32_t)(iv_ / ST) & 1u, abort_flag, a.status, kTimeoutSeqAttn);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (has_v && (t * 128 < used.x || (t + 1) * 128 > used.y)) {
        scrub(gen + (2 + sv) * C::TILE, 128, C::CH, CHUNK, t * 128, used, lane);
        fence_async_smem();
        __syncwarp();
      }
      tc_fence_after();
      for (int hf = 0; hf < 2; ++hf) {
        const bool pv = t >= first[hf] && t < last[hf], nx = t + 1 >= first[hf] && t + 1 < last[hf];
        if (!pv && !nx) continue;
        const uint32_t S = tmem + hf * 128, O = tmem + 256 + hf * DHP;
        if (pv) {
          ok = __all_sync(0xffffffffu, mbar_wait(bar_p(hf), (uint32_t)np[hf] & 1u, abort_flag, a.status, kTimeoutSeqAttn));
          if (!ok) break;
          tc_fence_after();
          if (lane == 0)
            for (int ks = 0; ks < 8; ++ks)
              mma_ts(O, S + ks * 8, mndesc(ring + sv * C::TILE, ks, CHUNK), id_o, (np[hf] > 0 || ks > 0) ? 1u : 0u);
          ++np[hf];
        }
        if (lane == 0) {
          if (nx)
            for (int ks = 0; ks < DHP / UK; ++ks)
              tc_mma(S, kdesc(base + hf * C::TILE, ks, CHUNK), kdesc(ring + sk * C::TILE, ks, CHUNK), id_s, ks > 0 ? 1u : 0u);
          tc_commit(bar_s(hf));                                   // next scores, or after the last tile the output
        }
        __syncwarp();
      }
      if (lane == 0) {
        if (has_k) tc_commit(empty(sk));
        if (has_v) tc_commit(empty(sv));
      }
      __syncwarp();
    }
  } else if ((warp >> 2) < a.halves) {
    const int hf = warp >> 2;
    const int trow = threadIdx.x & 127, row = row0 + (int)threadIdx.x;
    const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t S = tmem + lane_addr + hf * 128, O = tmem + lane_addr + 256 + hf * DHP;
    const float c2 = a.scale * LOG2E;
    const float slope2 = BIAS ? a.slopes[h] * LOG2E : 0.0f;
    float m = -INFINITY, sum = 0.0f;
    bool ok = true;
    const int n_own = last[hf] - first[hf];
    for (int i = 0; i < n_own && ok; ++i) {
      ok = mbar_wait(bar_s(hf), (uint32_t)i & 1u, abort_flag, a.status, kTimeoutSeqAttn);
      if (!ok) break;
      tc_fence_after();
      const int k0 = (first[hf] + i) * 128;
      float v[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32_issue(S + c * 32, v[c]);
      tmem_ld_wait(v[0], v[1]);
      tmem_ld_wait(v[2], v[3]);
      if (CAP || BIAS) {
        const float u = CAP ? 2.0f * c2 / a.cap : 0.0f, top = a.cap * LOG2E;
        const float d0 = (float)(row - k0);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            float s = CAP ? top * tanh_of(v[c][j] * u) : v[c][j] * c2;
            if (BIAS) s = fmaf(-slope2, fabsf(d0 - (float)(c * 32 + j)), s);
            v[c][j] = s;
          }
      }
      if (!__all_sync(0xffffffffu, iv.x <= k0 && iv.y >= k0 + 128)) {
        const int lo = iv.x - k0;
        const unsigned len = (unsigned)(iv.y - iv.x);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if ((unsigned)(c * 32 + j - lo) >= len) v[c][j] = -INFINITY;
      }
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int j = 0; j < 32; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) mx[c] = fmaxf(mx[c], v[c][j]);
      float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
      if (!(CAP || BIAS)) top *= c2;                              // scale > 0: the largest score stays the largest
      if (__any_sync(0xffffffffu, top > m + 8.0f)) {
        const float m_new = fmaxf(m, top);
        const float f = m == -INFINITY ? 0.0f : attn::ex2(m - m_new);
        sum *= f;
        m = m_new;
        if (i > 0) {                                              // the output so far is complete: bar_s follows it
#pragma unroll 1
          for (int c = 0; c < DHP; c += 32) {
            float o[32];
            tmem_ld32(O + c, o);
            uint32_t r[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(o[j] * f);
            tmem_st32(O + c, r);
          }
        }
      }
      const float mm = m == -INFINITY ? 0.0f : m;
      float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < 4; c += 2) {
        uint32_t r[32];
#pragma unroll
        for (int d = 0; d < 2; ++d)
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const float p0 = attn::ex2((CAP || BIAS) ? v[c + d][j] - mm : fmaf(v[c + d][j], c2, -mm));
            const float p1 = attn::ex2((CAP || BIAS) ? v[c + d][j + 1] - mm : fmaf(v[c + d][j + 1], c2, -mm));
            part[2 * d] += p0;
            part[2 * d + 1] += p1;
            r[d * 16 + j / 2] = pack_bf16x2(p0, p1);
          }
        tmem_st32(S + c * 16, r);
      }
      sum += (part[0] + part[1]) + (part[2] + part[3]);
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(bar_p(hf));
    }
    if (ok && n_own > 0) ok = mbar_wait(bar_s(hf), (uint32_t)n_own & 1u, abort_flag, a.status, kTimeoutSeqAttn);
    if (ok) ok = mbar_wait(bar_q, 0, abort_flag, a.status, kTimeoutSeqAttn);       // Q's tile takes the output
    if (ok) {
      tc_fence_after();
      const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
      uint8_t* out = gen + hf * C::TILE;
#pragma unroll 1
      for (int c = 0; c < DHP / 32; ++c) {
        float o[32];
        if (n_own > 0) tmem_ld32(O + c * 32, o);
#pragma unroll
        for (int j = 0; j < 32; ++j) o[j] = n_own > 0 ? o[j] * inv : 0.0f;
        sts_row32(out + (c >> 1) * CHUNK, trow, c & 1, o);
      }
      if (row < a.mask.M) a.lse[(size_t)h * a.ld + row] = sum > 0.0f || sum != sum ? m + log2f(sum) : INFINITY;
      fence_async_smem();
      group_sync(1 + hf);
      if (trow == 0) {
        for (int c = 0; c < C::CH; ++c)
          if (c * 64 < a.dim && row < a.mask.M) tma_store_3d(&map_out, base + hf * C::TILE + c * CHUNK, c * 64, h, row);
        tma_store_commit();
        tma_store_wait_all();
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
  }
}

// ---- backward ----------------------------------------------------------------------------------
// D_i = dO_i . o_i per head: 16 lanes a row and head, 8 columns a lane.
static __global__ void __launch_bounds__(256)
dot_kernel(const bf16* __restrict__ out, const bf16* __restrict__ dout, float* __restrict__ D, int M, int heads, int dim, int ld) {
  chain_begin();
  const long long item = ((long long)blockIdx.x * 256 + threadIdx.x) / 16;
  const int sub = threadIdx.x & 15;
  const bool on = item < (long long)M * heads;
  float s = 0.0f;
  if (on && sub * 8 < dim) {
    const size_t at = (size_t)item * dim + sub * 8;               // rows hold the heads side by side: item = row * heads + head
    float o[8], g[8];
    load_seg<8>(out + at, 8, o);
    load_seg<8>(dout + at, 8, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(o[i], g[i], s);
  }
#pragma unroll
  for (int k = 8; k > 0; k >>= 1) s += __shfl_xor_sync(0xffffffffu, s, k);
  if (on && sub == 0) D[(size_t)(item % heads) * ld + item / heads] = s;
}

template <int DHP>
struct BwdCfg {
  static constexpr int CH = DHP / 64;
  static constexpr uint32_t TILE = CH * CHUNK;                   // resident, 128 rows
  static constexpr uint32_t HALF = CH * HCHUNK;                  // streamed, 64 rows
  static constexpr uint32_t STAGE = 2 * HALF + 1024;             // two tiles, the rows' lse and D
  static constexpr int ST = DHP == 128 ? 4 : 6;
  static constexpr uint32_t SMEM = 2 * TILE + ST * STAGE + 1024 + 256;
};

// DKV = false: X1 = q, X2 = dO (rows of head h), Y1 = k, Y2 = v;  acc1 = dq.
// DKV = true:  X1 = k, X2 = v (keys of a key head), Y1 = q, Y2 = dO of every head of its group;  acc1 = dk, acc2 = dv.
template <int DHP, bool DKV, bool CAP, bool BIAS>
__global__ void __launch_bounds__(THREADS, 1)
backward_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_xg,
                const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_yg,
                const __grid_constant__ CUtensorMap map_out, const Args a) {
  using C = BwdCfg<DHP>;
  constexpr int ST = C::ST;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t ring = base + 2 * C::TILE, bars = ring + ST * C::STAGE;
  const uint32_t bar_x = bars, bar_done = bars + 8;
  auto bar_s = [&](int w) { return bars + 16u + 8u * w; };        // S and dP of the tile that group w works on
  auto bar_p = [&](int w) { return bars + 32u + 8u * w; };        // P and dS are in tensor memory
  auto full = [&](int s) { return bars + 48u + 8u * s; };
  auto empty = [&](int s) { return bars + 48u + 8u * (ST + s); };
  int* shared = reinterpret_cast<int*>(gen + 2 * C::TILE + ST * C::STAGE + 160);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(shared);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  int* extent = shared + 2;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int blocks_h = DKV ? a.kv : a.heads, group = a.heads / a.kv;
  const int tiles = (a.mask.M + 127) / 128;
  const int h = blockIdx.x % blocks_h;                            // head, or key head
  const int tile = a.mask.causal && !DKV ? tiles - 1 - (int)(blockIdx.x / blocks_h) : (int)(blockIdx.x / blocks_h);
  const int row0 = tile * 128;

  if (threadIdx.x == 0) {
    prefetch_tmap(&map_x); prefetch_tmap(&map_xg); prefetch_tmap(&map_y); prefetch_tmap(&map_yg); prefetch_tmap(&map_out);
    mbar_init(bar_x, 1);
    mbar_init(bar_done, 1);
    for (int i = 0; i < 2; ++i) { mbar_init(bar_s(i), 1); mbar_init(bar_p(i), 128); }
    for (int s = 0; s < ST; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    extent[0] = 0x7fffffff; extent[1] = 0;
    *abort_flag = 0;
    fence_async_smem();
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)tmem_slot)), "r"(TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  chain_begin();
  if (warp == 9 && lane == 0) {
    mbar_expect_tx(bar_x, 2 * C::TILE);
    for (int c = 0; c < C::CH; ++c) {
      tma_load_3d(base + c * CHUNK, &map_x, bar_x, c * 64, DKV ? a.heads + h : h, row0);
      if (DKV) tma_load_3d(base + C::TILE + c * CHUNK, &map_x, bar_x, c * 64, a.heads + a.kv + h, row0);
      else tma_load_3d(base + C::TILE + c * CHUNK, &map_xg, bar_x, c * 64, h, row0);
    }
  }
  int2 iv = make_int2(0, 0);
  if (warp < 8) {
    iv = interval<DKV>(a.mask, row0 + (int)(threadIdx.x & 127), lane);
    if (warp < 4) note_extent(extent, extent + 1, iv);
  }
  __syncthreads();
  const int T0 = extent[1] > extent[0] ? extent[0] / STREAM : 0;
  const int n_tiles = extent[1] > extent[0] ? (extent[1] + STREAM - 1) / STREAM - T0 : 0;
  const int total = DKV ? n_tiles * group : n_tiles;

  if (warp == 9) {
    if (lane == 0) {
      bool ok = true;
      int fills = 0;
      int g = 0, t = 0;
      for (int i = 0; i < total && ok; ++i) {
        const int s = i % ST;
        ok = mbar_wait(empty(s), ((uint32_t)(i / ST) & 1u) ^ 1u, abort_flag, a.status, kTimeoutSeqAttn);
        if (!ok) break;
        const uint32_t dst = ring + s * C::STAGE;
        const int r = (T0 + t) * STREAM;
        mbar_expect_tx(full(s), 2 * C::HALF + (DKV ? 2u * STREAM * 4u : 0u));
        for (int c = 0; c < C::CH; ++c) {
          if (DKV) {
            tma_load_3d(dst + c * HCHUNK, &map_y, full(s), c * 64, h * group + g, r);
            tma_load_3d(dst + C::HALF + c * HCHUNK, &map_yg, full(s), c * 64, h * group + g, r);
          } else {
            tma_load_3d(dst + c * HCHUNK, &map_y, full(s), c * 64, a.heads + h / group, r);
            tma_load_3d(dst + C::HALF + c * HCHUNK, &map_y, full(s), c * 64, a.heads + a.kv + h / group, r);
          }
        }
        if (DKV) {
          const size_t at = (size_t)(h * group + g) * a.ld + r;
          bulk_load(dst + 2 * C::HALF, a.lse + at, STREAM * 4, full(s));
          bulk_load(dst + 2 * C::HALF + STREAM * 4, a.D + at, STREAM * 4, full(s));
        }
        ++fills;
        if (++t == n_tiles) { t = 0; ++g; }
      }
      if (!ok) {
        for (int i = max(0, fills - ST); i < fills; ++i)
          for (uint32_t it = 0; it < (1u << 20) && !mbar_try_wait(full(i % ST), (uint32_t)(i / ST) & 1u); ++it) {}
      }
      for (uint32_t it = 0; it < (1u << 20) && !mbar_try_wait(bar_x, 0); ++it) {}
    }
  } else if (warp == 8) {
    const uint32_t id_s = attn::idesc128(STREAM, false, false), id_a = attn::idesc128(DHP, false, true);
    const int2 used = used_rows(a.mask);
    bool ok = total == 0 || __all_sync(0xffffffffu, mbar_wait(bar_x, 0, abort_flag, a.status, kTimeoutSeqAttn));
    int t = 0;
    for (int i = 0; i <= total && ok; ++i) {
      if (i < total) {
        const int s = i % ST;
        ok = __all_sync(0xffffffffu, mbar_wait(full(s), (uint32_t)(i / ST) & 1u, abort_flag, a.status, kTimeoutSeqAttn));
        if (!ok) break;
        const int r = (T0 + t) * STREAM;
        if (r < used.x || r + STREAM > used.y) {
          scrub(gen + 2 * C::TILE + s * C::STAGE, STREAM, 2 * C::CH, HCHUNK, r, used, lane);
          fence_async_smem();
          __syncwarp();
        }
        tc_fence_after();
        if (lane == 0) {
          const uint32_t S = tmem + 256 + (i & 1) * 128, y = ring + s * C::STAGE;
          for (int ks = 0; ks < DHP / UK; ++ks) tc_mma(S, kdesc(base, ks, CHUNK), kdesc(y, ks, HCHUNK), id_s, ks > 0 ? 1u : 0u);
          for (int ks = 0; ks < DHP / UK; ++ks)
            tc_mma(S + 64, kdesc(base + C::TILE, ks, CHUNK), kdesc(y + C::HALF, ks, HCHUNK), id_s, ks > 0 ? 1u : 0u);
          tc_commit(bar_s(i & 1));
        }
        __syncwarp();
        if (++t == n_tiles) t = 0;
      }
      if (i >= 1) {
        const int p = i - 1;
        ok = __all_sync(0xffffffffu, mbar_wait(bar_p(p & 1), (uint32_t)(p >> 1) & 1u, abort_flag, a.status, kTimeoutSeqAttn));
        if (!ok) break;
        tc_fence_after();
        if (lane == 0) {
          const uint32_t S = tmem + 256 + (p & 1) * 128, y = ring + (p % ST) * C::STAGE;
          if (DKV)
            for (int ks = 0; ks < STREAM / UK; ++ks)
              mma_ts(tmem + DHP, S + ks * 8, mndesc(y + C::HALF, ks, HCHUNK), id_a, (p > 0 || ks > 0) ? 1u : 0u);
          for (int ks = 0; ks < STREAM / UK; ++ks)
            mma_ts(tmem, S + 64 + ks * 8, mndesc(y, ks, HCHUNK), id_a, (p > 0 || ks > 0) ? 1u : 0u);
          tc_commit(empty(p % ST));
        }
        __syncwarp();
      }
    }
    if (ok && total > 0 && lane == 0) tc_commit(bar_done);
    __syncwarp();
  } else {
    const int w = warp >> 2;
    const int trow = threadIdx.x & 127, row = row0 + trow;
    const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t S = tmem + lane_addr + 256 + w * 128;
    const float c2 = a.scale * LOG2E;
    const float u = CAP ? 2.0f * c2 / a.cap : 0.0f, top = a.cap * LOG2E;
    float own_lse = INFINITY, own_D = 0.0f, slope2 = 0.0f;
    if (!DKV) {
      if (row < a.mask.M) { own_lse = a.lse[(size_t)h * a.ld + row]; own_D = a.D[(size_t)h * a.ld + row]; }
      if (BIAS) slope2 = a.slopes[h] * LOG2E;
    }
    bool ok = true;
    for (int i = w; i < total && ok; i += 2) {
      const int t = DKV ? i % n_tiles : i;
      const int k0 = (T0 + t) * STREAM;
      if (DKV && BIAS) slope2 = a.slopes[h * group + i / n_tiles] * LOG2E;
      ok = mbar_wait(bar_s(w), (uint32_t)(i >> 1) & 1u, abort_flag, a.status, kTimeoutSeqAttn);
      if (!ok) break;
      if (DKV) {                                                  // the rows' lse and D came with the tile
        ok = mbar_wait(full(i % ST), (uint32_t)(i / ST) & 1u, abort_flag, a.status, kTimeoutSeqAttn);
        if (!ok) break;
      }
      tc_fence_after();
      const float* col = reinterpret_cast<const float*>(gen + 2 * C::TILE + (i % ST) * C::STAGE + 2 * C::HALF);
      const bool whole = __all_sync(0xffffffffu, iv.x <= k0 && iv.y >= k0 + STREAM);
      const int lo = iv.x - k0;
      const unsigned len = (unsigned)(iv.y - iv.x);
      const float d0 = (float)(row - k0);
      uint32_t pr[32], dr[32];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float s[32], dp[32];
        tmem_ld32_issue(S + c * 32, s);
        tmem_ld32_issue(S + 64 + c * 32, dp);
        tmem_ld_wait(s, dp);
#pragma unroll
        for (int q = 0; q < 32; q += 4) {
          float4 L4 = make_float4(own_lse, own_lse, own_lse, own_lse), D4 = make_float4(own_D, own_D, own_D, own_D);
          if (DKV) {
            L4 = *reinterpret_cast<const float4*>(col + c * 32 + q);
            D4 = *reinterpret_cast<const float4*>(col + STREAM + c * 32 + q);
          }
          const float Lv[4] = {L4.x, L4.y, L4.z, L4.w}, Dv[4] = {D4.x, D4.y, D4.z, D4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = q + e;
            float x, slope = 1.0f;
            if (CAP) {
              const float th = tanh_of(s[j] * u);
              slope = fmaf(-th, th, 1.0f);
              x = fmaf(top, th, -Lv[e]);
            } else {
              x = fmaf(s[j], c2, -Lv[e]);
            }
            if (BIAS) x = fmaf(-slope2, fabsf(d0 - (float)(c * 32 + j)), x);
            float p = attn::ex2(x);
            float ds = p * (dp[j] - Dv[e]);
            if (CAP) ds *= slope;
            if (!whole && (unsigned)(c * 32 + j - lo) >= len) { p = 0.0f; ds = 0.0f; }
            s[j] = p;
            dp[j] = ds;
          }
        }
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
          if (DKV) pr[c * 16 + j / 2] = pack_bf16x2(s[j], s[j + 1]);
          dr[c * 16 + j / 2] = pack_bf16x2(dp[j], dp[j + 1]);
        }
      }
      if (DKV) tmem_st32(S, pr);
      tmem_st32(S + 64, dr);
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(bar_p(w));
    }
    if (ok && total > 0) ok = mbar_wait(bar_done, 0, abort_flag, a.status, kTimeoutSeqAttn);
    if (ok) ok = mbar_wait(bar_x, 0, abort_flag, a.status, kTimeoutSeqAttn);
    if (ok) {
      tc_fence_after();
      // dk and dq are staged in X1's tile, dv in X2's.  dk, dv: a group each; dq: the groups share its 64-column pieces
      const int c0 = DKV ? 0 : w, c1 = DKV ? C::CH : min(w + 1, C::CH);
      const bool second = DKV && w == 1;
      const float f = second ? 1.0f : a.scale;
      uint8_t* out = gen + (second ? C::TILE : 0);
      const int block = DKV ? a.heads + (w == 1 ? a.kv : 0) + h : h;
#pragma unroll 1
      for (int c = c0 * 2; c < c1 * 2; ++c) {
        float o[32];
        if (total > 0) tmem_ld32(tmem + lane_addr + (second ? DHP : 0) + c * 32, o);
#pragma unroll
        for (int j = 0; j < 32; ++j) o[j] = total > 0 ? o[j] * f : 0.0f;
        sts_row32(out + (c >> 1) * CHUNK, trow, c & 1, o);
      }
      fence_async_smem();
      group_sync(1 + w);
      if (trow == 0) {
        for (int c = c0; c < c1; ++c)
          if (c * 64 < a.dim) tma_store_3d(&map_out, base + (second ? C::TILE : 0) + c * CHUNK, c * 64, block, row0);
        tma_store_commit();
        tma_store_wait_all();
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
  }
}

}  // namespace seqattn
}  // namespace et
