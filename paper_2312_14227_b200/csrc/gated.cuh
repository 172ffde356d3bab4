// Gated layer (ET_LAYER_GATED):  Z = a W + b,  W = [gate | up] of 2 h columns,  out = act(Z_gate) * Z_up.
//
// Forward on the tensor cores: one kernel forms both projections, the activation and the product.  A pair of CTAs (cta_group::2)
// works on 256 rows x H columns of the output: CTA 0 of the pair loads the H gate columns of W, CTA 1 the H up columns, and the
// pair's accumulator holds gate and up of one output column H columns apart in the same thread's row: the product needs no
// exchange.  Same ring and hand-over of accumulators as gemm_tc_kernel (tcgen05 in tensor memory, two accumulator stages, TMA).  The
// epilogue's two groups stage Z_gate, Z_up and the product in 128 x 64 chunks for TMA stores (Z is what the backward pass needs).
// Tensor-bound like the dense layer of 2 h columns; the epilogue writes 6 bytes an output.
// H = 128 (256 columns of accumulator); 64 where 128-wide tiles would leave CTA pairs without work.
//
// Backward: dZ_gate = g Z_up act'(Z_gate), dZ_up = g act(Z_gate).  Below a dense or gated layer they are formed in the epilogue of that layer's
// error-gradient product, from its accumulator (GatedDgradEpi): g is neither rounded nor stored, and the bias sums come with it.  Elsewhere
// one pass over g and Z forms them (gated_backward_kernel).  The error gradient dZ W^T and the weight gradient a^T dZ are those of a
// dense layer with 2 h columns.
//
// Rounding: the product and dZ are bf16, as what a dense layer stores.  Z of a bf16 stack is kept in fp16: the gradient is read off values
// of Z, and their 2^-11 leaves dZ's own rounding as the only one that counts (error of dX against 64 bits 2.4e-3 instead of 3.4e-3, of which the last
// rounding alone is 1.7e-3).  Z beyond 65504 is kept as 65504; the product is formed before that, from fp32.  Below 2^-14 the steps of fp16 are 2^-24
// whatever the value: a factor of dZ is then off by up to 2^-25, the smaller Z the more of it (3 % at 1e-6, all of it below 2^-25).  A ReLU's slope
// jumps there: a gate above 0 is kept above 0.
#pragma once

#include <type_traits>

#include "dropout.cuh"
#include "gemm_tc.cuh"

namespace et {

constexpr int kActSilu = 3;
constexpr float kLeastZ = 5.9604644775390625e-8f;                   // 2^-24, the smallest number of fp16

// T: storage type.  bf16 stacks take the exponential and reciprocal units' own results (2^-22, far below a bf16 step; an exponential beyond fp32
// gives 0), fp32 stacks expf and a true quotient.
template <typename T> __device__ __forceinline__ float sigmoid_of(float z);
template <> __device__ __forceinline__ float sigmoid_of<bf16>(float z) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e + 1.0f));
  return r;
}
template <> __device__ __forceinline__ float sigmoid_of<float>(float z) { return 1.0f / (1.0f + expf(-z)); }
template <typename T>
__device__ __forceinline__ float gate_apply(float z, int act) {
  return act == kActSilu ? z * sigmoid_of<T>(z) : act_apply(z, act);
}
// value and slope
template <typename T>
__device__ __forceinline__ float2 gate_both(float z, int act) {
  if (act == kActSilu) {
    const float g = sigmoid_of<T>(z), f = z * g;
    return make_float2(f, fmaf(f, 1.0f - g, g));                    // g + z g (1 - g)
  }
  return make_float2(act_apply(z, act), act_grad(z, act));
}

// fp16 as Z is kept: held at the largest finite value, NaN stays NaN
__device__ __forceinline__ uint32_t pack_z(float a, float b) {
  asm("min.NaN.f32 %0, %0, 0f477FE000;\n\tmax.NaN.f32 %0, %0, 0fC77FE000;" : "+f"(a));
  asm("min.NaN.f32 %0, %0, 0f477FE000;\n\tmax.NaN.f32 %0, %0, 0fC77FE000;" : "+f"(b));
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void unpack_z(const uint4& q, float (&t)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    t[2 * i] = f.x;
    t[2 * i + 1] = f.y;
  }
}

// Epilogue of the error-gradient product above a gated layer.  slot 0: in Z_gate, out dZ_gate; slot 1: in Z_up, out dZ_up.
struct GatedDgradEpi {
  static constexpr int kSlots = 2;
  bool has_in[2], has_out[2];
  int act;
  float* colsum;     // [row blocks of 32][2 h] or nullptr
  int h;

  __device__ __forceinline__ void combine(int, int, float (&v)[32], float (&s0)[32], float (&s1)[32]) const {
    auto all = [&](auto kind) {                                     // one test for 32 values
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const float2 f = gate_both<bf16>(s0[i], decltype(kind)::value);
        s0[i] = v[i] * s1[i] * f.y;
        s1[i] = v[i] * f.x;
      }
    };
    if (act == kActSilu) all(std::integral_constant<int, kActSilu>());
    else if (act == kActGelu) all(std::integral_constant<int, kActGelu>());
    else all(std::integral_constant<int, kActRelu>());
  }
  __device__ __forceinline__ void column_sums(int row_block, int col0, int nv, float (&s0)[32], float (&s1)[32], int lane) const {
    if (colsum == nullptr) return;
    warp_column_sums(s0, lane);
    warp_column_sums(s1, lane);
    if (lane < nv) {
      float* out = colsum + (size_t)row_block * 2 * h + col0 + lane;
      out[0] = s0[0];
      out[h] = s1[0];
    }
  }
};
template <> struct tc::EpiHalfIn<GatedDgradEpi> { static constexpr bool value = true; };

namespace gated {

using namespace et::tc;

__device__ __forceinline__ bool group_all(int id, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 q, %2, 0;\n\t"
      "barrier.cta.red.and.pred p, %1, 128, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r) : "r"(id), "r"((uint32_t)x) : "memory");
  return r != 0;
}
__device__ __forceinline__ void sts_z32(uint8_t* chunk, int row, int half, const float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *reinterpret_cast<uint4*>(chunk + epi_chunk_off(row, half * 4 + j)) =
        make_uint4(pack_z(v[j * 8], v[j * 8 + 1]), pack_z(v[j * 8 + 2], v[j * 8 + 3]), pack_z(v[j * 8 + 4], v[j * 8 + 5]), pack_z(v[j * 8 + 6], v[j * 8 + 7]));
}

template <int H>
struct Cfg {
  static constexpr int BN = 2 * H;
  static constexpr uint32_t B_BYTES = H * BK * 2;                // this CTA's half: gate or up
  static constexpr uint32_t STAGE = A_STAGE_BYTES + B_BYTES;
  static constexpr uint32_t EPI = EPI_GROUPS * 3 * EPI_CHUNK_BYTES;
  static constexpr int STAGES = H == 128 ? 4 : 5;
  static constexpr uint32_t SMEM = STAGES * STAGE + EPI + SMEM_SLACK;
  static_assert(SMEM <= SMEM_LIMIT, "shared memory");
};
struct Params {
  int rows, h, kb;           // rows, output columns, 64-deep blocks of the contraction
  int tiles_m, tiles_n;
  int b_3d;                  // W's halves by one 3-D copy a stage (h a multiple of 64)
  int act;
  const bf16* bias;          // [2 h]
  uint32_t* status;
};
struct Maps {
  CUtensorMap a;             // input, 64 columns x 128 rows
  CUtensorMap w[2];          // gate, up
  CUtensorMap out[3];        // Z_gate, Z_up, product: 64 x 128
};
constexpr int THREADS = 320; // warp 0: TMA, warp 1: MMA + TMEM, warps 2-9: two epilogue groups

template <int H>
__global__ void __launch_bounds__(THREADS, 1) __cluster_dims__(2, 1, 1)
gated_forward_kernel(const __grid_constant__ Maps maps, const Params p) {
  using C = Cfg<H>;
  constexpr int STAGES = C::STAGES;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  const int unit0 = blockIdx.x >> 1, unit_step = gridDim.x >> 1;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t epi_base = base + STAGES * C::STAGE, bars = epi_base + C::EPI;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (STAGES + s); };
  auto acc_full = [&](int s) { return bars + 8u * (2 * STAGES + s); };
  auto acc_empty = [&](int s) { return bars + 8u * (2 * STAGES + 2 + s); };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + STAGES * C::STAGE + C::EPI + 8 * (2 * STAGES + 4));
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    prefetch_tmap(&maps.a);
    prefetch_tmap(&maps.w[rank]);
    for (int i = 0; i < 3; ++i) prefetch_tmap(&maps.out[i]);
    for (int s = 0; s < STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(acc_full(s), 1); mbar_init(acc_empty(s), 16); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)tmem_slot)), "r"(TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  chain_begin();
  const int units = p.tiles_m * p.tiles_n;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t fills[STAGES];
#pragma unroll
      for (int s = 0; s < STAGES; ++s) fills[s] = 0;
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int u = unit0; u < units && ok; u += unit_step) {
        const int m0 = u / p.tiles_n * 2 * BM + (int)rank * BM, n0 = u % p.tiles_n * H;
        for (int kb = 0; kb < p.kb; ++kb) {
          ok = mbar_wait(empty(stage), phase ^ 1u, abort_flag, p.status, kTimeoutProducer);
          if (!ok) break;
          const uint32_t sa = base + stage * C::STAGE, sb = sa + A_STAGE_BYTES, bar = full(stage);
          if (leader) mbar_expect_tx(bar, 2u * C::STAGE);        // both CTAs' copies report to CTA 0
          tma_load_2d_pair(sa, &maps.a, bar, kb * BK, m0);
          if (p.b_3d) tma_load_3d_pair(sb, &maps.w[rank], bar, 0, kb * BK, n0 >> 6);
          else
            for (int c = 0; c < H / 64; ++c) tma_load_2d_pair(sb + c * CHUNK_BYTES, &maps.w[rank], bar, n0 + c * 64, kb * BK);
          ++fills[stage];
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) {
        if (leader) {
#pragma unroll
          for (int s = 0; s < STAGES; ++s) {
            if (fills[s] == 0) continue;
            bool landed = false;
            for (uint32_t it = 0; it < (1u << 20) && !landed; ++it) landed = mbar_try_wait(full(s), (fills[s] - 1u) & 1u);
            if (!landed) atomicCAS(p.status, 0u, (uint32_t)kTimeoutDrain);
          }
        } else {
          for (int it = 0; it < 2000; ++it) __nanosleep(1000);
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && leader) {
      constexpr uint32_t idesc = make_idesc<2 * BM, C::BN, false, true>();
      const uint64_t desc_a = make_desc(base, 16, 1024), desc_b = make_desc(base + A_STAGE_BYTES, CHUNK_BYTES, 1024);
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      for (int u = unit0; u < units && ok; u += unit_step) {
        ok = mbar_wait(acc_empty(acc), acc_phase ^ 1u, abort_flag, p.status, kTimeoutMma);
        if (!ok) break;
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)(acc * ACC_STRIDE);
        for (int kb = 0; kb < p.kb; ++kb) {
          ok = mbar_wait(full(stage), phase, abort_flag, p.status, kTimeoutMma);
          if (!ok) break;
          tc_fence_after();
          const uint64_t da = desc_a + (uint64_t)((uint32_t)stage * (C::STAGE >> 4)), db = desc_b + (uint64_t)((uint32_t)stage * (C::STAGE >> 4));
#pragma unroll
          for (int k = 0; k < BK / UK; ++k) tc_mma_pair(d, da + k * (32u >> 4), db + k * (2048u >> 4), idesc, (kb > 0 || k > 0) ? 1u : 0u);
          tc_commit_pair(empty(stage));
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        tc_commit_pair(acc_full(acc));
        if (++acc == ACC_STAGES) { acc = 0; acc_phase ^= 1u; }
      }
    }
  } else {
    constexpr int NCH = H / 64;                     // output chunks of 64 columns in a tile
    const int g = (warp - 2) >> 2, quad = warp & 3, trow = quad * 32 + lane;
    const bool store_thread = (threadIdx.x - 64) % 128 == 0;
    uint8_t* buf = gen + STAGES * C::STAGE + g * 3 * EPI_CHUNK_BYTES;
    const uint32_t src = epi_base + (uint32_t)g * 3u * EPI_CHUNK_BYTES;
    int acc = 0, it = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int u = unit0; u < units && ok; u += unit_step, ++it) {
      const int m0 = u / p.tiles_n * 2 * BM + (int)rank * BM, n0 = u % p.tiles_n * H;
      // the group goes on together or not at all: its barriers below count on all 128 threads
      ok = group_all(1 + g, mbar_wait(acc_full(acc), acc_phase, abort_flag, p.status, kTimeoutEpilogue));
      if (!ok) break;
      tc_fence_after();
      const uint32_t taddr = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(acc * ACC_STRIDE);
      const int c = NCH == 2 ? g : 0;               // this group's chunk; with one chunk a tile the groups take turns
      const int col0 = n0 + c * 64;
      const bool mine = (NCH == 2 || (it & 1) == g) && col0 < p.h;
      if (mine) {
        if (store_thread) tma_store_wait_read<0>(); // the last chunk's stores have read the buffers
        asm volatile("bar.sync %0, 128;" ::"r"(1 + g) : "memory");
#pragma unroll 1
        for (int hf = 0; hf < 2; ++hf) {
          float zg[32], zu[32], t[32];
          tmem_ld32_issue(taddr + c * 64 + hf * 32, zg);
          tmem_ld32_issue(taddr + H + c * 64 + hf * 32, zu);
          tmem_ld_wait(zg, zu);
          if (hf == 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(acc_empty(acc), 0u);
          }
          const int col = col0 + hf * 32;
          load_seg<32>(p.bias + col, p.h - col, t);
#pragma unroll
          for (int i = 0; i < 32; ++i) zg[i] += t[i];
          load_seg<32>(p.bias + p.h + col, p.h - col, t);
#pragma unroll
          for (int i = 0; i < 32; ++i) zu[i] += t[i];
          sts_z32(buf + EPI_CHUNK_BYTES, trow, hf, zu);
          if (p.act == kActRelu) {                  // a positive gate keeps its slope: it stays positive as it is kept
            float kept[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) kept[i] = zg[i] > 0.0f ? fmaxf(zg[i], kLeastZ) : zg[i];
            sts_z32(buf, trow, hf, kept);
          } else {
            sts_z32(buf, trow, hf, zg);
          }
          if (p.act == kActSilu) {                  // one test for 32 values
#pragma unroll
            for (int i = 0; i < 32; ++i) zg[i] = gate_apply<bf16>(zg[i], kActSilu) * zu[i];
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) zg[i] = act_apply(zg[i], p.act) * zu[i];
          }
          sts_row32(buf + 2 * EPI_CHUNK_BYTES, trow, hf, zg);
        }
        fence_async_smem();
        asm volatile("bar.sync %0, 128;" ::"r"(1 + g) : "memory");
        if (store_thread) {
          if (m0 < p.rows)
            for (int i = 0; i < 3; ++i) tma_store_2d(&maps.out[i], src + (uint32_t)i * EPI_CHUNK_BYTES, col0, m0);
          tma_store_commit();
        }
      } else {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(acc_empty(acc), 0u);
      }
      if (++acc == ACC_STAGES) { acc = 0; acc_phase ^= 1u; }
    }
    if (store_thread) tma_store_wait_all();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
  }
}

}  // namespace gated

// fp32 stacks (FMA pipes): the tile of gemm_simt_kernel with two accumulators, gate and up.  32-row tiles: fp32 stacks are small.
constexpr int kGatedSimtM = 32, kGatedSimtN = 32, kGatedSimtK = 16;
static __global__ void __launch_bounds__(256)
gated_forward_simt_kernel(const float* __restrict__ A, const float* __restrict__ W, const float* __restrict__ bias, float* __restrict__ Z,
                          float* __restrict__ out, int M, int K, int h, int act) {
  __shared__ float As[kGatedSimtK][kGatedSimtM + 1], Bs[2][kGatedSimtK][kGatedSimtN];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;           // 16 x 16 threads, 2 x 2 outputs each
  const int i0 = row_block() * kGatedSimtM, j0 = blockIdx.x * kGatedSimtN;
  float acc[2][2][2] = {};
  for (int k0 = 0; k0 < K; k0 += kGatedSimtK) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int idx = threadIdx.x + e * 256, kk = idx & 15, ii = idx >> 4;
      As[kk][ii] = i0 + ii < M && k0 + kk < K ? A[(size_t)(i0 + ii) * K + k0 + kk] : 0.0f;
      const int jj = idx & 31, kb = idx >> 5;
      const bool in = j0 + jj < h && k0 + kb < K;
      const size_t at = (size_t)(k0 + kb) * 2 * h + j0 + jj;
      Bs[0][kb][jj] = in ? W[at] : 0.0f;
      Bs[1][kb][jj] = in ? W[at + h] : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < kGatedSimtK; ++kk)
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int w = 0; w < 2; ++w) acc[w][q][r] = fmaf(As[kk][ty * 2 + q], Bs[w][kk][tx * 2 + r], acc[w][q][r]);
    __syncthreads();
  }
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int i = i0 + ty * 2 + q, j = j0 + tx * 2 + r;
      if (i >= M || j >= h) continue;
      const float zg = acc[0][q][r] + bias[j], zu = acc[1][q][r] + bias[h + j];
      Z[(size_t)i * 2 * h + j] = zg;
      Z[(size_t)i * 2 * h + h + j] = zu;
      out[(size_t)i * h + j] = gate_apply<float>(zg, act) * zu;
    }
}

// dZ from g [M x h] and Z [M x 2 h]; a thread takes 8 columns of a row.
__device__ __forceinline__ void load_z(const float* Z, int n, float (&t)[8]) { load_seg<8>(Z, n, t); }
__device__ __forceinline__ void load_z(const bf16* Z, int, float (&t)[8]) { unpack_z(*reinterpret_cast<const uint4*>(Z), t); }   // h % 8 == 0: whole runs
template <typename T>
__device__ __forceinline__ void gated_backward_run(const T* g, const T* Z, T* dZ, size_t row, int h, int col, int n, int act, float (&a)[8], float (&b)[8]) {
  float v[8];
  const size_t at = row * 2 * h + col;
  load_seg<8>(g + row * h + col, n, v);
  load_z(Z + at, n, a);
  load_z(Z + at + h, n, b);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 f = gate_both<T>(a[i], act);
    a[i] = v[i] * b[i] * f.y;
    b[i] = v[i] * f.x;
  }
  store_seg<8>(dZ + at, n, a);
  store_seg<8>(dZ + at + h, n, b);
}
template <typename T>
__global__ void __launch_bounds__(256)
gated_backward_kernel(const T* __restrict__ g, const T* __restrict__ Z, T* __restrict__ dZ, long long M, int h, int act) {
  chain_begin();
  const int per_row = (h + 7) / 8;
  const long long item = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long row = item / per_row;
  if (row >= M) return;
  const int col = (int)(item - row * per_row) * 8;
  float a[8], b[8];
  gated_backward_run<T>(g, Z, dZ, (size_t)row, h, col, min(8, h - col), act, a, b);
}
// The same with the column sums of dZ over runs of kGatedRows rows in part[run][2 h]: the bias gradient without reading dZ again.  A block
// takes one run and 256 columns of each half, a thread four rows of eight columns, their loads in flight together; the rows' sums are
// joined in a fixed order.  8192 x 5632 in bf16: 83 us (without sums 77, and 52 for the pass that sums dZ columns).
constexpr int kGatedRows = 32;
template <typename T>
__global__ void __launch_bounds__(256)
gated_backward_sums_kernel(const T* __restrict__ g, const T* __restrict__ Z, T* __restrict__ dZ, float* __restrict__ part, long long M, int h, int act) {
  chain_begin();
  __shared__ float sums[8][2][256];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, run = row_block();
  if ((long long)run * kGatedRows >= M) return;
  const int col = blockIdx.x * 256 + lane * 8, n = min(8, h - col);
  const long long r0 = (long long)run * kGatedRows + w;
  float sa[8] = {}, sb[8] = {};
  if (n == 8 && h % 8 == 0) {
    constexpr int B = sizeof(T) == 2 ? 4 : 2;                       // rows in flight
#pragma unroll
    for (int r = 0; r < 4; r += B) {
      RawChunk<T> x[B], zg[B], zu[B];
#pragma unroll
      for (int i = 0; i < B; ++i) {
        const long long row = r0 + (r + i) * 8;
        if (row >= M) break;
        const size_t at = (size_t)row * 2 * h + col;
        x[i] = load_chunk(g + (size_t)row * h + col);
        zg[i] = load_chunk(Z + at);
        zu[i] = load_chunk(Z + at + h);
      }
#pragma unroll
      for (int i = 0; i < B; ++i) {
        const long long row = r0 + (r + i) * 8;
        if (row >= M) break;
        const size_t at = (size_t)row * 2 * h + col;
        float v[8], a[8], b[8];
        raw_unpack(x[i], v);
        if constexpr (sizeof(T) == 2) {
          unpack_z(zg[i].q[0], a);
          unpack_z(zu[i].q[0], b);
        } else {
          raw_unpack(zg[i], a);
          raw_unpack(zu[i], b);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 f = gate_both<T>(a[j], act);
          a[j] = v[j] * b[j] * f.y;
          b[j] = v[j] * f.x;
          sa[j] += a[j];
          sb[j] += b[j];
        }
        store_chunk(dZ + at, a);
        store_chunk(dZ + at + h, b);
      }
    }
  } else if (n > 0) {
    for (long long row = r0; row < min((long long)(run + 1) * kGatedRows, M); row += 8) {
      float a[8], b[8];
      gated_backward_run<T>(g, Z, dZ, (size_t)row, h, col, n, act, a, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) { sa[i] += a[i]; sb[i] += b[i]; }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) { sums[w][0][i * 32 + lane] = sa[i]; sums[w][1][i * 32 + lane] = sb[i]; }
  __syncthreads();
  const int c = blockIdx.x * 256 + threadIdx.x, at = (threadIdx.x & 7) * 32 + (threadIdx.x >> 3);
  if (c >= h) return;
  float s[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 8; ++i) { s[0] += sums[i][0][at]; s[1] += sums[i][1][at]; }
  float* out = part + (size_t)run * 2 * h + c;
  out[0] = s[0];
  out[h] = s[1];
}

}  // namespace et
