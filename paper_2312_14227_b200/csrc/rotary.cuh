// Rotary positions with one to three axes (ET_LAYER_ROTARY).  Of every query and key head the first 2 R columns are R pairs;
// pair k turns by the angle  position[axis(k)] * f(k):   (x, y) -> (x cos - y sin, y cos + x sin).  The gradient turns back.
//
// Positions are whole numbers, so the angle in turns, position * f / 2 pi, is only needed modulo 1: the host rounds f / 2 pi to a
// 64-bit binary fraction, and the low 64 bits of the integer product are the fraction of a turn, exact to position * 2^-65,
// however far the position.  No table of angles is read.
//
// Bound by HBM: in place (inside a stack) the rotated heads are read and written once, else the whole row.  A thread turns 8
// columns (16 or 32 bytes) of every head of its row with one set of cosines and sines; the heads are cut over blockIdx.y
// where the rows alone would leave the GPU short of warps.  Heads go four (fp32: two) at a time, their loads in flight together: 32760 rows of
// 16 + 16 + 16 heads of 128 in bf16, not in place, 135 us = 6.0 TB/s (a head at a time: 206 us).
#pragma once

#include "dropout.cuh"

namespace et {

constexpr int kRotaryMaxPairs = 128;
struct RotaryTable {
  uint64_t turn[kRotaryMaxPairs];      // f / 2 pi as a fraction of 2^64
  uint8_t axis[kRotaryMaxPairs];
};
struct RotaryArgs {
  const int32_t* positions;            // [axes][M] or nullptr: the row's number modulo `len`
  long long M;
  int len, dim, pairs, heads, all;     // heads turned; all: blocks of `dim` columns in a row
  bool adjacent, copy, back;           // copy: columns that are not turned are written, too; back: the other way
};

__device__ __forceinline__ void turn_of(uint64_t f, int position, bool back, float* c, float* s) {
  const uint64_t frac = (uint64_t)(int64_t)position * f;
  // signed fraction of a half turn, [-1, 1): 24 bits of it, an error of 2^-24 pi / 2 at most, that of an fp32 angle near pi
  sincospif((float)(int32_t)(uint32_t)(frac >> 32) * 4.656612873077393e-10f, s, c);
  if (back) *s = -*s;
}

template <typename T> __device__ __forceinline__ void copy_chunk(T* p, const RawChunk<T>& r) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = r.q[i];
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(256)
rotary_kernel(const T* in, T* out, const __grid_constant__ RotaryTable tab, const RotaryArgs a) {
  chain_begin();
  constexpr int V = VEC ? 8 : 1;
  // a thread's columns: halves: V pairs, their first columns at k and their second at pairs + k; adjacent: V / 2 (or 1) pairs
  const int per_pair = a.adjacent ? (VEC ? 4 : 1) : V;
  const int slots = (a.pairs + per_pair - 1) / per_pair;
  const long long item = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  const long long row = item / slots;
  if (row >= a.M) return;
  const int k = (int)(item - row * slots) * per_pair;
  float c[V], s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (i >= per_pair) break;
    const int axis = tab.axis[k + i];
    const int p = a.positions != nullptr ? a.positions[axis * a.M + row] : (int)(row % a.len);
    turn_of(tab.turn[k + i], p, a.back, &c[i], &s[i]);
  }
  const size_t at = (size_t)row * a.all * a.dim;
  const int step = gridDim.y;
  constexpr int B = VEC ? 16 / (int)sizeof(T) / 2 : 1;              // heads at a time: 4 of bf16, 2 of fp32, loads in flight together
  for (int h0 = blockIdx.y; h0 < a.heads; h0 += B * step) {
    if (VEC) {
      RawChunk<T> p0[B], p1[B];
      const int second = a.adjacent ? 0 : a.pairs, from = a.adjacent ? 2 * k : k;
#pragma unroll
      for (int i = 0; i < B; ++i) {
        const int h = h0 + i * step;
        if (h >= a.heads) break;
        const T* p = in + at + (size_t)h * a.dim + from;
        p0[i] = load_chunk(p);
        if (!a.adjacent) p1[i] = load_chunk(p + second);
      }
#pragma unroll
      for (int i = 0; i < B; ++i) {
        const int h = h0 + i * step;
        if (h >= a.heads) break;
        T* p = out + at + (size_t)h * a.dim + from;
        float x[8], y[8];
        raw_unpack(p0[i], x);
        if (a.adjacent) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            y[2 * j] = x[2 * j] * c[j] - x[2 * j + 1] * s[j];
            y[2 * j + 1] = x[2 * j + 1] * c[j] + x[2 * j] * s[j];
          }
          store_chunk(p, y);
        } else {
          raw_unpack(p1[i], y);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float u = x[j] * c[j] - y[j] * s[j];
            y[j] = y[j] * c[j] + x[j] * s[j];
            x[j] = u;
          }
          store_chunk(p, x);
          store_chunk(p + second, y);
        }
      }
    } else {
      const size_t o = at + (size_t)h0 * a.dim, i0 = a.adjacent ? o + 2 * k : o + k, i1 = a.adjacent ? i0 + 1 : i0 + a.pairs;
      const float x = to_f32(in[i0]), y = to_f32(in[i1]);
      out[i0] = from_f32<T>(x * c[0] - y * s[0]);
      out[i1] = from_f32<T>(y * c[0] + x * s[0]);
    }
  }
  if (!a.copy) return;
  // the rest of the turned heads, and the heads that are not turned: one run of the row's last columns
  const int slot = k / per_pair, rest = a.dim - 2 * a.pairs;
  for (int h = blockIdx.y; h < a.heads && rest > 0; h += step)
    for (int j = slot * V; j < rest; j += slots * V) {
      const size_t o = at + (size_t)h * a.dim + 2 * a.pairs + j;
      if (VEC) copy_chunk(out + o, load_chunk(in + o));
      else out[o] = in[o];
    }
  const int tail = (a.all - a.heads) * a.dim, stride = slots * V * step;
  const size_t o = at + (size_t)a.heads * a.dim;
  for (int j0 = (blockIdx.y * slots + slot) * V; j0 < tail; j0 += 4 * stride) {
    if (VEC) {
      RawChunk<T> x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (j0 + i * stride < tail) x[i] = load_chunk(in + o + j0 + i * stride);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (j0 + i * stride < tail) copy_chunk(out + o + j0 + i * stride, x[i]);
    } else {
      for (int i = 0; i < 4; ++i)
        if (j0 + i * stride < tail) out[o + j0 + i * stride] = in[o + j0 + i * stride];
    }
  }
}

}  // namespace et
