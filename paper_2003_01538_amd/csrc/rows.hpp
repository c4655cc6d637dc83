// Softmax statistics of a row of logits, for the operators that read rows of
// any length (log probabilities, distillation).
//
// m is the largest logit, at least the lowest finite number: a row of nothing
// but -inf then sums to 0 instead of NaN, and a finite lowest value (some
// masks) still counts.  s = sum e^((z - m) c) and t = sum e^((z - m) c) (z - m) are kept
// in fp32, c = 1 / temperature.
#pragma once

#include <float.h>
#include <math.h>

#include "common.hpp"
#include "device.hpp"

namespace fs {

constexpr int ROW_T = 256;  // threads of a workgroup

__device__ __forceinline__ float row_load(const float* p) { return *p; }
__device__ __forceinline__ float row_load(const uint16_t* p) { return bf2f(*p); }
__device__ __forceinline__ void row_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void row_store(uint16_t* p, float v) { *p = f2bf(v); }

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// Sum or maximum over the workgroup, the same in every thread; `sh` holds one
// value per wave and is free again after the call.
__device__ __forceinline__ float block_sum(float v, float* sh) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.f;
  for (int w = 0; w < ROW_T / 64; ++w) v += sh[w];
  __syncthreads();
  return v;
}
__device__ __forceinline__ float block_max(float v, float* sh) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = sh[0];
  for (int w = 1; w < ROW_T / 64; ++w) v = fmaxf(v, sh[w]);
  __syncthreads();
  return v;
}

// m, s, t of a row, in every thread
template <class T>
__device__ void row_stats(const T* z, int C, float c, float* sh, float& m, float& s, float& t) {
  float best = -FLT_MAX;
  for (int i = threadIdx.x; i < C; i += ROW_T) best = fmaxf(best, row_load(z + i));
  m = block_max(best, sh);
  s = t = 0.f;
  for (int i = threadIdx.x; i < C; i += ROW_T) {
    const float d = row_load(z + i) - m, e = expf(d * c);
    s += e;
    t += e > 0.f ? e * d : 0.f;
  }
  s = block_sum(s, sh);
  t = block_sum(t, sh);
}

}  // namespace fs
