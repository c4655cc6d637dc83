// Matrix product with bias, activation and residual on a caller's tensors:
// y[m][n] = act(sum_k x[m][k] w[n][k] + bias[n] (+ res)) (+ res).
//
// A workgroup makes a 64 x 64 tile of y: 16-wide slices of its rows of x and w
// go through LDS as fp32, each thread sums a 4 x 4 patch.
#include "common.hpp"
#include "device.hpp"

#include "flexserve.h"

namespace fs {

namespace {

__device__ __forceinline__ float load_f(const float* p) { return *p; }
__device__ __forceinline__ float load_f(const uint16_t* p) { return bf2f(*p); }

// bias, residual, activation and the one rounding of output (m, n)
__device__ __forceinline__ void linear_store(const LinearArgs& a, int m, int n, float v) {
  if (a.bias) v += a.bias[n];
  float r = 0.f;
  if (a.res) {
    const int64_t o = (int64_t)m * a.ldres + n;
    r = a.out_f32 ? static_cast<const float*>(a.res)[o] : bf2f(static_cast<const uint16_t*>(a.res)[o]);
  }
  if (a.res_first) v += r;
  if (a.act == FS_ACT_RELU) v = v > 0.f ? v : 0.f;
  else if (a.act == FS_ACT_GELU) v = 0.5f * v * (1.f + erff(v * 0.70710678f));
  else if (a.act == FS_ACT_SILU) v = v / (1.f + expf(-v));
  if (!a.res_first && a.res) v += r;
  const int64_t o = (int64_t)m * a.ldy + n;
  if (a.out_f32) static_cast<float*>(a.y)[o] = v;
  else static_cast<uint16_t*>(a.y)[o] = f2bf(v);
}

template <class T>
__global__ void __launch_bounds__(256) k_linear(LinearArgs a) {
  __shared__ float xs[16][65], ws[16][65];
  const int tiles_n = (a.N + 63) / 64;
  const int m0 = blockIdx.x / tiles_n * 64, n0 = blockIdx.x % tiles_n * 64;
  const int tid = threadIdx.x, tm = tid / 16 * 4, tn = tid % 16 * 4;
  const T* x = static_cast<const T*>(a.x);
  const T* w = static_cast<const T*>(a.w);
  float acc[4][4] = {};
  for (int k0 = 0; k0 < a.K; k0 += 16) {
    for (int i = tid; i < 64 * 16; i += 256) {
      const int r = i / 16, k = k0 + i % 16;
      xs[i % 16][r] = k < a.K && m0 + r < a.M ? load_f(x + (int64_t)(m0 + r) * a.ldx + k) : 0.f;
      ws[i % 16][r] = k < a.K && n0 + r < a.N ? load_f(w + (int64_t)(n0 + r) * a.ldw + k) : 0.f;
    }
    __syncthreads();
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xs[k][tm + i], ws[k][tn + j], acc[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (m0 + tm + i < a.M && n0 + tn + j < a.N) linear_store(a, m0 + tm + i, n0 + tn + j, acc[i][j]);
}

}  // namespace

void launch_linear(const LinearArgs& a, Prec p, hipStream_t s) {
  const int64_t tiles = (int64_t)((a.M + 63) / 64) * ((a.N + 63) / 64);
  if (p == BF16) hipLaunchKernelGGL(k_linear<uint16_t>, dim3((unsigned)tiles), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_linear<float>, dim3((unsigned)tiles), dim3(256), 0, s, a);
}

}  // namespace fs
