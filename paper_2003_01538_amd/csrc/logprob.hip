// Log probabilities of given classes under the softmax of rows of logits, the
// entropy, and the most probable classes:
//   ln p_c = (z_c - m) - ln s,   H = ln s - t / s
// with the row's statistics m, s, t.  One workgroup per row.
#include "rows.hpp"

namespace fs {

namespace {

// a comes before b among the alternatives: larger logit, then lower class
__device__ __forceinline__ bool before(float va, int ia, float vb, int ib) { return va > vb || (va == vb && ia < ib); }

template <class T>
__global__ void __launch_bounds__(ROW_T) k_logprob(LogprobArgs a) {
  __shared__ float sh[ROW_T / 64];
  __shared__ int si[ROW_T / 64];
  for (int64_t row = blockIdx.x; row < a.R; row += gridDim.x) {
    const T* z = static_cast<const T*>(a.z) + row * a.ld;
    float m, s, t;
    row_stats(z, a.C, 1.f, sh, m, s, t);
    const float ls = logf(s);
    if (a.entropy && threadIdx.x == 0) a.entropy[row] = s == 0.f ? 0.f : ls - t / s;
    for (int i = threadIdx.x; i < a.T; i += ROW_T) {
      const int c = a.classes[row * a.T + i];
      const float v = c >= 0 && c < a.C ? row_load(z + c) : -INFINITY;
      a.logp[row * a.T + i] = v == -INFINITY ? -INFINITY : (v - m) - ls;
    }
    float pv = INFINITY;  // the alternative found last
    int pi = -1;
    for (int k = 0; k < a.K; ++k) {
      float v = -INFINITY;
      int c = a.C;
      for (int i = threadIdx.x; i < a.C; i += ROW_T) {
        const float x = row_load(z + i);
        if (before(pv, pi, x, i) && before(x, i, v, c) && x > -INFINITY) { v = x; c = i; }
      }
      wave_argmax(v, c);
      if ((threadIdx.x & 63) == 0) { sh[threadIdx.x >> 6] = v; si[threadIdx.x >> 6] = c; }
      __syncthreads();
      v = sh[0]; c = si[0];
      for (int w = 1; w < ROW_T / 64; ++w)
        if (before(sh[w], si[w], v, c)) { v = sh[w]; c = si[w]; }
      __syncthreads();
      const bool none = c == a.C;
      if (threadIdx.x == 0) {
        a.top_ids[row * a.K + k] = none ? -1 : c;
        a.top_logp[row * a.K + k] = none ? -INFINITY : (v - m) - ls;
      }
      pv = none ? -INFINITY : v;
      pi = c;
    }
  }
}

}  // namespace

void launch_logprob(const LogprobArgs& a, Prec p, hipStream_t s) {
  const dim3 grid(a.R < (1 << 20) ? a.R : 1 << 20);
  if (p == BF16) hipLaunchKernelGGL(k_logprob<uint16_t>, grid, dim3(ROW_T), 0, s, a);
  else hipLaunchKernelGGL(k_logprob<float>, grid, dim3(ROW_T), 0, s, a);
}

}  // namespace fs
