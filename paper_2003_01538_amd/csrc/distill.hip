// Distillation from a teacher's top classes.  With q the softmax of a row's
// teacher entries and p that of its logits, both at a temperature,
//   loss = sum_j q_j (ln q_j - ln p[id_j]),
//   d loss / d logits_c = (p_c - sum of q_j with id_j = c) / temperature.
// One workgroup per row.
#include "rows.hpp"


namespace fs {

namespace {

constexpr int ROW_T = 256;

template <class T>
__device__ void row_stats(const T* z, int C, float c, float* sh, float& m, float& s, float& t) {
  float best = -FLT_MAX;
  for (int i = threadIdx.x; i < C; i += ROW_T) best = fmaxf(best, RowT<T>::one(z + i));
  m = block_max<ROW_T>(best, sh);
  s = t = 0.f;
  for (int i = threadIdx.x; i < C; i += ROW_T) s += expf((RowT<T>::one(z + i) - m) * c);
  s = block_sum<ROW_T>(s, sh);
}

// The row's teacher in LDS: q[j] (0 for an entry that is left out) and id[j]
// (-1 for one).  Returns whether the teacher has any mass.
__device__ bool teacher(const DistillArgs& a, int64_t row, float c, float* q, int* id, float* sh) {
  const int j = threadIdx.x;
  float u = -INFINITY;
  int k = -1;
  if (j < a.K) {
    k = a.ids[row * a.K + j];
    if (k < 0 || k >= a.C) k = -1;
    else u = a.u[row * a.K + j];
  }
  const bool mass = __syncthreads_or(!(u == -INFINITY));
  const float m = block_max<ROW_T>(fmaxf(u, -FLT_MAX), sh);
  const float e = k < 0 ? 0.f : expf((u - m) * c);
  const float s = block_sum<ROW_T>(e, sh);
  if (j < a.K) { q[j] = mass ? e / s : 0.f; id[j] = k; }
  __syncthreads();
  return mass;
}

template <class T, bool STATS>
__global__ void __launch_bounds__(ROW_T) k_distill(DistillArgs a) {
  __shared__ float sh[ROW_T / 64], q[MAX_TOP];
  __shared__ int id[MAX_TOP];
  const float c = 1.f / a.temperature;
  for (int64_t row = blockIdx.x; row < a.R; row += gridDim.x) {
    const T* z = static_cast<const T*>(a.z) + row * a.ld;
    const bool mass = teacher(a, row, c, q, id, sh);
    float m, l;
    if constexpr (STATS) {
      float s, t;
      row_stats(z, a.C, c, sh, m, s, t);
      l = s == 0.f ? 0.f : logf(s);
      if (s == 0.f) m = -INFINITY;
      if (a.stats && threadIdx.x == 0) { a.stats[row * 2] = m; a.stats[row * 2 + 1] = l; }
    } else {
      m = a.stats[row * 2];
      l = a.stats[row * 2 + 1];
    }
    // this thread's teacher entry: the student's logit and log probability there, read before any gradient is written
    const int j = threadIdx.x;
    const int cj = j < a.K ? id[j] : -1;
    float lp = 0.f;
    if (cj >= 0) {
      const float x = RowT<T>::one(z + cj);
      lp = x == -INFINITY ? -INFINITY : (x - m) * c - l;
    }
    if (STATS && a.loss) {
      float part = 0.f;
      if (cj >= 0 && q[j] != 0.f) part = q[j] * (logf(q[j]) - lp);
      const float loss = block_sum<ROW_T>(part, sh);
      if (threadIdx.x == 0) a.loss[row] = mass ? loss : 0.f;
    }
    if (a.grad) {
      T* g = static_cast<T*>(a.grad) + row * a.ldg;
      const float wt = (a.weight ? a.weight[row] : 1.f) * c;
      __syncthreads();
      for (int i = threadIdx.x; i < a.C; i += ROW_T) {
        const float x = RowT<T>::one(z + i);
        RowT<T>::put(g + i, !mass ? 0.f : x == -INFINITY ? 0.f : expf((x - m) * c - l) * wt);
      }
      __syncthreads();
      if (mass && cj >= 0) {
        float sum = 0.f;  // entries of one class write the same value
        for (int i = 0; i < a.K; ++i) sum += id[i] == cj ? q[i] : 0.f;
        RowT<T>::put(g + cj, (expf(lp) - sum) * wt);
      }
    }
    __syncthreads();
  }
}

}  // namespace

void launch_distill(const DistillArgs& a, Prec p, hipStream_t s) {
  const dim3 grid(a.R < (1 << 20) ? a.R : 1 << 20);
  if (p == BF16) hipLaunchKernelGGL((k_distill<uint16_t, true>), grid, dim3(ROW_T), 0, s, a);
  else hipLaunchKernelGGL((k_distill<float, true>), grid, dim3(ROW_T), 0, s, a);
}

void launch_distill_grad(const DistillArgs& a, Prec p, hipStream_t s) {
  const dim3 grid(a.R < (1 << 20) ? a.R : 1 << 20);
  if (p == BF16) hipLaunchKernelGGL((k_distill<uint16_t, false>), grid, dim3(ROW_T), 0, s, a);
  else hipLaunchKernelGGL((k_distill<float, false>), grid, dim3(ROW_T), 0, s, a);
}

}  // namespace fs
