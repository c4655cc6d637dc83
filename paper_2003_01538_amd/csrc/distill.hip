// Distillation from a teacher's top classes.  With q the softmax of a row's
// teacher entries and p that of its logits, both at a temperature,
//   loss = sum_j q_j (ln q_j - ln p[id_j]),
//   d loss / d logits_c = (p_c - sum of q_j with id_j = c) / temperature.
//
// Memory bounds all of it, so the row is read once wherever it can be: a workgroup
// holds its row in registers (k_distill_held: up to 256 KB of a CU's 512) between the
// statistics and the gradient.  Longer rows are read twice (k_distill_long), the
// second time mostly from the last-level cache.  Few long rows are cut into segments
// for more workgroups: one launch for the statistics, through the scratch memory,
// and one for loss and gradient.  The gradient alone, from given statistics, is one
// pass in segments.
//
// The gradient is written as weight / temperature * p everywhere, then, after a
// barrier of the workgroup that wrote them, again at the teacher's classes, where all
// entries of a class write the same value.
#include "rows.hpp"

#include "flexserve.h"

#include <algorithm>

namespace fs {

namespace {

// The teacher's entries of a row, entry n NT + t with thread t, and what the
// workgroup shares of them.
template <int NT>
struct Shared {
  float red[NT / 64][2], q[MAX_TOP];
  int id[MAX_TOP];
};
template <class T, int NT>
struct Teacher {
  static constexpr int E = (MAX_TOP + NT - 1) / NT;
  int id[E];    // -1: none, or left out
  float u[E];   // then e^((u - max) c), then q
  float z[E];   // the student's logit of the class

  __device__ __forceinline__ void load(const DistillArgs& a, int64_t row, const T* zr) {
#pragma unroll
    for (int n = 0; n < E; ++n) {
      const int j = n * NT + threadIdx.x;
      id[n] = j < a.K ? a.ids[row * a.K + j] : -1;
      u[n] = j < a.K ? a.u[row * a.K + j] : -INFINITY;
      if (id[n] < 0 || id[n] >= a.C) { id[n] = -1; u[n] = -INFINITY; }
    }
#pragma unroll
    for (int n = 0; n < E; ++n) z[n] = id[n] >= 0 && zr ? RowT<T>::one(zr + id[n]) : -INFINITY;
  }
  // the student's logits have arrived: what lies there may be overwritten
  __device__ __forceinline__ void settle() {
#pragma unroll
    for (int n = 0; n < E; ++n) __asm__ volatile("" : "+v"(z[n]));
  }
  __device__ __forceinline__ float max() const {
    float m = -FLT_MAX;
#pragma unroll
    for (int n = 0; n < E; ++n) m = fmaxf(m, u[n]);
    return m;
  }
  __device__ __forceinline__ float exps(float m, float k2) {
    float s = 0.f;
#pragma unroll
    for (int n = 0; n < E; ++n) {
      u[n] = __builtin_amdgcn_exp2f((u[n] - m) * k2);
      s += u[n];
    }
    return s;
  }
  // q, given the sum of exps(); visible to the workgroup after its next barrier
  __device__ __forceinline__ void share(float s, Shared<NT>& S) {
    const float inv = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
    for (int n = 0; n < E; ++n) {
      const int j = n * NT + threadIdx.x;
      u[n] = id[n] < 0 ? 0.f : u[n] * inv;
      if (j < MAX_TOP) { S.q[j] = u[n]; S.id[j] = id[n]; }
    }
  }
};

// (m, l): the row's statistics, l = ln s; m is -inf in a row without classes
struct Stats {
  float m, l;
};
__device__ __forceinline__ Stats stats_of(float m, float s) { return s == 0.f ? Stats{-INFINITY, 0.f} : Stats{m, logf(s)}; }
__device__ __forceinline__ float ln_p(const Stats& st, float z, float c) { return z == -INFINITY ? -INFINITY : (z - st.m) * c - st.l; }

// This thread's part of the loss.
template <class T, int NT>
__device__ __forceinline__ float loss_part(const Teacher<T, NT>& t, const Stats& st, float c) {
  float part = 0.f;
#pragma unroll
  for (int n = 0; n < Teacher<T, NT>::E; ++n)
    if (t.id[n] >= 0 && t.u[n] != 0.f) part += t.u[n] * (logf(t.u[n]) - ln_p(st, t.z[n], c));
  return part;
}

// The gradient without the teacher: scale * e^((z - m) c - l).  Rows whose
// teacher has no mass are 0, as are classes at -inf whatever the row holds.
struct Grad {
  float m, k2, l2, scale;
  bool zero, care;  // all 0; classes at -inf need a look
  __device__ __forceinline__ Grad(const Stats& st, float c, float weight, bool mass)
      : m(st.m), k2(LOG2E * c), l2(LOG2E * st.l), scale(weight * c), zero(!mass || st.m == -INFINITY),
        care(!(fabsf(st.l) < INFINITY) || !(fabsf(scale) < INFINITY)) {}
  __device__ __forceinline__ float at(float z) const {
    const float p = __builtin_amdgcn_exp2f(fmaf(z - m, k2, -l2)) * scale;
    return zero || (care && z == -INFINITY) ? 0.f : p;
  }
  template <class T>
  __device__ __forceinline__ u32x4 vec(u32x4 v) const {
    constexpr int VEC = RowT<T>::VEC;
    float f[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] = __builtin_amdgcn_exp2f(fmaf(RowT<T>::get(v, e) - m, k2, -l2)) * scale;
    if (zero || care) {  // the same for the whole workgroup
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[e] = at(RowT<T>::get(v, e));
    }
    return RowT<T>::pack(f);
  }
};

// The vectors that row_chunk loads, as gradients.
template <class T, int NT, int NV, bool ONCE>
__device__ __forceinline__ void put_chunk(T* g, int64_t from, int64_t end, const u32x4 (&v)[NV], const Grad& gr) {
  constexpr int VEC = RowT<T>::VEC;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t i = from + (int64_t)(j * NT + (int)threadIdx.x) * VEC;
    const u32x4 q = gr.template vec<T>(v[j]);
    if (from + (int64_t)(j + 1) * NT * VEC <= end) store_vec<ONCE>(g + i, q);  // the same for the whole workgroup
    else put_vec(g, i, end, q);
  }
}

// The gradient at the teacher's classes in first .. end - 1, after the barrier that follows
// the others'.
template <class T, int NT>
__device__ __forceinline__ void put_teacher(const DistillArgs& a, T* g, const Teacher<T, NT>& t, const Shared<NT>& S, const Stats& st,
                                            const Grad& gr, float c, int64_t first, int64_t end) {
#pragma unroll
  for (int n = 0; n < Teacher<T, NT>::E; ++n) {
    const int k = t.id[n];
    if (k < first || k >= end) continue;
    float sum = 0.f;
    for (int j = 0; j < a.K; ++j) sum += S.id[j] == k ? S.q[j] : 0.f;
    const float p = st.m == -INFINITY || t.z[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(t.z[n] - gr.m, gr.k2, -gr.l2));
    RowT<T>::put(g + k, (p - sum) * gr.scale);
  }
}

// The workgroup's stores have been made: others to the same places come after.  A wave's own
// ordinary stores keep their order without a wait; that those past the caches (ONCE) keep it
// with ordinary ones behind them is promised nowhere.
template <int NT, bool ONCE>
__device__ __forceinline__ void written() {
  if constexpr (NT > 64 || ONCE) __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

__device__ __forceinline__ float weight_of(const DistillArgs& a, int64_t row) { return a.weight ? a.weight[row] : 1.f; }

// Rows of at most NT * NV vectors.  Up to 16 vectors a thread four waves share a SIMD,
// so that one row's loads run beside another's stores.
template <class T, int NT, int NV, bool ONCE>
__global__ void __launch_bounds__(NT, NV > 16 ? 2 : 4) k_distill_held(DistillArgs a) {
  using RT = RowT<T>;
  constexpr int VEC = RT::VEC;
  __shared__ Shared<NT> S;
  const float c = 1.f / a.temperature, k2 = LOG2E * c;
  for (int64_t row = blockIdx.x; row < a.R; row += gridDim.x) {
    const T* z = static_cast<const T*>(a.z) + row * a.ld;
    const int C = row_end(a.C);
    u32x4 v[NV];
    row_chunk<T, NT, NV, ONCE>(z, 0, C, v);
    Teacher<T, NT> t;
    t.load(a, row, z);
    float m = -FLT_MAX, um = t.max();
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) m = fmaxf(m, RT::get(v[j], e));
    forget(v);
    block_max2<NT>(m, um, S.red);
    float s = 0.f, us = t.exps(um, k2);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) s += __builtin_amdgcn_exp2f((RT::get(v[j], e) - m) * k2);
    forget(v);
    block_sum2<NT>(s, us, S.red);
    t.share(us, S);
    const Stats st = stats_of(m, s);
    if (a.stats && threadIdx.x == 0) { a.stats[row * 2] = st.m; a.stats[row * 2 + 1] = st.l; }
    if (a.loss) {
      const float loss = block_sum<NT>(loss_part(t, st, c), &S.red[0][0]);
      if (threadIdx.x == 0) a.loss[row] = loss;  // 0 without mass: every q is
    }
    if (a.grad) {
      T* g = static_cast<T*>(a.grad) + row * a.ldg;
      const Grad gr(st, c, weight_of(a, row), us != 0.f);
      t.settle();
      __syncthreads();  // the row and its teacher's classes have been read (the gradient may lie over them)
      put_chunk<T, NT, NV, ONCE>(g, 0, row_end(C), v, gr);
      written<NT, ONCE>();
      if (us != 0.f) put_teacher<T, NT>(a, g, t, S, st, gr, c, 0, a.C);
    }
    __syncthreads();
  }
}

// Statistics of z[first .. end - 1] over the workgroup: m and s.
template <class T, int NT, int NV>
__device__ __forceinline__ RowStats<false> walk_stats(const T* z, int64_t first, int64_t end, float k2, float (*sh)[2]) {
  using RT = RowT<T>;
  constexpr int VEC = RT::VEC, CHUNK = NT * NV * VEC;
  RowStats<false> st;
  u32x4 v[NV], next[NV];
  row_chunk<T, NT, NV, false>(z, first, end, v);
  for (int64_t from = first; from < end; from += CHUNK) {
    const bool more = from + CHUNK < end;
    if (more) row_chunk<T, NT, NV, false>(z, from + CHUNK, end, next);
    float best = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) best = fmaxf(best, RT::get(v[j], e));
    if (best > st.m) st.lift(best, k2);
    RowStats<false> part = st.empty();
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) part.add(RT::get(v[j], e), k2);
    st.join(part);
    if (more)
#pragma unroll
      for (int j = 0; j < NV; ++j) v[j] = next[j];
  }
  st.over_block<NT>(k2, sh);
  return st;
}

// The gradient without the teacher, of z[first .. end - 1].
template <class T, int NT, int NV, bool ONCE>
__device__ __forceinline__ void walk_grad(const T* z, T* g, int64_t first, int64_t end, const Grad& gr) {
  constexpr int CHUNK = NT * NV * RowT<T>::VEC;
  u32x4 v[NV], next[NV];
  row_chunk<T, NT, NV, ONCE>(z, first, end, v);
  for (int64_t from = first; from < end; from += CHUNK) {
    const bool more = from + CHUNK < end;
    if (more) row_chunk<T, NT, NV, ONCE>(z, from + CHUNK, end, next);
    put_chunk<T, NT, NV, ONCE>(g, from, end, v, gr);
    if (more)
#pragma unroll
      for (int j = 0; j < NV; ++j) v[j] = next[j];
  }
}

// Rows of any length, read once for the statistics and once for the gradient.
template <class T, int NT, int NV>
__global__ void __launch_bounds__(NT) k_distill_long(DistillArgs a) {
  __shared__ Shared<NT> S;
  const float c = 1.f / a.temperature, k2 = LOG2E * c;
  for (int64_t row = blockIdx.x; row < a.R; row += gridDim.x) {
    const T* z = static_cast<const T*>(a.z) + row * a.ld;
    Teacher<T, NT> t;
    t.load(a, row, z);
    const RowStats<false> rs = walk_stats<T, NT, NV>(z, 0, row_end(a.C), k2, S.red);
    const Stats st = stats_of(rs.m, rs.s);
    const float us = block_sum<NT>(t.exps(block_max<NT>(t.max(), &S.red[0][0]), k2), &S.red[0][0]);
    t.share(us, S);
    if (a.stats && threadIdx.x == 0) { a.stats[row * 2] = st.m; a.stats[row * 2 + 1] = st.l; }
    if (a.loss) {
      const float loss = block_sum<NT>(loss_part(t, st, c), &S.red[0][0]);
      if (threadIdx.x == 0) a.loss[row] = loss;
    }
    if (a.grad) {
      T* g = static_cast<T*>(a.grad) + row * a.ldg;
      const Grad gr(st, c, weight_of(a, row), us != 0.f);
      t.settle();
      __syncthreads();
      walk_grad<T, NT, NV, false>(z, g, 0, row_end(a.C), gr);
      written<NT, false>();
      if (us != 0.f) put_teacher<T, NT>(a, g, t, S, st, gr, c, 0, a.C);
    }
    __syncthreads();
  }
}

// The scratch memory of rows in segments: the segments' statistics, then the
// students' logits at the teachers' classes, since the gradient may be written over
// them before the loss is formed.
struct Part {
  float m, s;
};
__device__ __forceinline__ float* scratch_z(const DistillArgs& a, int segs) {
  return reinterpret_cast<float*>(static_cast<Part*>(a.scratch) + (int64_t)a.R * segs);
}

template <class T, int NT, int NV>
__global__ void __launch_bounds__(NT) k_distill_stats(DistillArgs a, int segs, int seg) {
  __shared__ float sh[NT / 64][2];
  const int row = blockIdx.x / segs, first = (blockIdx.x - row * segs) * seg;
  const T* z = static_cast<const T*>(a.z) + (int64_t)row * a.ld;
  if (first == 0)
    for (int j = threadIdx.x; j < a.K; j += NT) {
      const int k = a.ids[(int64_t)row * a.K + j];
      scratch_z(a, segs)[(int64_t)row * a.K + j] = k >= 0 && k < a.C ? RowT<T>::one(z + k) : -INFINITY;
    }
  const RowStats<false> st = walk_stats<T, NT, NV>(z, first, min((int64_t)a.C, (int64_t)first + seg), LOG2E / a.temperature, sh);
  if (threadIdx.x == 0) static_cast<Part*>(a.scratch)[blockIdx.x] = Part{st.m, st.s};
}

// Loss (the first segment's workgroup) and gradient of a segment.  PARTS: the
// statistics are `parts` parts in the scratch memory; otherwise a.stats holds them.
template <class T, int NT, int NV, bool PARTS, bool ONCE>
__global__ void __launch_bounds__(NT) k_distill_segment(DistillArgs a, int segs, int seg, int parts) {
  __shared__ Shared<NT> S;
  const float c = 1.f / a.temperature, k2 = LOG2E * c;
  const int64_t items = (int64_t)a.R * segs;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t row = item / segs, first = (item - row * segs) * seg, end = min((int64_t)a.C, first + seg);
    const T* z = static_cast<const T*>(a.z) + row * a.ld;
    Teacher<T, NT> t;
    t.load(a, row, PARTS ? nullptr : z);
    float us = block_sum<NT>(t.exps(block_max<NT>(t.max(), &S.red[0][0]), k2), &S.red[0][0]);
    t.share(us, S);
    Stats st;
    if constexpr (PARTS) {
      RowStats<false> rs;
      for (int i = threadIdx.x; i < parts; i += NT) {
        const Part p = static_cast<const Part*>(a.scratch)[row * parts + i];
        RowStats<false> q;
        q.m = p.m; q.s = p.s;
        const float m = fmaxf(rs.m, q.m);
        rs.lift(m, k2);
        q.lift(m, k2);
        rs.s += q.s;
      }
#pragma unroll
      for (int n = 0; n < Teacher<T, NT>::E; ++n)
        if (t.id[n] >= 0) t.z[n] = scratch_z(a, parts)[row * a.K + n * NT + threadIdx.x];
      rs.over_block<NT>(k2, S.red);
      st = stats_of(rs.m, rs.s);
      if (first == 0) {
        if (a.stats && threadIdx.x == 0) { a.stats[row * 2] = st.m; a.stats[row * 2 + 1] = st.l; }
        if (a.loss) {
          const float loss = block_sum<NT>(loss_part(t, st, c), &S.red[0][0]);
          if (threadIdx.x == 0) a.loss[row] = loss;
        }
      }
    } else {
      st = Stats{a.stats[row * 2], a.stats[row * 2 + 1]};
    }
    if (a.grad) {
      T* g = static_cast<T*>(a.grad) + row * a.ldg;
      const Grad gr(st, c, weight_of(a, row), us != 0.f);
      t.settle();
      __syncthreads();  // this segment's classes of the teacher have been read
      walk_grad<T, NT, NV, ONCE>(z, g, first, end, gr);
      written<NT, ONCE>();
      if (us != 0.f) put_teacher<T, NT>(a, g, t, S, st, gr, c, first, end);
    }
    __syncthreads();
  }
}

constexpr int64_t GRID = 1 << 20;  // workgroups walk the rows beyond
constexpr int SEGS = 512;          // segments of all rows whose statistics are split
static_assert(SEGS * (sizeof(Part) + MAX_TOP * sizeof(float)) <= FS_ROW_SCRATCH_BYTES, "scratch");

// A row's segments: `want` of them, whole chunks each.
struct Cut {
  int segs, seg;
};
Cut cut_row(int C, int chunk, int64_t want) {
  const int chunks = (int)(((int64_t)C + chunk - 1) / chunk);
  const int n = (int)std::max<int64_t>(1, std::min<int64_t>(chunks, want));
  const int per = (chunks + n - 1) / n;
  return {(chunks + per - 1) / per, (int)std::min<int64_t>((int64_t)per * chunk, INT32_MAX)};
}

template <class T, int NT, bool PARTS, bool ONCE>
void segments(const DistillArgs& a, Cut cut, int parts, hipStream_t s) {
  const int64_t items = (int64_t)a.R * cut.segs;
  hipLaunchKernelGGL((k_distill_segment<T, NT, 4, PARTS, ONCE>), dim3((unsigned)std::min(items, GRID)), dim3(NT), 0, s, a, cut.segs, cut.seg, parts);
}

// Rows in the registers of NT threads, by the first of so many vectors each that holds them.
template <class T, int NT, bool ONCE, int NV, int... MORE>
bool held(const DistillArgs& a, hipStream_t s) {
  if (a.C <= NT * NV * RowT<T>::VEC) {
    hipLaunchKernelGGL((k_distill_held<T, NT, NV, ONCE>), dim3((unsigned)std::min<int64_t>(a.R, GRID)), dim3(NT), 0, s, a);
    return true;
  }
  if constexpr (sizeof...(MORE) > 0) return held<T, NT, ONCE, MORE...>(a, s);
  return false;
}

template <class T>
void launch_t(const DistillArgs& a, hipStream_t s) {
  constexpr int VEC = RowT<T>::VEC;  // 16 bytes
  // the fewest threads and vectors that hold the row, since places without a class cost as
  // much as others (bf16 with gradients: 60000 rows of 2500 classes 155 us with 128 x 4
  // vectors against 280 with 256 x 4; 8000 rows of 17000 101 with 256 x 10, 131 with 256 x
  // 16; 4000 of 34000 112 with 512 x 10, 159 with 512 x 16); read twice, 4096 rows of 8192
  // fp32 take 69 us against 55
  if (held<T, 64, false, 4>(a, s) || held<T, 128, false, 4, 6>(a, s) || held<T, 256, false, 4>(a, s)) return;
  const bool once = beyond_cache((int64_t)a.R * a.C * (int)sizeof(T) * (a.grad ? 2 : 1));
  if (once ? held<T, 256, true, 6, 8, 10, 12, 14, 16>(a, s) : held<T, 256, false, 6, 8, 10, 12, 14, 16>(a, s)) return;
  if (once ? held<T, 512, true, 10, 12, 14, 16>(a, s) : held<T, 512, false, 10, 12, 14, 16>(a, s)) return;
  // beyond 128 KB a row, too few rows for the chip go in segments (fp32, 131072 classes,
  // with gradients: 8 rows 10 us against 23, 64 rows 25 against 32, 128 rows 45 against 41)
  if (a.scratch && a.R <= 64) {
    const Cut cut = cut_row(a.C, 256 * 4 * VEC, SEGS / a.R);
    hipLaunchKernelGGL((k_distill_stats<T, 256, 4>), dim3((unsigned)(a.R * cut.segs)), dim3(256), 0, s, a, cut.segs, cut.seg);
    return segments<T, 256, true, false>(a, a.grad ? cut : Cut{1, a.C}, cut.segs, s);
  }
  if (once ? held<T, 512, true, 20, 24, 28, 32>(a, s) : held<T, 512, false, 20, 24, 28, 32>(a, s)) return;
  hipLaunchKernelGGL((k_distill_long<T, 1024, 4>), dim3((unsigned)std::min<int64_t>(a.R, GRID)), dim3(1024), 0, s, a);
}

// About 4096 segments of whole chunks, the chunk by the row's length: 120000 rows of
// 1001 fp32 205 us with one wave a row, 460 with four; 60000 rows of 2049 193 with two
// waves, 248 with four; 8000 rows of 16384 200 with two, 184 with four.
template <class T, int NT, bool ONCE>
void grad_segments(const DistillArgs& a, hipStream_t s) {
  segments<T, NT, false, ONCE>(a, cut_row(a.C, NT * 4 * RowT<T>::VEC, std::max<int64_t>(1, 4096 / a.R)), 0, s);
}
template <class T>
void launch_grad_t(const DistillArgs& a, hipStream_t s) {
  constexpr int VEC = RowT<T>::VEC;
  if (a.C <= 64 * 4 * VEC) return grad_segments<T, 64, false>(a, s);
  const bool once = beyond_cache((int64_t)a.R * a.C * (int)sizeof(T) * 2);
  if (a.C <= 64 * 8 * VEC) return once ? grad_segments<T, 64, true>(a, s) : grad_segments<T, 64, false>(a, s);
  if (a.C <= 512 * 4 * VEC) return once ? grad_segments<T, 128, true>(a, s) : grad_segments<T, 128, false>(a, s);
  return once ? grad_segments<T, 256, true>(a, s) : grad_segments<T, 256, false>(a, s);
}

}  // namespace

void launch_distill(const DistillArgs& a, Prec p, hipStream_t s) {
  if (p == BF16) launch_t<uint16_t>(a, s);
  else launch_t<float>(a, s);
}

void launch_distill_grad(const DistillArgs& a, Prec p, hipStream_t s) {
  if (p == BF16) launch_grad_t<uint16_t>(a, s);
  else launch_grad_t<float>(a, s);
}

}  // namespace fs
