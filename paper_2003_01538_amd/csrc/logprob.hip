// Log probabilities of given classes under the softmax of rows of logits, the
// entropy, and the most probable classes:
//   ln p_c = (z_c - m) - ln s,   H = ln s - t / s
// with the row's statistics m, s, t (rows.hpp).
//
// One pass over the logits: a workgroup walks its row (or its segment of a row)
// in chunks that it holds in registers.  Each thread folds its logits into
// running statistics; the same registers then serve the selection.  A logit is
// a candidate when it is larger than the K-th best so far, `bar`; candidates go to a
// list in LDS as (logit, class) in one whole number that orders them, and the list
// is cut to its K best, by counting for each entry those before it, once it has
// grown by SLACK.  After the first chunk few threads see a candidate (K in K/i of the
// i-th chunk), so that the selection costs little more than the comparison with the
// thread's maximum, which the statistics need anyway.  In a chunk with too many
// candidates to list (the first one; rising rows) a threshold between the K-th and
// the LIST-th best is searched bit by bit, first over the threads' maxima, which
// mostly give one, else over the chunk.
//
// When there are few rows they are cut into segments, one workgroup each; the
// segments' statistics and K best go to the scratch memory, and a second launch
// joins them with the same selection.
#include "rows.hpp"

#include "flexserve.h"

#include <algorithm>

namespace fs {

namespace {

// A logit and its class as one number: the larger logit is the larger, of equal
// logits (+0 and -0 are equal) the lower class.  0: none.
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t b = __float_as_uint(z + 0.f);
  return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint64_t entry(float z, int c) { return uint64_t(order_key(z)) << 32 | ~uint32_t(c); }
__device__ __forceinline__ float entry_logit(uint64_t e) {
  const uint32_t k = uint32_t(e >> 32);
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ int entry_class(uint64_t e) { return int(~uint32_t(e)); }

constexpr int SLACK = 64;  // entries that the list grows by before it is cut

template <int NT>
struct Selection {
  static constexpr int LIST = NT == 64 ? 512 : 1024;
  uint64_t list[LIST];
  uint64_t top[MAX_TOP];
  uint32_t maxima[NT];
  int hits[3], n, count[NT / 64];
};

// Sum over the workgroup of a number that is already the wave's.
template <int NT>
__device__ __forceinline__ int block_count(int v, int* sh) {
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) v += sh[w];
    __syncthreads();
  }
  return v;
}

// Cut the list's n entries to the K best, in falling order; returns how many remain.
template <int NT>
__device__ int cut(Selection<NT>& S, int n, int K) {
  for (int i = threadIdx.x; i < n; i += NT) {
    const uint64_t own = S.list[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += S.list[j] > own ? 1 : 0;
    if (rank < K) S.top[rank] = own;
  }
  __syncthreads();
  n = min(n, K);
  for (int i = threadIdx.x; i < n; i += NT) S.list[i] = S.top[i];
  if (threadIdx.x == 0) S.n = n;
  __syncthreads();
  return n;
}

// One chunk's candidates into the list.  get(j, z, c): this thread's j-th of NE
// logits and its class; best: the largest of them (-inf: none).  `bar` is the
// K-th best logit so far (-inf: fewer than K), n the list's length, `turn` counts the
// calls; the three are the same in every thread.
template <int NT, int NE, class Get>
__device__ __forceinline__ void select_chunk(Selection<NT>& S, int K, float best, Get&& get, float& bar, int& n, int turn) {
  constexpr int LIST = Selection<NT>::LIST;
  const int lane = threadIdx.x & 63;
  const uint64_t wave_hits = __ballot(best > bar);
  int hits;
  if constexpr (NT == 64) {
    hits = __popcll(wave_hits);
  } else {
    // three counters in turn: the one of two calls on is cleared while no wave can be there yet
    if (wave_hits && lane == 0) atomicAdd(&S.hits[turn % 3], (int)__popcll(wave_hits));
    __syncthreads();
    hits = S.hits[turn % 3];
    if (threadIdx.x == 0) S.hits[(turn + 2) % 3] = 0;
  }
  if (hits == 0) return;

  uint64_t least = 0;  // entries below this are not listed
  const bool many = n + hits * NE > LIST;
  if (many) {
    if (n > K) n = cut(S, n, K);
    const int most = LIST - n;
    // over the threads' maxima: the key that K or a few more of them reach
    uint32_t key = 0;
    if (hits > K) {
      S.maxima[threadIdx.x] = best > bar ? order_key(best) : 0;
      __syncthreads();
      uint32_t mx[NT / 64];
#pragma unroll
      for (int w = 0; w < NT / 64; ++w) mx[w] = S.maxima[w * 64 + lane];
      for (int bit = 31; bit >= 0; --bit) {
        const uint32_t up = key | 1u << bit;
        int c = 0;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) c += (int)__popcll(__ballot(mx[w] >= up));
        if (c < K) continue;
        key = up;
        if (c <= K + (K >> 3) + 2) break;
      }
    }
    least = uint64_t(key) << 32;
    // too many logits of the chunk there: over the chunk, down to the class
    auto reach = [&](uint64_t lo) {
      int c = 0;
#pragma unroll
      for (int j = 0; j < NE; ++j) {
        float z;
        int k;
        get(j, z, k);
        c += (int)__popcll(__ballot(z > bar && entry(z, k) >= lo));
      }
      return block_count<NT>(c, S.count);
    };
    if (reach(least) > most) {
      least = 0;
      for (int bit = 63; bit >= 0; --bit) {
        const uint64_t up = least | 1ull << bit;
        const int c = reach(up);
        if (c < K) continue;
        least = up;
        if (c <= most) break;
      }
    }
  }
  if (wave_hits) {
#pragma unroll
    for (int j = 0; j < NE; ++j) {
      float z;
      int k;
      get(j, z, k);
      const uint64_t e = entry(z, k);
      const bool take = z > bar && e >= least;
      const uint64_t b = __ballot(take);
      if (!b) continue;
      int at = 0;
      if (lane == 0) at = atomicAdd(&S.n, (int)__popcll(b));
      at = __builtin_amdgcn_readfirstlane(at);
      if (take) S.list[at + __popcll(b & ((1ull << lane) - 1))] = e;
    }
  }
  __syncthreads();
  n = S.n;
  if (n >= K + SLACK || many) {
    __syncthreads();  // S.n has been read
    n = cut(S, n, K);
  }
  if (n == K && K > 0) bar = entry_logit(S.list[K - 1]);
}

template <int NT>
__device__ __forceinline__ void select_begin(Selection<NT>& S) {
  if (threadIdx.x == 0) S.hits[0] = S.hits[1] = S.hits[2] = S.n = 0;
  __syncthreads();
}

// ln p of the given classes, entropy and alternatives of a row from its statistics and its list.
template <class T, int NT>
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t row, const T* z, const RowStats<true>& st,
                                          Selection<NT>& S, int n) {
  const float ls = logf(st.s);
  if (a.entropy && threadIdx.x == 0) a.entropy[row] = st.s == 0.f ? 0.f : ls - st.t / st.s;
  for (int i = threadIdx.x; i < a.T; i += NT) {
    const int c = a.classes[row * a.T + i];
    const float v = c >= 0 && c < a.C ? RowT<T>::one(z + c) : -INFINITY;
    a.logp[row * a.T + i] = v == -INFINITY ? -INFINITY : (v - st.m) - ls;
  }
  for (int i = threadIdx.x; i < a.K; i += NT) {
    a.top_ids[row * a.K + i] = i < n ? entry_class(S.list[i]) : -1;
    a.top_logp[row * a.K + i] = i < n ? (entry_logit(S.list[i]) - st.m) - ls : -INFINITY;
  }
}

// A segment's results in the scratch memory: m, s, t, the number of entries, and the entries.
struct Part {
  float m, s, t;
  int n;
};

// Row blockIdx / segs, segment blockIdx % segs of `seg` classes; SPLIT: to the scratch memory.
template <class T, int NT, int NV, bool SPLIT>
__global__ void __launch_bounds__(NT) k_logprob(LogprobArgs a, int segs, int seg) {
  using RT = RowT<T>;
  constexpr int VEC = RT::VEC, NE = NV * VEC, CHUNK = NT * NE;
  __shared__ Selection<NT> S;
  __shared__ float sh[NT / 64];
  const int64_t items = (int64_t)a.R * segs;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t row = SPLIT ? item / segs : item;
    const int64_t first = SPLIT ? (item - row * segs) * seg : 0;
    const int64_t end = SPLIT ? min((int64_t)a.C, first + seg) : a.C;
    const T* z = static_cast<const T*>(a.z) + row * a.ld;
    select_begin(S);
    RowStats<true> st;
    float bar = -INFINITY;
    int n = 0, turn = 0;
    u32x4 v[NV], next[NV];
    row_chunk<T, NT, NV>(z, first, end, v);
    for (int64_t from = first; from < end; from += CHUNK, ++turn) {
      const bool more = from + CHUNK < end;
      if (more) row_chunk<T, NT, NV>(z, from + CHUNK, end, next);
      float best = -INFINITY;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) best = fmaxf(best, RT::get(v[j], e));
      if (best > st.m) st.lift(best, LOG2E);
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) st.add(RT::get(v[j], e), LOG2E);
      if (a.K > 0) {
        const int base = (int)from + (int)threadIdx.x * VEC;
        select_chunk<NT, NE>(S, a.K, best, [&](int j, float& x, int& c) {
          x = RT::get(v[j / VEC], j % VEC);
          c = base + j / VEC * NT * VEC + j % VEC;
        }, bar, n, turn);
      }
      if (more)
#pragma unroll
        for (int j = 0; j < NV; ++j) v[j] = next[j];
    }
    __syncthreads();
    if (a.K > 0) n = cut(S, n, a.K);
    st.over_block<NT>(LOG2E, sh);
    if constexpr (SPLIT) {
      Part* part = static_cast<Part*>(a.scratch) + item;
      uint64_t* list = reinterpret_cast<uint64_t*>(static_cast<Part*>(a.scratch) + items) + item * a.K;
      if (threadIdx.x == 0) *part = Part{st.m, st.s, st.t, n};
      for (int i = threadIdx.x; i < a.K; i += NT) list[i] = i < n ? S.list[i] : 0;
    } else {
      write_row<T, NT>(a, row, z, st, S, n);
    }
    __syncthreads();
  }
}

constexpr int JOIN_T = 256, JOIN_E = 8;

// The segments of a row, joined.
template <class T>
__global__ void __launch_bounds__(JOIN_T) k_logprob_join(LogprobArgs a, int segs) {
  __shared__ Selection<JOIN_T> S;
  __shared__ float sh[JOIN_T / 64];
  const int64_t row = blockIdx.x;
  const Part* part = static_cast<const Part*>(a.scratch) + row * segs;
  const uint64_t* list = reinterpret_cast<const uint64_t*>(static_cast<const Part*>(a.scratch) + (int64_t)a.R * segs) + row * segs * a.K;
  select_begin(S);
  RowStats<true> st;
  for (int i = threadIdx.x; i < segs; i += JOIN_T) {
    const Part p = part[i];
    RowStats<true> q;
    q.m = p.m; q.s = p.s; q.t = p.t;
    const float m = fmaxf(st.m, q.m);
    st.lift(m, LOG2E);
    q.lift(m, LOG2E);
    st.s += q.s;
    st.t += q.t;
  }
  float bar = -INFINITY;
  int n = 0, turn = 0;
  // equal logits in later entries have higher classes, as select_chunk's bar needs: segments
  // are in the order of their classes, and so are equal logits inside one
  for (int from = 0; from < segs * a.K; from += JOIN_T * JOIN_E, ++turn) {
    uint64_t e[JOIN_E];
    float best = -INFINITY;
#pragma unroll
    for (int j = 0; j < JOIN_E; ++j) {
      const int i = from + j * JOIN_T + threadIdx.x;
      e[j] = i < segs * a.K ? list[i] : 0;
      if (e[j]) best = fmaxf(best, entry_logit(e[j]));
    }
    select_chunk<JOIN_T, JOIN_E>(S, a.K, best, [&](int j, float& x, int& c) {
      x = e[j] ? entry_logit(e[j]) : -INFINITY;
      c = entry_class(e[j]);
    }, bar, n, turn);
  }
  __syncthreads();
  if (a.K > 0) n = cut(S, n, a.K);
  st.over_block<JOIN_T>(LOG2E, sh);
  write_row<T, JOIN_T>(a, row, static_cast<const T*>(a.z) + row * a.ld, st, S, n);
}

template <class T>
void launch_t(const LogprobArgs& a, hipStream_t s) {
  constexpr int64_t GRID = 1 << 20;  // workgroups walk the rows beyond
  if (a.C <= 2048) {
    hipLaunchKernelGGL((k_logprob<T, 64, 16 / RowT<T>::VEC, false>), dim3((unsigned)std::min<int64_t>(a.R, GRID)), dim3(64), 0, s, a, 1, a.C);
    return;
  }
  constexpr int CHUNK = 256 * 4 * RowT<T>::VEC;
  int64_t segs = 1;
  if (a.scratch && a.R < 512) segs = std::min<int64_t>((a.C + CHUNK - 1) / CHUNK, std::max<int64_t>(1, 512 / a.R));
  if (segs > 1) {
    const int chunks = (a.C + CHUNK - 1) / CHUNK;
    const int seg = (int)((chunks + segs - 1) / segs) * CHUNK;
    segs = (a.C + seg - 1) / seg;
    hipLaunchKernelGGL((k_logprob<T, 256, 4, true>), dim3((unsigned)(a.R * segs)), dim3(256), 0, s, a, (int)segs, seg);
    hipLaunchKernelGGL((k_logprob_join<T>), dim3((unsigned)a.R), dim3(JOIN_T), 0, s, a, (int)segs);
    return;
  }
  hipLaunchKernelGGL((k_logprob<T, 256, 4, false>), dim3((unsigned)std::min<int64_t>(a.R, GRID)), dim3(256), 0, s, a, 1, a.C);
}

}  // namespace

// At most 512 segments in all, each of a Part and K entries.
static_assert(512 * (sizeof(Part) + MAX_TOP * 8) <= FS_ROW_SCRATCH_BYTES, "scratch");

void launch_logprob(const LogprobArgs& a, Prec p, hipStream_t s) {
  if (p == BF16) launch_t<uint16_t>(a, s);
  else launch_t<float>(a, s);
}

}  // namespace fs
