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
// candidates to list (the first one; rising rows) a logit that K of the threads'
// maxima reach bounds them: for K <= 40 (and in a wave's own rows) the K-th of 64 groups' maxima, found by
// counting, else one found bit by bit over all of them.  Only if that leaves too
// many, one between the chunk's K-th and LIST-th best is searched bit by bit.
//
// When there are few rows they are cut into segments, one workgroup each; the
// segments' statistics and K best go to the scratch memory, and a second launch
// joins them with the same selection.
//
// What bounds it: memory for many long rows (2048 x 131072 fp32, K = 20, 188 us, 5.7 TB/s),
// the vector ALU for those of bf16 (8000 x 32768 170 to 178 us, 2.9 to 3.1 TB/s), a row's own steps for
// many short ones (100000 x 1000, K = 5, 128 to 135 us in both types; 300000 x 100 223 us), the counting
// of the list for many alternatives (16000 x 1000 fp32, K = 64, 65 us, K = 128 144 us);
// for few the chain of loads, reductions and selection of a workgroup, two of them when
// rows are split (one row of 131072 6.2 + 5.1 us).
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
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ float entry_logit(uint64_t e) { return key_logit(uint32_t(e >> 32)); }
__device__ __forceinline__ int entry_class(uint64_t e) { return int(~uint32_t(e)); }

constexpr int SLACK = 64;  // entries that the list grows by before it is cut

template <int NT>
struct Selection {
  static constexpr int LIST = NT == 64 ? 512 : 1024;
  __attribute__((aligned(16))) uint64_t list[LIST + 8];
  uint64_t top[MAX_TOP];
  float maxima[NT];
  __attribute__((aligned(16))) float group[NT / 64][64];
  int hits[3], n, count[NT / 64];
};

// What a workgroup knows of its selection, the same in every thread: the K-th
// best logit so far (-inf: fewer than K), the list's length, whether the list is
// cut (at most K entries in falling order), and the number of chunks seen.
struct Progress {
  float bar = -INFINITY;
  int n = 0;
  bool sorted = true;
  int turn = 0;
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

// Cut the list to the K best, in falling order: an entry's place is the number of
// those before it.  Every thread has seen p.n.
template <int NT>
__device__ __forceinline__ void cut(Selection<NT>& S, Progress& p, int K) {
  if (p.sorted) return;
  const int n = p.n;
  if (threadIdx.x < 8) S.list[n + threadIdx.x] = 0;  // comes after every entry
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += NT) {
    const uint64_t own = S.list[i];
    int rank = 0;
    for (int j = 0; j < n; j += 8) {
      uint64_t e[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) e[u] = S.list[j + u];
#pragma unroll
      for (int u = 0; u < 8; ++u) rank += e[u] > own ? 1 : 0;
    }
    if (rank < K) S.top[rank] = own;
  }
  __syncthreads();
  p.n = min(n, K);
  for (int i = threadIdx.x; i < p.n; i += NT) S.list[i] = S.top[i];
  if (threadIdx.x == 0) S.n = p.n;
  p.sorted = true;
  __syncthreads();
}

// The K-th largest of the 64 lanes' values, K <= 64; `own`: the wave's 64 floats, aligned to 16 bytes.
__device__ __forceinline__ float kth_of_wave(float g, int K, float* own) {
  own[threadIdx.x & 63] = g;
  int before = 0;
#pragma unroll
  for (int i = 0; i < 64; i += 4) {
    const floatx4 q = *reinterpret_cast<const floatx4*>(own + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) before += q[e] > g ? 1 : 0;
  }
  return -row_wave_max(before < K ? -g : -INFINITY);
}

// a[j] of registers, by halving with masks (as a choice of elements the compiler
// makes it a comparison with every index for every step)
template <int N>
__device__ __forceinline__ uint32_t pick(const uint32_t (&a)[N], int j) {
  uint32_t t[N];
#pragma unroll
  for (int i = 0; i < N; ++i) t[i] = a[i];
#pragma unroll
  for (int s = N / 2; s > 0; s /= 2) {
    const uint32_t m = j & s ? ~0u : 0u;
#pragma unroll
    for (int i = 0; i < s; ++i) t[i] = (t[i + s] & m) | (t[i] & ~m);
  }
  return t[0];
}

// The largest number of which count() says at least K, searched from the highest
// bit down; ends early once count() says at most `most`.  It lies in lo .. hi.
template <class Count>
__device__ __forceinline__ uint32_t search(uint32_t lo, uint32_t hi, int K, int most, Count&& count) {
  const int bits = lo == hi ? 0 : 32 - __builtin_clz(lo ^ hi);  // those above are the same
  uint32_t x = bits == 32 ? 0 : lo >> bits << bits;
  for (int bit = bits - 1; bit >= 0; --bit) {
    const int c = count(x | 1u << bit);
    if (c < K) continue;
    x |= 1u << bit;
    if (c <= most) break;
  }
  return x;
}

// One chunk's candidates into the list.  get(j, z, c): this thread's j-th of NE
// logits and its class, entry_of(j) the same as an entry for a j that is not a
// constant; best: the largest of them (-inf: none).  TIES: a logit equal to the bar may
// be of a lower class than those before it, so it is a candidate too.
template <int NT, int NE, bool TIES, class Get, class EntryOf>
__device__ __forceinline__ void select_chunk(Selection<NT>& S, Progress& p, int K, float best, Get&& get, EntryOf&& entry_of) {
  constexpr int LIST = Selection<NT>::LIST;
  const int lane = threadIdx.x & 63, turn = p.turn++;
  const uint64_t wave_hits = __ballot(best > p.bar || (TIES && best == p.bar && best > -INFINITY));
  int hits;
  if constexpr (NT == 64) {
    hits = (int)__popcll(wave_hits);
  } else {
    // three counters in turn: the one of two calls on is cleared while no wave can be there yet
    if (wave_hits && lane == 0) atomicAdd(&S.hits[turn % 3], (int)__popcll(wave_hits));
    if (turn == 0) S.maxima[threadIdx.x] = best;
    __syncthreads();
    hits = S.hits[turn % 3];
    if (threadIdx.x == 0) S.hits[(turn + 2) % 3] = 0;
  }
  if (hits == 0) return;

  // candidates: z >= from, the bar or the logit next above it
  float from = TIES && p.bar > -INFINITY ? p.bar : key_logit(order_key(p.bar) + 1);
  const bool many = p.n + hits * NE > LIST || (NT == 64 && hits > K);  // a wave finds a threshold in less time than it ranks a long list
  if (many) {
    cut(S, p, K);
    // a logit that K or a few more of the threads' maxima reach, of groups of threads if those are enough
    if (hits >= K) {
      float q[NT / 64], g;  // the maxima; the largest of each group of NT / 64
      if constexpr (NT == 64) {
        g = q[0] = best;
      } else {
        if (turn > 0) {
          S.maxima[threadIdx.x] = best;
          __syncthreads();
        }
        g = -INFINITY;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) {
          q[w] = S.maxima[w * 64 + lane];
          g = fmaxf(g, q[w]);
        }
      }
      if (K <= (NT == 64 ? 64 : 40) && (int)__popcll(__ballot(g >= from)) >= K) {
        from = fmaxf(from, kth_of_wave(g, K, S.group[threadIdx.x >> 6]));
      } else {
        const uint32_t k = search(order_key(from), order_key(row_wave_max(g)), K, K + (K >> 3) + 2, [&](uint32_t k) {
          int c = 0;
#pragma unroll
          for (int w = 0; w < NT / 64; ++w) c += (int)__popcll(__ballot(q[w] >= key_logit(k)));
          return c;
        });
        from = fmaxf(from, key_logit(k));
      }
    }
  }
  // list them, all of a wave's in one place; false: there is no room for them
  auto list = [&](auto&& takes) {
    uint32_t mine = 0;  // bit j: this thread's j-th logit
#pragma unroll
    for (int j = 0; j < NE; ++j) {
      float z;
      int c;
      get(j, z, c);
      mine |= (takes(z, c) ? 1u : 0u) << j;
    }
    const int count = __popc(mine), upto = wave_scan(count), all = __builtin_amdgcn_readlane(upto, 63);
    if (all == 0) return;
    int at = 0;
    if (lane == 0) at = atomicAdd(&S.n, all);
    at = __builtin_amdgcn_readfirstlane(at);
    if (at + all > LIST) return;  // seen below, by every thread
    at += upto - count;
    while (__ballot(mine != 0))  // mostly one or two of a thread's logits
      if (mine) {
        S.list[at++] = entry_of(__ffs(mine) - 1);
        mine &= mine - 1;
      }
  };
  static_assert(NE <= 32, "a bit for each logit");
  if (many || wave_hits) list([&](float z, int) { return z >= from; });
  __syncthreads();
  if (many && S.n > LIST) {
    // the K-th best logit of the chunk, and of those equal to it the lowest classes
    const int most = LIST - p.n;
    __syncthreads();
    if (threadIdx.x == 0) S.n = p.n;
    auto reach = [&](float x, uint32_t last) {
      __asm__ volatile("" : "+v"(x));  // keeps the comparisons of a rare path out of the registers of the common one
      int n = 0;
#pragma unroll
      for (int j = 0; j < NE; ++j) {
        float z;
        int c;
        get(j, z, c);
        n += (int)__popcll(__ballot(z > x || (z == x && uint32_t(c) <= last)));
      }
      return block_count<NT>(n, S.count);
    };
    const uint32_t top = order_key(INFINITY);  // keys above are no logit's
    const float kth = key_logit(search(order_key(from), top, K, most, [&](uint32_t k) { return k > top ? 0 : reach(fmaxf(from, key_logit(k)), ~0u); }));
    from = fmaxf(from, kth);
    const uint32_t last = ~search(0, ~0u, K, most, [&](uint32_t k) { return reach(from, ~k); });
    __syncthreads();
    list([&](float z, int c) { return z > from || (z == from && uint32_t(c) <= last); });
    __syncthreads();
  }
  p.n = S.n;
  p.sorted = false;
  if (p.n >= K + SLACK || many) cut(S, p, K);
  if (p.sorted && p.n == K) p.bar = entry_logit(S.list[K - 1]);
}

template <int NT>
__device__ __forceinline__ void select_begin(Selection<NT>& S) {
  if (threadIdx.x == 0) S.hits[0] = S.hits[1] = S.hits[2] = S.n = 0;
  __syncthreads();
}

// ln p of the given classes, entropy and alternatives of a row from its statistics and its list.
// `mine`: given_logit of this thread's first given class, loaded before the walk.
template <class T>
__device__ __forceinline__ float given_logit(const LogprobArgs& a, int64_t row, const T* z, int i) {
  if (i >= a.T) return -INFINITY;
  const int c = a.classes[row * a.T + i];
  return c >= 0 && c < a.C ? RowT<T>::one(z + c) : -INFINITY;
}
template <class T, int NT>
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t row, const T* z, float mine, const RowStats<true>& st,
                                          Selection<NT>& S, int n) {
  const float ls = logf(st.s);
  if (a.entropy && threadIdx.x == 0) a.entropy[row] = st.s == 0.f ? 0.f : ls - st.t / st.s;
  for (int i = threadIdx.x; i < a.T; i += NT) {
    const float v = i < NT ? mine : given_logit(a, row, z, i);
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
template <class T, int NT, int NV, bool SPLIT, bool ONCE>
__global__ void __launch_bounds__(NT) k_logprob(LogprobArgs a, int segs, int seg) {
  using RT = RowT<T>;
  constexpr int VEC = RT::VEC, NE = NV * VEC, CHUNK = NT * NE;
  __shared__ Selection<NT> S;
  __shared__ float sh[NT / 64][2];
  const int64_t items = (int64_t)a.R * segs;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t row = SPLIT ? item / segs : item;
    const int64_t first = SPLIT ? (item - row * segs) * seg : 0;
    const int64_t end = SPLIT ? min((int64_t)a.C, first + seg) : row_end(a.C);
    const T* z = static_cast<const T*>(a.z) + row * a.ld;
    select_begin(S);
    RowStats<true> st;
    Progress p;
    u32x4 v[NV], next[NV];
    row_chunk<T, NT, NV, ONCE>(z, first, end, v);
    const float mine = SPLIT ? 0.f : given_logit(a, row, z, threadIdx.x);
    for (int64_t from = first; from < end; from += CHUNK) {
      const bool more = from + CHUNK < end;
      if (more) row_chunk<T, NT, NV, ONCE>(z, from + CHUNK, end, next);
      float best = -INFINITY;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) best = fmaxf(best, RT::get(v[j], e));
      if (best > st.m) st.lift(best, LOG2E);
      RowStats<true> part = st.empty();
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) part.add(RT::get(v[j], e), LOG2E);
      st.join(part);
      if (a.K > 0) {
        const int base = (int)from + (int)threadIdx.x * VEC;
        select_chunk<NT, NE, false>(S, p, a.K, best, [&](int j, float& x, int& c) {
          int at = base;
          u32x4 raw = v[j / VEC];
          __asm__ volatile("" : "+v"(at), "+v"(raw));  // classes and fp32 logits are formed where they are used, not kept
          x = RT::get(raw, j % VEC);
          c = at + j / VEC * NT * VEC + j % VEC;
        }, [&](int j) {
          uint32_t words[NV * 4];
#pragma unroll
          for (int i = 0; i < NV * 4; ++i) words[i] = v[i / 4][i % 4];
          const uint32_t w = pick(words, j * 4 / VEC);
          const float x = VEC == 4 ? __uint_as_float(w) : __uint_as_float(j & 1 ? w & 0xffff0000u : w << 16);
          return entry(x, base + j / VEC * NT * VEC + j % VEC);
        });
      }
      if (more)
#pragma unroll
        for (int j = 0; j < NV; ++j) v[j] = next[j];
    }
    cut(S, p, a.K);
    st.over_block<NT>(LOG2E, sh);
    if constexpr (SPLIT) {
      Part* part = static_cast<Part*>(a.scratch) + item;
      uint64_t* list = reinterpret_cast<uint64_t*>(static_cast<Part*>(a.scratch) + items) + item * a.K;
      if (threadIdx.x == 0) *part = Part{st.m, st.s, st.t, p.n};
      for (int i = threadIdx.x; i < a.K; i += NT) list[i] = i < p.n ? S.list[i] : 0;
    } else {
      write_row<T, NT>(a, row, z, mine, st, S, p.n);
    }
    __syncthreads();
  }
}

constexpr int JOIN_T = 256, JOIN_E = 8;

// The segments of a row, joined.  The best of every segment come first, so that
// the threads' first entries are the largest.
template <class T>
__global__ void __launch_bounds__(JOIN_T) k_logprob_join(LogprobArgs a, int segs) {
  __shared__ Selection<JOIN_T> S;
  __shared__ float sh[JOIN_T / 64][2];
  const int64_t row = blockIdx.x;
  const Part* part = static_cast<const Part*>(a.scratch) + row * segs;
  const uint64_t* list = reinterpret_cast<const uint64_t*>(static_cast<const Part*>(a.scratch) + (int64_t)a.R * segs) + row * segs * a.K;
  const T* z = static_cast<const T*>(a.z) + row * a.ld;
  const int entries = segs * a.K;
  uint64_t e[JOIN_E];
  auto load = [&](int from) {
#pragma unroll
    for (int j = 0; j < JOIN_E; ++j) {
      const int i = from + j * JOIN_T + threadIdx.x;
      e[j] = i < entries ? list[(i % segs) * a.K + i / segs] : 0;
    }
  };
  load(0);
  const float mine = given_logit(a, row, z, threadIdx.x);
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
  Progress p;
  for (int from = 0; from < entries; from += JOIN_T * JOIN_E) {
    if (from > 0) load(from);
    float best = -INFINITY;
#pragma unroll
    for (int j = 0; j < JOIN_E; ++j)
      if (e[j]) best = fmaxf(best, entry_logit(e[j]));
    select_chunk<JOIN_T, JOIN_E, true>(S, p, a.K, best, [&](int j, float& x, int& c) {
      x = e[j] ? entry_logit(e[j]) : -INFINITY;
      c = entry_class(e[j]);
    }, [&](int j) {
      uint32_t lo[JOIN_E], hi[JOIN_E];
#pragma unroll
      for (int i = 0; i < JOIN_E; ++i) {
        lo[i] = uint32_t(e[i]);
        hi[i] = uint32_t(e[i] >> 32);
      }
      return uint64_t(pick(hi, j)) << 32 | pick(lo, j);
    });
  }
  cut(S, p, a.K);
  st.over_block<JOIN_T>(LOG2E, sh);
  write_row<T, JOIN_T>(a, row, z, mine, st, S, p.n);
}

constexpr int SEGS = 1024;  // segments of all rows that are split

template <class T, int NT, int NV>
void whole(const LogprobArgs& a, hipStream_t s) {
  constexpr int64_t GRID = 1 << 20;  // workgroups walk the rows beyond
  const dim3 grid((unsigned)std::min<int64_t>(a.R, GRID));
  // more than the last-level cache holds is not kept there: 2048 x 131072 fp32 204 us against 197
  if (NT <= 256 && beyond_cache((int64_t)a.R * a.C * (int)sizeof(T))) hipLaunchKernelGGL((k_logprob<T, NT, NV, false, NT <= 256>), grid, dim3(NT), 0, s, a, 1, a.C);
  else hipLaunchKernelGGL((k_logprob<T, NT, NV, false, false>), grid, dim3(NT), 0, s, a, 1, a.C);
}

template <class T>
void launch_t(const LogprobArgs& a, hipStream_t s) {
  constexpr int VEC = RowT<T>::VEC, NV = 16 / VEC;  // 16 logits a thread at a time: with 32, registers limit the waves (bf16, 2048 x 131072: 258 us against 179)
  // a wave per row for short or many rows, as long as its 64 maxima tell the K best from the
  // rest (fp32: 96 rows of 1000, K = 5, 4.8 us against 5.4 with two waves; 60000 of 2049, K = 16,
  // 151 against 205 and, with four, 338; 8000 of 32768 199 against 209 and 221; 16000 of 1000 at K = 41
  // 35 against 61, at K = 64 158 against 66), with no more logits a thread than the row has
  // (300000 rows of 100 218 us with 4, 370 with 16).  Many rows that fit it with 4 go so for any K
  // (300000 of 100 at K = 64 368 us against 914 with two waves of 16 logits, at K = 128 383 against 1763
  // with four; 1000 of 250 at K = 64 18 against 13).
  if (a.C <= 64 * VEC && (a.K <= 48 || a.R >= 4000)) return whole<T, 64, 1>(a, s);
  if (a.K <= 48) {
    if (a.C <= 128 * VEC && NV > 2) return whole<T, 64, 2>(a, s);
    if (a.C <= 2048 || a.R >= 4000) return whole<T, 64, NV>(a, s);
  }
  // two waves for fewer rows or more alternatives (2000 of 10000, K = 20, 28 us against 32 with one
  // or four; 2000 of 1000, K = 64, 12 against 19 with four; 16000 of 1000 at K = 128 628 against 146)
  if (a.K <= 80 && (a.C <= 2048 || a.R >= 2000)) return whole<T, 128, NV>(a, s);
  // few long rows in segments, down to the numbers of rows where whole ones take as long
  // (fp32, K = 20: one row of 131072 classes 10.7 us against 29.4, 61 rows 21 against 35, 200
  // rows 38 against 39; of 32000 10.4 against 11.7, 61 rows 12.9 against 13.1, 128 rows 15.1
  // against 14.0; one row of 16384 9.9 against 8.0)
  constexpr int CHUNK = 256 * 16;
  if (a.scratch && a.C > 16384 && a.R < (a.C > 32768 ? 200 : 100)) {
    const int chunks = (a.C - 1) / CHUNK + 1, most = std::min(chunks, SEGS / a.R);
    const int seg = (chunks - 1) / most + 1, segs = (chunks - 1) / seg + 1;
    if (segs > 1) {
      hipLaunchKernelGGL((k_logprob<T, 256, NV, true, false>), dim3((unsigned)(a.R * segs)), dim3(256), 0, s, a, segs, seg * CHUNK);
      hipLaunchKernelGGL((k_logprob_join<T>), dim3((unsigned)a.R), dim3(JOIN_T), 0, s, a, segs);
      return;
    }
  }
  // four waves per row, more when there are too few rows for the chip (fp32, K = 20: one
  // row of 8192 8.2 us with 16 waves, 6.1 with 8, 7.9 with 4; 256 rows of 131072 44, 52 and
  // 79; 512 rows 76, 64 and 82; 1000 rows of 10000 34, 23 and 18)
  if (a.R < 512 && a.C > 8192) return whole<T, 1024, NV>(a, s);
  if ((a.R < 512 && a.C > 4096) || (a.R < 1024 && a.C > 32768)) return whole<T, 512, NV>(a, s);
  return whole<T, 256, NV>(a, s);
}

}  // namespace

// A Part and K entries of each segment.
static_assert(SEGS * (sizeof(Part) + MAX_TOP * 8) <= FS_ROW_SCRATCH_BYTES, "scratch");

void launch_logprob(const LogprobArgs& a, Prec p, hipStream_t s) {
  if (p == BF16) launch_t<uint16_t>(a, s);
  else launch_t<float>(a, s);
}

}  // namespace fs
