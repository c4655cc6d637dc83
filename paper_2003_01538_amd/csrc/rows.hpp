// Rows of logits of any length and alignment, and their softmax statistics,
// for the operators that read such rows (log probabilities, distillation).
//
// m is the largest logit, at least the lowest finite number: a row of nothing
// but -inf then sums to 0 instead of NaN, and a finite lowest value (some masks)
// still counts.  s = sum e^((z - m) c) and t = sum e^((z - m) c) (z - m) are kept
// in fp32, c = 1 / temperature.  z - m is formed before the scaling, so the error
// of an exponential follows its distance from the maximum, not the logit's size.
#pragma once

#include <float.h>
#include <math.h>

#include "common.hpp"
#include "device.hpp"

namespace fs {

constexpr float LOG2E = 1.44269504f;
constexpr float FAR = -200.f;  // e^FAR is 0 in fp32: a bound for z - m where it is multiplied by such an exponential

// 16 bytes of a row at any element: the hardware takes vector accesses at
// every byte address.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_at2 __attribute__((aligned(2)));
typedef u32x2 u32x2_at4 __attribute__((aligned(4)));
typedef uint32_t u32_at2 __attribute__((aligned(2)));

template <class T> struct RowT;
template <> struct RowT<float> {
  static constexpr int VEC = 4;
  typedef u32x4_at4 Vec;
  static __device__ __forceinline__ float get(u32x4 v, int e) { return __uint_as_float(v[e]); }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
  static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
  static __device__ __forceinline__ u32x4 pack(const float* f) {
    return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
};
template <> struct RowT<uint16_t> {  // bf16
  static constexpr int VEC = 8;
  typedef u32x4_at2 Vec;
  static __device__ __forceinline__ float get(u32x4 v, int e) {
    return __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
  }
  static __device__ __forceinline__ float one(const uint16_t* p) { return bf2f(*p); }
  static __device__ __forceinline__ void put(uint16_t* p, float v) { *p = f2bf(v); }
  static __device__ __forceinline__ u32x4 pack(const float* f) {
    const uint4 u = f8_to_bf8(f);
    return u32x4{u.x, u.y, u.z, u.w};
  }
};

// Whether a call that moves so many bytes gains by keeping none of them in a cache: well
// beyond the last-level one of 256 MB (distillation with gradients, fp32, 4096 rows of 16384, 537 MB,
// 105 us against 111; 2048 rows, 268 MB, the same tensors again and again, 47 against 46).
inline bool beyond_cache(int64_t bytes) { return bytes > int64_t(400) << 20; }

// A vector of a row.  ONCE: no cache is to keep it.
template <bool ONCE, class T>
__device__ __forceinline__ u32x4 load_vec(const T* p) {
  const auto* v = reinterpret_cast<const typename RowT<T>::Vec*>(p);
  return ONCE ? __builtin_nontemporal_load(v) : *v;
}
template <bool ONCE, class T>
__device__ __forceinline__ void store_vec(T* p, u32x4 v) {
  auto* to = reinterpret_cast<typename RowT<T>::Vec*>(p);
  if (ONCE) __builtin_nontemporal_store(v, to);
  else *to = v;
}

// Elements i .. i + VEC - 1 of a row that ends at `end`; -inf behind the end.  A
// row's last vector is put together from pieces of 4, 2 and 1 elements, the last first.
template <class T>
__device__ __forceinline__ u32x4 row_vec(const T* z, int64_t i, int64_t end) {
  constexpr int VEC = RowT<T>::VEC;
  if (i + VEC <= end) return load_vec<false>(z + i);
  const int r = (int)(end > i ? end - i : 0);
  const T* p = z + i;
  if constexpr (VEC == 8) {
    uint64_t lo = 0xff80ff80ff80ff80ull, hi = lo;  // -inf
    if (r & 1) {
      hi = hi << 16 | lo >> 48;
      lo = lo << 16 | p[r & 6];
    }
    if (r & 2) {
      const uint32_t w = *reinterpret_cast<const u32_at2*>(p + (r & 4));
      hi = hi << 32 | lo >> 32;
      lo = lo << 32 | w;
    }
    if (r & 4) {
      const u32x2 w = *reinterpret_cast<const u32x2_at2*>(p);
      hi = lo;
      lo = w[0] | uint64_t(w[1]) << 32;
    }
    return u32x4{uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32)};
  } else {
    constexpr uint32_t NEG = 0xff800000u;  // -inf
    u32x4 v = {NEG, NEG, NEG, NEG};
    if (r & 1) v[0] = __float_as_uint(p[r & 2]);
    if (r & 2) {
      const u32x2 w = *reinterpret_cast<const u32x2_at4*>(p);
      v = u32x4{w[0], w[1], v[0], NEG};
    }
    return v;
  }
}

// ... and those of the vector's elements that lie before the end, written.
template <class T>
__device__ __forceinline__ void put_vec(T* g, int64_t i, int64_t end, u32x4 v) {
  constexpr int VEC = RowT<T>::VEC;
  if (i + VEC <= end) {
    store_vec<false>(g + i, v);
    return;
  }
  const int r = (int)(end > i ? end - i : 0);
  T* p = g + i;
  if constexpr (VEC == 8) {
    if (r & 4) *reinterpret_cast<u32x2_at2*>(p) = u32x2{v[0], v[1]};
    if (r & 2) *reinterpret_cast<u32_at2*>(p + (r & 4)) = r & 4 ? v[2] : v[0];
    if (r & 1) p[r & 6] = (uint16_t)(r & 4 ? (r & 2 ? v[3] : v[2]) : (r & 2 ? v[1] : v[0]));
  } else {
    if (r & 2) *reinterpret_cast<u32x2_at4*>(p) = u32x2{v[0], v[1]};
    if (r & 1) p[r & 2] = __uint_as_float(r & 2 ? v[2] : v[0]);
  }
}

// NV vectors of a workgroup's chunk of NT * NV vectors that begins at `from`:
// thread t holds vectors t, t + NT, ...
template <class T, int NT, int NV, bool ONCE>
__device__ __forceinline__ void row_chunk(const T* z, int64_t from, int64_t end, u32x4 (&v)[NV]) {
  constexpr int VEC = RowT<T>::VEC;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t i = from + (int64_t)(j * NT + (int)threadIdx.x) * VEC;
    if (from + (int64_t)(j + 1) * NT * VEC <= end) v[j] = load_vec<ONCE>(z + i);  // the same for the whole workgroup
    else v[j] = row_vec(z, i, end);
  }
}

// A row's length, formed again for every row, so that nothing that follows from it
// for a thread's vectors is kept in registers from row to row.
__device__ __forceinline__ int row_end(int C) {
  __asm__ volatile("" : "+s"(C));
  return C;
}

// What a phase made of the vectors (fp32 logits, masks) is formed again in the next
// instead of being kept in registers.
template <int NV>
__device__ __forceinline__ void forget(u32x4 (&v)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) __asm__ volatile("" : "+v"(v[j]));
}

// Wavefront reductions in registers: within rows of 16 lanes, then a row's last
// lane to the next row, then the lower half's to the upper; lane 63 has all.  Six
// steps of a few cycles each, where a shuffle through LDS takes some 60.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp(float keep, float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(keep), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float row_wave_max(float v) {
  v = fmaxf(v, dpp<0x111, 0xf>(v, v));  // row_shr 1, 2, 4, 8
  v = fmaxf(v, dpp<0x112, 0xf>(v, v));
  v = fmaxf(v, dpp<0x114, 0xf>(v, v));
  v = fmaxf(v, dpp<0x118, 0xf>(v, v));
  v = fmaxf(v, dpp<0x142, 0xa>(v, v));  // row_bcast 15 into rows 1 and 3
  v = fmaxf(v, dpp<0x143, 0xc>(v, v));  // row_bcast 31 into rows 2 and 3
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float row_wave_sum(float v) {
  v += dpp<0x111, 0xf>(0.f, v);
  v += dpp<0x112, 0xf>(0.f, v);
  v += dpp<0x114, 0xf>(0.f, v);
  v += dpp<0x118, 0xf>(0.f, v);
  v += dpp<0x142, 0xa>(0.f, v);
  v += dpp<0x143, 0xc>(0.f, v);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Sum over the lanes up to this one.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// Sum or maximum over a workgroup of NT threads, the same in every thread; `sh`
// holds one value per wave and is free again after the call.
template <int NT>
__device__ __forceinline__ float block_sum(float v, float* sh) {
  v = row_wave_sum(v);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) v += sh[w];
    __syncthreads();
  }
  return v;
}
template <int NT>
__device__ __forceinline__ float block_max(float v, float* sh) {
  v = row_wave_max(v);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v = fmaxf(v, sh[w]);
    __syncthreads();
  }
  return v;
}

// Two sums or maxima at the price of one.
template <int NT>
__device__ __forceinline__ void block_max2(float& a, float& b, float (*sh)[2]) {
  a = row_wave_max(a);
  b = row_wave_max(b);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) { sh[threadIdx.x >> 6][0] = a; sh[threadIdx.x >> 6][1] = b; }
    __syncthreads();
    a = sh[0][0]; b = sh[0][1];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) { a = fmaxf(a, sh[w][0]); b = fmaxf(b, sh[w][1]); }
    __syncthreads();
  }
}
template <int NT>
__device__ __forceinline__ void block_sum2(float& a, float& b, float (*sh)[2]) {
  a = row_wave_sum(a);
  b = row_wave_sum(b);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) { sh[threadIdx.x >> 6][0] = a; sh[threadIdx.x >> 6][1] = b; }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) { a += sh[w][0]; b += sh[w][1]; }
    __syncthreads();
  }
}

// Running statistics of the logits that a thread has seen.  k2 = log2(e) c.
// T: whether t is wanted (c is 1 then).
template <bool T>
struct RowStats {
  float m = -FLT_MAX, s = 0.f, t = 0.f;
  // raise the maximum to mn
  __device__ __forceinline__ void lift(float mn, float k2) {
    const float d = m - mn, f = __builtin_amdgcn_exp2f(d * k2);
    if constexpr (T) t = f * (t + fmaxf(d, FAR) * s);
    s *= f;
    m = mn;
  }
  __device__ __forceinline__ void add(float z, float k2) {
    const float d = z - m, e = __builtin_amdgcn_exp2f(d * k2);
    s += e;
    if constexpr (T) t = fmaf(e, fmaxf(d, FAR), t);
  }
  // A chunk's sums are made apart and joined, so that a long row's roundings are those of
  // as many additions as it has chunks rather than classes.
  __device__ __forceinline__ RowStats empty() const {
    RowStats r;
    r.m = m;
    return r;
  }
  __device__ __forceinline__ void join(const RowStats& chunk) {
    s += chunk.s;
    if constexpr (T) t += chunk.t;
  }
  template <int NT>
  __device__ __forceinline__ void over_block(float k2, float (*sh)[2]) {
    lift(block_max<NT>(m, &sh[0][0]), k2);
    if constexpr (T) block_sum2<NT>(s, t, sh);
    else s = block_sum<NT>(s, &sh[0][0]);
  }
};

}  // namespace fs
