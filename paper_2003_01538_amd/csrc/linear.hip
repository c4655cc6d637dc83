// Matrix product with bias, activation and residual on a caller's tensors:
// y[m][n] = act(sum_k x[m][k] w[n][k] + bias[n] (+ res)) (+ res).
//
// Five kernels.  k_linear_few is for outputs of few tiles: a workgroup makes a
// small tile, 16 x 16 to 64 x 32, and its waves split the reduction, each loading its operands
// straight into registers (nothing is shared, so nothing is staged), and their
// sums meet in LDS in wave order.  k_linear_stream is its form for up to 64 aligned
// rows.  k_linear_tile is for many tiles: operands go through LDS, each wave sums
// its part of the tile over the whole reduction.  fp32, whose matrix instructions take
// eight times as long, has two of its own besides, which bring whole lines through
// registers and LDS: k_linear_wave for few tiles, k_linear_mid for tiles of 32 x 32 to 128 x 64.
// Rows may lie at any distance and alignment; which kernel runs, with which tile, is a rule on
// sizes and alignment (launch_t).
//
// What bounds them: up to 16 rows the weights' way from memory (4096 features, K =
// 25088, bf16, one row 37 us, 5.5 TB/s); up to 64 rows that of x from L2 to every
// workgroup (32 rows 51 us, 12 TB/s); bf16 products of 4096 x 8192 x 4096 the power
// that the matrix cores may take (216 to 229 us, 1.20 to 1.27 PFLOP/s, with their pipes
// busy 73 % of the time at 1.7 GHz; the vendor's library 180 to 189 us; 238 to 256 us with GELU and
// residual); fp32 products the matrix cores' rate (4096^3 947 us, 145 TFLOP/s; rows 3 elements
// apart 1010 to 1041 us), mid-sized ones the rest of the last round of tiles (580 x 1891, K = 4785, 130
// us, 81 TFLOP/s), long reductions over few outputs what a CU brings from L2, 50 to 100 GB/s
// (74 x 128, K = 18816, 28 us).
//
// MFMA operands: A = weights, B = x, so that a lane's accumulators hold
// consecutive features n of one row m.  The order of k inside a 16-byte piece
// and between the pieces of a step is free as long as both operands share it.
#include "common.hpp"
#include "device.hpp"
#include "lds_dma.hpp"

#include "flexserve.h"

#include <algorithm>

namespace fs {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
typedef u32x2 u32x2_at2 __attribute__((aligned(2)));
typedef floatx4 floatx4_at4 __attribute__((aligned(4)));

template <class T> struct LinT;
template <> struct LinT<uint16_t> {  // bf16
  static constexpr int VEC = 8;
  static __device__ __forceinline__ floatx4 mma16(u32x4 w, u32x4 x, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
  }
  static __device__ __forceinline__ floatx16 mma32(u32x4 w, u32x4 x, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
  }
};
template <> struct LinT<float> {
  static constexpr int VEC = 4;
  static __device__ __forceinline__ floatx4 mma16(u32x4 w, u32x4 x, floatx4 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[e]), __uint_as_float(x[e]), c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ floatx16 mma32(u32x4 w, u32x4 x, floatx16 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w[e]), __uint_as_float(x[e]), c, 0, 0, 0);
    return c;
  }
};

// 16 bytes of a row at any element: the hardware takes vector accesses at every byte
// address, but those between two words (bf16 rows an odd number of elements apart) at down
// to a third of the rate.  ODD: some rows lie so; the words that hold the 16 bytes are
// loaded, and shifted when they have arrived.  (The halves of words beside the 16 bytes
// go nowhere; no word is loaded that holds nothing of the row.)  In k_linear_tile, whose
// loads have a K-tile's time, this gained nothing (4096^3 227 us against 214).
template <bool ODD> struct Piece {
  u32x4 v;
  template <class T> __device__ __forceinline__ void load(const T* at) { v = *reinterpret_cast<const u32x4_at4*>(at); }
  __device__ __forceinline__ u32x4 get() const { return v; }
};
template <> struct Piece<true> {
  u32x4 v;
  uint32_t last, shift;
  template <class T> __device__ __forceinline__ void load(const T* at) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(at), odd = a & 2;
    v = *reinterpret_cast<const u32x4_at4*>(a - odd);
    last = *reinterpret_cast<const uint32_t*>(a - odd + 12 + 2 * odd);  // the fourth word again, or the one behind it
    shift = uint32_t(odd) * 8;
  }
  __device__ __forceinline__ u32x4 get() const {
    return u32x4{__builtin_amdgcn_alignbit(v[1], v[0], shift), __builtin_amdgcn_alignbit(v[2], v[1], shift),
                 __builtin_amdgcn_alignbit(v[3], v[2], shift), __builtin_amdgcn_alignbit(last, v[3], shift)};
  }
};

// 16 bytes with zeros behind the row's end: the last 16 bytes of the row, shifted.
template <class T>
__device__ __forceinline__ u32x4 piece(const T* row, int k, int K) {
  constexpr int VEC = LinT<T>::VEC;
  if (K < VEC) {  // no 16 bytes to load
    T t[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) t[e] = k + e < K ? row[k + e] : T(0);
    return __builtin_bit_cast(u32x4, t);
  }
  const int from = min(k, K - VEC), bits = min(k - from, VEC) * (int)sizeof(T) * 8;
  const u32x4 v = *reinterpret_cast<const u32x4_at2*>(row + from);
  const uint64_t lo = v[0] | uint64_t(v[1]) << 32, hi = v[2] | uint64_t(v[3]) << 32;
  uint64_t l = lo, h = hi;
  if (bits >= 128) {
    l = h = 0;
  } else if (bits >= 64) {
    l = hi >> (bits - 64);
    h = 0;
  } else if (bits > 0) {
    l = lo >> bits | hi << (64 - bits);
    h = hi >> bits;
  }
  return u32x4{uint32_t(l), uint32_t(l >> 32), uint32_t(h), uint32_t(h >> 32)};
}

// 64 lanes' 16 bytes at their offsets to LDS, in lane order.
__device__ __forceinline__ void load_lds(__amdgpu_buffer_rsrc_t r, char* to, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)to, 16, off, 0, 0, 0);
}

// e^(-x), or 2^(-x) for x in units of ln 2, where F32 asks for its error not to grow with
// x: what the rounding of hi = x log2(e) left out (lo) enters as a factor 1 - lo ln 2.
template <bool F32>
__device__ __forceinline__ float exp_of(float hi, float lo) {
  const float e = __builtin_amdgcn_exp2f(-hi);
  return F32 ? e * fmaf(-0.693147182f, lo, 1.f) : e;
}

// v Phi(v).  Phi(-x) = e^(-x^2 / 2) R(x), R the normal distribution's Mills ratio over
// sqrt(2 pi), as u P(u) with u = 1 / (1 + 0.305 x): P is the polynomial of degree 7 with the
// least largest relative error on 0 <= x <= 14.2, 9.4e-8 (a linear programme on Chebyshev
// points).  So the error is relative down to the last normal number: 10 steps of 2^-24 for
// fp32 outputs, and for bf16 ones, whose exponent's rounding stays (1.1e-5 at x = 13.2), far
// below half a step.  4096 x 8192 bf16 outputs of K = 4096 take 243 to 250 us, as with a
// shorter fit of erf, whose error is absolute (1.5e-7: of gelu(-8) 1e-2); erff took 80 us more.
template <bool F32>
__device__ __forceinline__ float gelu(float v) {
  const float x = fminf(fabsf(v), 20.f), u = __builtin_amdgcn_rcpf(fmaf(0.305f, x, 1.f));
  float p = 0.036699425f;
  p = fmaf(p, u, -0.15298922f);
  p = fmaf(p, u, 0.18571836f);
  p = fmaf(p, u, -0.037978083f);
  p = fmaf(p, u, 0.12102229f);
  p = fmaf(p, u, 0.1034207f);
  p = fmaf(p, u, 0.12246685f);
  p = fmaf(p, u, 0.121639736f);
  const float c = 0.72134752f, sq = x * x, hi = sq * c;  // log2(e) / 2
  float lo = 0.f;
  if (F32) lo = fmaf(sq, c, -hi) + fmaf(fmaf(x, x, -sq), c, sq * 9.63e-9f);
  const float q = p * u * exp_of<F32>(hi, lo);  // Phi(-|v|)
  return v * (v < 0.f ? q : 1.f - q);
}

// v / (1 + e^-v); beyond +-200 the exponential is 0 or infinite.
template <bool F32>
__device__ __forceinline__ float silu(float v) {
  const float c = 1.44269504f, x = F32 ? fminf(fmaxf(v, -200.f), 200.f) : v, hi = x * c;
  return v * __builtin_amdgcn_rcpf(1.f + exp_of<F32>(hi, F32 ? fmaf(x, c, -hi) + x * 1.926e-8f : 0.f));
}

// F32: the type of what is made of it.
template <bool F32>
__device__ __forceinline__ floatx4 activate(floatx4 v, int act) {
  if (act == FS_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = v[e] > 0.f ? v[e] : 0.f;
  } else if (act == FS_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = gelu<F32>(v[e]);
  } else if (act == FS_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = silu<F32>(v[e]);
  }
  return v;
}

// Bias, residual and activation, in fp32.
template <bool F32>
__device__ __forceinline__ floatx4 epilogue(const LinearArgs& a, floatx4 v, floatx4 bias, floatx4 res) {
  v += bias;
  if (a.res_first) v += res;
  v = activate<F32>(v, a.act);
  if (a.res && !a.res_first) v += res;
  return v;
}

// Four outputs or residuals at any element: raw as loaded, widened, narrowed and stored.
template <bool F32> struct Out4 {
  typedef floatx4 Raw;
  static __device__ __forceinline__ Raw load(const void* p, int64_t o) { return *reinterpret_cast<const floatx4_at4*>(static_cast<const float*>(p) + o); }
  static __device__ __forceinline__ floatx4 wide(Raw r) { return r; }
  static __device__ __forceinline__ void store(void* p, int64_t o, floatx4 v) { *reinterpret_cast<floatx4_at4*>(static_cast<float*>(p) + o) = v; }
};
template <> struct Out4<false> {
  typedef u32x2 Raw;
  static __device__ __forceinline__ Raw load(const void* p, int64_t o) { return *reinterpret_cast<const u32x2_at2*>(static_cast<const uint16_t*>(p) + o); }
  static __device__ __forceinline__ floatx4 wide(Raw q) {
    return floatx4{__uint_as_float(q[0] << 16), __uint_as_float(q[0] & 0xffff0000u), __uint_as_float(q[1] << 16), __uint_as_float(q[1] & 0xffff0000u)};
  }
  static __device__ __forceinline__ void store(void* p, int64_t o, floatx4 v) {
    *reinterpret_cast<u32x2_at2*>(static_cast<uint16_t*>(p) + o) = __builtin_bit_cast(u32x2, __builtin_convertvector(v, bf16x4));
  }
};

// The bias of features n .. n + 3, 0 for those that do not exist.
struct Bias4 {
  floatx4 v = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ Bias4(const LinearArgs& a, int n) {
    if (!a.bias) return;
    if (n + 4 <= a.N) {
      v = *reinterpret_cast<const floatx4_at4*>(a.bias + n);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < a.N) v[e] = a.bias[n + e];
    }
  }
};

// The residual of outputs (m, n .. n + 3), 0 for those that do not exist.
__device__ __forceinline__ floatx4 residual4(const LinearArgs& a, int m, int n) {
  floatx4 r = {0.f, 0.f, 0.f, 0.f};
  if (!a.res || m >= a.M) return r;
  const int64_t o = (int64_t)m * a.ldres + n;
  const float* const f = static_cast<const float*>(a.res) + o;
  const uint16_t* const h = static_cast<const uint16_t*>(a.res) + o;
  if (n + 4 <= a.N) return a.out_f32 ? Out4<true>::load(a.res, o) : Out4<false>::wide(Out4<false>::load(a.res, o));
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < a.N) r[e] = a.out_f32 ? f[e] : bf2f(h[e]);
  return r;
}

// Those of outputs (m, n .. n + 3) that exist, from their sums.
__device__ __forceinline__ void finish4(const LinearArgs& a, int m, int n, floatx4 v, const Bias4& bias, floatx4 res) {
  if (m >= a.M || n >= a.N) return;
  v = a.out_f32 ? epilogue<true>(a, v, bias.v, res) : epilogue<false>(a, v, bias.v, res);
  const int64_t o = (int64_t)m * a.ldy + n;
  if (n + 4 <= a.N) {
    if (a.out_f32) Out4<true>::store(a.y, o, v);
    else Out4<false>::store(a.y, o, v);
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < a.N) {
      if (a.out_f32) static_cast<float*>(a.y)[o + e] = v[e];
      else static_cast<uint16_t*>(a.y)[o + e] = f2bf(v[e]);
    }
}

// --------------------------------------------------------------- few tiles
// A tile of 16 FN features x 16 FM rows.  Step s of the reduction is a run of
// 128 bytes of each row: lane group g = lane / 16 takes 32 of them in two
// pieces, so that a step's loads use whole cache lines.  Wave w takes steps w,
// w + NW, ..., U of them in flight.
template <class T, int FM, int FN, int NW, int U, bool ODD>
__global__ void __launch_bounds__(NW * 64) k_linear_few(LinearArgs a) {
  using L = LinT<T>;
  constexpr int VEC = L::VEC, STEP = 8 * VEC;
  __shared__ floatx4 part[NW][FM * FN][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tiles_n = (a.N + 16 * FN - 1) / (16 * FN);
  const int n0 = blockIdx.x % tiles_n * (16 * FN), m0 = blockIdx.x / tiles_n * (16 * FM);
  const int off = (lane >> 4) * 2 * VEC;
  // rows that do not exist read row 0: they enter only outputs that do not exist
  const T* wr[FN];
  const T* xr[FM];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int n = n0 + j * 16 + (lane & 15);
    wr[j] = static_cast<const T*>(a.w) + (int64_t)(n < a.N ? n : 0) * a.ldw;
  }
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int m = m0 + i * 16 + (lane & 15);
    xr[i] = static_cast<const T*>(a.x) + (int64_t)(m < a.M ? m : 0) * a.ldx;
  }
  // the outputs that this thread finishes: block (i, j) of 16 x 16, in which lane l
  // holds row l % 16 and features 4 (l / 16) ..
  static_assert(FM * FN <= NW, "a block per wave");
  const int om = m0 + wave / FN * 16 + (lane & 15), on = n0 + wave % FN * 16 + (lane >> 4) * 4;
  const bool finishes = wave < FM * FN;
  const Bias4 bias(a, finishes ? on : a.N);
  const floatx4 res = residual4(a, finishes ? om : a.M, on);

  floatx4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

  auto products = [&](const u32x4 (&w)[FN][2], const u32x4 (&x)[FM][2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = L::mma16(w[j][h], x[i][h], acc[i][j]);
  };
  u32x4 w[FN][2], x[FM][2];
  int k = wave * STEP;
  for (; k + (U - 1) * NW * STEP + STEP <= a.K; k += U * NW * STEP) {
    Piece<ODD> pw[U][FN][2], px[U][FM][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int ku = k + u * NW * STEP + off;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int j = 0; j < FN; ++j) pw[u][j][h].load(wr[j] + ku + h * VEC);
#pragma unroll
        for (int i = 0; i < FM; ++i) px[u][i][h].load(xr[i] + ku + h * VEC);
      }
    }
    __builtin_amdgcn_sched_barrier(0);  // all loads are under way before the first product waits
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int j = 0; j < FN; ++j) w[j][h] = pw[u][j][h].get();
#pragma unroll
        for (int i = 0; i < FM; ++i) x[i][h] = px[u][i][h].get();
      }
      products(w, x);
    }
  }
  for (; k < a.K; k += NW * STEP) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < FN; ++j) w[j][h] = piece(wr[j], k + off + h * VEC, a.K);
#pragma unroll
      for (int i = 0; i < FM; ++i) x[i][h] = piece(xr[i], k + off + h * VEC, a.K);
    }
    products(w, x);
  }

#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) part[wave][i * FN + j][lane] = acc[i][j];
  __syncthreads();
  if (!finishes) return;
  floatx4 s = part[0][wave][lane];
#pragma unroll
  for (int q = 1; q < NW; ++q) s += part[q][wave][lane];
  finish4(a, om, on, s, bias, res);
}

// The same for up to 64 aligned rows, where time is that of bringing x to every
// workgroup out of L2.  Each wave brings its own steps through LDS by loads
// that write it: those take whole 128-byte lines of 8 rows, where the loads into
// registers take half lines of 16.  Nothing is shared between the waves, so there is no
// barrier: a wave waits for its own loads, S steps of which are on their way.
template <class T, int FM, int NW, int S>
__global__ void __launch_bounds__(NW * 64) k_linear_stream(LinearArgs a) {
  using L = LinT<T>;
  constexpr int VEC = L::VEC, STEP = 8 * VEC, ES = sizeof(T);
  constexpr int STAGE = (1 + FM) * 16 * ROW, LOADS = 2 * (1 + FM);  // bytes and load instructions of a step
  static_assert(S * STAGE >= FM * 1024, "the sums fit where the steps were");
  __shared__ __attribute__((aligned(1024))) char lds[NW * S * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16;
  const int steps = (a.K + STEP - 1) / STEP;
  char* const own = lds + wave * S * STAGE;

  // load p fills rows 8 p .. of the stage (16 of w, then x), chunks as in lds_dma.hpp;
  // rows that do not exist read the last one
  const __amdgpu_buffer_rsrc_t rw = rsrc(static_cast<const T*>(a.w) + (int64_t)n0 * a.ldw, (uint32_t)(((min(16, a.N - n0) - 1) * a.ldw + a.K) * ES));
  const __amdgpu_buffer_rsrc_t rx = rsrc(a.x, (uint32_t)(((a.M - 1) * a.ldx + a.K) * ES));
  const int kc[2] = {((lane & 7) ^ swz(lane >> 3)) * VEC, ((lane & 7) ^ swz(8 + (lane >> 3))) * VEC};
  uint32_t off[LOADS];
#pragma unroll
  for (int p = 0; p < LOADS; ++p) {
    const int r = p * 8 + (lane >> 3);
    off[p] = (uint32_t)(((p < 2 ? min(r, a.N - n0 - 1) * a.ldw : min(r - 16, a.M - 1) * a.ldx) + kc[p & 1]) * ES);
  }
  auto fetch = [&](int s, int stage) {  // zeros behind the end, by the same number of loads
    const uint32_t kb[2] = {s * STEP + kc[0] < a.K ? (uint32_t)(s * STEP * ES) : OOB, s * STEP + kc[1] < a.K ? (uint32_t)(s * STEP * ES) : OOB};
#pragma unroll
    for (int p = 0; p < LOADS; ++p) load_lds(p < 2 ? rw : rx, own + stage * STAGE + p * 1024, off[p] + kb[p & 1]);
  };

  const int om = wave * 16 + (lane & 15), on = n0 + (lane >> 4) * 4;
  const bool finishes = wave < FM;
  const Bias4 bias(a, finishes ? on : a.N);
  const floatx4 res = residual4(a, finishes ? om : a.M, on);
  __builtin_amdgcn_sched_barrier(0);

  floatx4 acc[FM];
#pragma unroll
  for (int i = 0; i < FM; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int t = 0; t < S; ++t) fetch(wave + t * NW, t);
  int stage = 0;
  for (int s = wave; s < steps; s += NW) {
    wait_vmcnt<(S - 1) * LOADS>();
    __asm__ __volatile__("" ::: "memory");
    const char* at = own + stage * STAGE + (lane & 15) * ROW;
    u32x4 w[2], x[FM][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // lane groups 0, 1, 2, 3 take chunks 0, 2, 1, 3: the groups that LDS serves together
      // then differ in the lowest bit, and no two of their rows meet in a bank
      const int c = ((4 * h + ((lane >> 4 & 1) << 1 | lane >> 5)) ^ swz(lane & 15)) << 4;
      w[h] = *reinterpret_cast<const u32x4*>(at + c);
#pragma unroll
      for (int i = 0; i < FM; ++i) x[i][h] = *reinterpret_cast<const u32x4*>(at + (1 + i) * 16 * ROW + c);
    }
    __asm__ __volatile__("" ::: "memory");
    wait_lgkm0();  // the operands are in registers: the stage may be filled again
    __asm__ __volatile__("" ::: "memory");
    fetch(s + S * NW, stage);
    stage = stage + 1 == S ? 0 : stage + 1;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < FM; ++i) acc[i] = L::mma16(w[h], x[i][h], acc[i]);
  }
  wait_vmcnt<0>();
  __syncthreads();
  floatx4* const part = reinterpret_cast<floatx4*>(lds);
#pragma unroll
  for (int i = 0; i < FM; ++i) part[(wave * FM + i) * 64 + lane] = acc[i];
  __syncthreads();
  if (!finishes) return;
  floatx4 s = part[wave * 64 + lane];
#pragma unroll
  for (int q = 1; q < NW; ++q) s += part[(q * FM + wave) * 64 + lane];
  finish4(a, om, on, s, bias, res);
}

// --------------------------------------------- few fp32 tiles of any alignment
// A tile of 16 FN features x 16 FM rows; wave w takes K-tiles w, w + NW, ... of the
// reduction (128 bytes a row) as k_linear_stream does, but through registers, so that
// rows may lie at any element: whole lines of 8 rows a load, D K-tiles on their way, then
// through LDS of the wave's own into MFMA order.  LDS serves a wave's accesses in order,
// so one buffer a wave is enough and nothing waits for another wave before the end.
template <int FM, int FN, int NW, int D>
__global__ void __launch_bounds__(NW * 64) k_linear_wave(LinearArgs a) {
  constexpr int KT = 32, P = 2 * (FM + FN), BUF = (FM + FN) * 16 * ROW;
  static_assert(FM * FN * 1024 <= BUF, "a wave's sums fit where its operands were");
  static_assert(FM * FN <= NW, "a block per wave");
  static_assert(D % 2 == 0, "a K-tile's registers follow from its place in the loop");
  __shared__ __attribute__((aligned(1024))) char lds[NW * BUF];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tiles_n = (a.N + 16 * FN - 1) / (16 * FN);
  const int n0 = blockIdx.x % tiles_n * (16 * FN), m0 = blockIdx.x / tiles_n * (16 * FM);
  const float* const xb = static_cast<const float*>(a.x) + (int64_t)m0 * a.ldx;
  const float* const wb = static_cast<const float*>(a.w) + (int64_t)n0 * a.ldw;

  // load p: tile rows 8 p .. 8 p + 7 (w's rows first), lane l chunk l % 8 of row l / 8; rows
  // that do not exist read the last one: they enter only outputs that do not exist
  uint32_t off[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int r = (p < 2 * FN ? p : p - 2 * FN) * 8 + (lane >> 3), last = (p < 2 * FN ? a.N - n0 : a.M - m0) - 1;
    off[p] = (uint32_t)((min(r, last) * (p < 2 * FN ? a.ldw : a.ldx) + (lane & 7) * 4) * 4);
  }
  char* const own = lds + wave * BUF;
  char* const put[2] = {own + (lane >> 3) * ROW + (((lane & 7) ^ swz(lane >> 3)) << 4),
                        own + (8 + (lane >> 3)) * ROW + (((lane & 7) ^ swz(8 + (lane >> 3))) << 4)};
  const int whole = a.K / KT, n = whole > wave ? (whole - wave - 1) / NW + 1 : 0;

  const int om = m0 + wave / FN * 16 + (lane & 15), on = n0 + wave % FN * 16 + (lane >> 4) * 4;
  const bool finishes = wave < FM * FN;
  const Bias4 bias(a, finishes ? on : a.N);
  const floatx4 res = residual4(a, finishes && on < a.N ? om : a.M, on);

  u32x4 reg[D][P];
  auto from = [&](int p, int k0) { return reinterpret_cast<const float*>(reinterpret_cast<const char*>((p < 2 * FN ? wb : xb) + k0) + off[p]); };
  auto fetch = [&](int s, u32x4 (&to)[P]) {  // the wave's s-th K-tile
#pragma unroll
    for (int p = 0; p < P; ++p) to[p] = *reinterpret_cast<const u32x4_at4*>(from(p, (s * NW + wave) * KT));
  };
  floatx4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  u32x4 w[2][2][FN], x[2][2][FM];
  // a K-tile from registers to operands of set t
  auto turn = [&](const u32x4 (&from)[P], auto t) {
    __asm__ __volatile__("" ::: "memory");
#pragma unroll
    for (int p = 0; p < P; ++p) *reinterpret_cast<u32x4*>(put[p & 1] + (p >> 1) * 16 * ROW) = from[p];
    __asm__ __volatile__("" ::: "memory");
    const char* at = own + (lane & 15) * ROW;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = ((4 * h + ((lane >> 4 & 1) << 1 | lane >> 5)) ^ swz(lane & 15)) << 4;  // as in k_linear_stream
#pragma unroll
      for (int j = 0; j < FN; ++j) w[t][h][j] = *reinterpret_cast<const u32x4*>(at + j * 16 * ROW + c);
#pragma unroll
      for (int i = 0; i < FM; ++i) x[t][h][i] = *reinterpret_cast<const u32x4*>(at + (FN + i) * 16 * ROW + c);
    }
    __asm__ __volatile__("" ::: "memory");
  };
  auto mma = [&](auto t) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[t][h][j][e]), __uint_as_float(x[t][h][i][e]), acc[i][j], 0, 0, 0);
  };

#pragma unroll
  for (int d = 0; d < D; ++d)
    if (d < n) fetch(d, reg[d]);
  if (n > 0) {
    turn(reg[0], std::integral_constant<int, 0>{});
    if (D < n) fetch(D, reg[0]);
  }
  for (int s = 0; s < n; s += D)
    static_for<0, D>([&](auto d) {
      constexpr int NEXT = (d + 1) % D;
      if (s + d >= n) return;
      if (s + d + 1 < n) {
        turn(reg[NEXT], std::integral_constant<int, (d + 1) & 1>{});
        if (s + d + 1 + D < n) fetch(s + d + 1 + D, reg[NEXT]);
      }
      __builtin_amdgcn_sched_barrier(0);  // the next K-tile is under way before the MFMAs
      mma(std::integral_constant<int, d & 1>{});
      __builtin_amdgcn_sched_barrier(0);
    });

  if (a.K % KT && wave == whole % NW) {  // the rest of the reduction
#pragma unroll
    for (int p = 0; p < P; ++p) reg[0][p] = piece(from(p, 0) - (lane & 7) * 4, whole * KT + (lane & 7) * 4, a.K);
    turn(reg[0], std::integral_constant<int, 0>{});
    mma(std::integral_constant<int, 0>{});
  }
  floatx4* const part = reinterpret_cast<floatx4*>(own);
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) part[(i * FN + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  if (!finishes) return;
  floatx4 s = reinterpret_cast<const floatx4*>(lds)[wave * 64 + lane];
#pragma unroll
  for (int q = 1; q < NW; ++q) s += reinterpret_cast<const floatx4*>(lds + q * BUF)[wave * 64 + lane];
  finish4(a, om, on, s, bias, res);
}

// ------------------------------------------------- fp32 tiles of any alignment
// A tile of 32 FM rows x 32 FN features by G groups of 2 x 2 waves.  Group g sums
// K-tiles g, g + G, ... (128 bytes a row), each of its waves FM x FN blocks of 16 x 16 over
// all of a K-tile.  Rows pass through registers, D K-tiles ahead, into one of two LDS
// buffers (laid out as in lds_dma.hpp), so that they may lie at any element; a K-tile
// costs one barrier, which the MFMAs on the second half of its operands cover.
template <int FM, int FN, int G, int D>
__global__ void __launch_bounds__(G * 256) k_linear_mid(LinearArgs a) {
  constexpr int KT = 32, BM = 32 * FM, BN = 32 * FN, P = FM + FN, BUF = (BM + BN) * ROW;
  __shared__ __attribute__((aligned(1024))) char lds[G * 2 * BUF];
  static_assert((G - 1) * FM * FN * 4096 <= G * 2 * BUF, "the other groups' sums fit where the operands were");
  static_assert(D % 2 == 0, "a K-tile's buffer and registers follow from its place in the loop");
  const int tid = threadIdx.x & 255, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = wave >> 2, wm = wave >> 1 & 1, wn = wave & 1;

  // tiles as in k_linear_tile: consecutive ones on one XCD, in groups of 8 tile rows
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
  const int id = xcd_remap(blockIdx.x, gridDim.x);
  const int group = id / (8 * tiles_n), in = id - group * 8 * tiles_n;
  const int rows = min(8, tiles_m - group * 8);
  const int m0 = (group * 8 + in % rows) * BM, n0 = in / rows * BN;
  const float* const xb = static_cast<const float*>(a.x) + (int64_t)m0 * a.ldx;
  const float* const wb = static_cast<const float*>(a.w) + (int64_t)n0 * a.ldw;

  // thread t, piece p: tile row 32 p + t / 8 (x's rows first), chunk t % 8; rows that do not
  // exist read the last one: they enter only outputs that do not exist
  const int prow = tid >> 3, kc = (tid & 7) * 4;
  uint32_t off[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int r = prow + (p < FM ? p : p - FM) * 32, last = (p < FM ? a.M - m0 : a.N - n0) - 1;
    off[p] = (uint32_t)((min(r, last) * (p < FM ? a.ldx : a.ldw) + kc) * 4);
  }
  char* const own = lds + g * 2 * BUF;
  char* const put = own + prow * ROW + (((tid & 7) ^ swz(prow)) << 4);
  const int whole = a.K / KT, n = (whole + G - 1) / G;  // K-tiles, and those of a group (zeros behind the last)

  u32x4 reg[D][P];
  auto from = [&](int p, int k0) { return reinterpret_cast<const float*>(reinterpret_cast<const char*>((p < FM ? xb : wb) + k0) + off[p]); };
  auto fetch = [&](int s, u32x4 (&to)[P]) {  // the group's s-th K-tile
    if (G == 1 || s * G + g < whole) {       // the same for the whole wave
#pragma unroll
      for (int p = 0; p < P; ++p) to[p] = *reinterpret_cast<const u32x4_at4*>(from(p, (s * G + g) * KT));
    } else {
#pragma unroll
      for (int p = 0; p < P; ++p) to[p] = u32x4{0, 0, 0, 0};
    }
  };
  auto store = [&](int b, const u32x4 (&from)[P]) {
#pragma unroll
    for (int p = 0; p < P; ++p) *reinterpret_cast<u32x4*>(put + b * BUF + p * 32 * ROW) = from[p];
  };
  floatx4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

  // half h of a K-tile's operands: lane groups 0, 1, 2, 3 take chunks 0, 2, 1, 3 of the half, as in k_linear_stream
  u32x4 x[2][FM], w[2][FN];
  const char* const at = own + (lane & 15) * ROW;
  auto read = [&](int b, int h) {
    const int c = ((4 * h + ((lane >> 4 & 1) << 1 | lane >> 5)) ^ swz(lane & 15)) << 4;
#pragma unroll
    for (int i = 0; i < FM; ++i) x[h][i] = *reinterpret_cast<const u32x4*>(at + b * BUF + (wm * FM + i) * 16 * ROW + c);
#pragma unroll
    for (int j = 0; j < FN; ++j) w[h][j] = *reinterpret_cast<const u32x4*>(at + b * BUF + (BM + (wn * FN + j) * 16) * ROW + c);
  };
  auto mma = [&](int h) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[h][j][e]), __uint_as_float(x[h][i][e]), acc[i][j], 0, 0, 0);
  };
  auto meet = [&] {
    __asm__ __volatile__("" ::: "memory");
    wait_lgkm0();  // this wave's part of the next K-tile is in LDS, its operands of this one in registers
    wg_barrier();
  };

#pragma unroll
  for (int d = 0; d < D; ++d)
    if (d < n) fetch(d, reg[d]);
  if (n > 0) {
    store(0, reg[0]);
    if (D < n) fetch(D, reg[0]);
    meet();
    read(0, 0);
  }
  for (int s = 0; s < n; s += D)
    static_for<0, D>([&](auto d) {
      constexpr int NEXT = (d + 1) % D;
      if (s + d >= n) return;
      read(d & 1, 1);
      if (s + d + 1 < n) {
        store((d + 1) & 1, reg[NEXT]);
        if (s + d + 1 + D < n) fetch(s + d + 1 + D, reg[NEXT]);
      }
      __builtin_amdgcn_sched_barrier(0);  // reads and stores are under way before the MFMAs
      mma(0);
      __builtin_amdgcn_sched_barrier(0);
      meet();
      if (s + d + 1 < n) read((d + 1) & 1, 0);
      __builtin_amdgcn_sched_barrier(0);
      mma(1);
      __builtin_amdgcn_sched_barrier(0);
    });

  if (a.K % KT) {  // the rest of the reduction, by the first group
    if (G == 1 || g == 0) {
#pragma unroll
      for (int p = 0; p < P; ++p) reg[0][p] = piece(from(p, 0) - kc, whole * KT + kc, a.K);
      store(n & 1, reg[0]);
    }
    meet();
    if (G == 1 || g == 0) {
      read(n & 1, 0);
      read(n & 1, 1);
      mma(0);
      mma(1);
    }
  }
  if constexpr (G > 1) {  // the groups' sums, in their order
    floatx4* const part = reinterpret_cast<floatx4*>(lds) + (wave & 3) * 64 + lane;
    __syncthreads();
    if (g > 0) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) part[((g - 1) * FM * FN + i * FN + j) * 256] = acc[i][j];
    }
    __syncthreads();
    if (g > 0) return;
#pragma unroll
    for (int q = 0; q < G - 1; ++q)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] += part[(q * FM * FN + i * FN + j) * 256];
  }
  // block (i, j): lane l holds row l % 16 and features 4 (l / 16) ..
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int on = n0 + (wn * FN + j) * 16 + (lane >> 4) * 4, om = m0 + wm * FM * 16 + (lane & 15);
    const Bias4 bias(a, on);
    floatx4 res[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) res[i] = on < a.N ? residual4(a, om + i * 16, on) : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < FM; ++i) finish4(a, om + i * 16, on, acc[i][j], bias, res[i]);
  }
}

// -------------------------------------------------------------- many tiles
// A tile of BM rows x BN features on WM x WN waves.  K-tiles of 128 bytes a row
// lie in LDS as in lds_dma.hpp, NBUF of them in turn.  DMA: the loads write LDS
// themselves (rows aligned to 16 bytes); otherwise they pass through registers.
template <class T, int BM, int BN, int WM, int WN, bool DMA, int NBUF>
__global__ void __launch_bounds__(WM * WN * 64) k_linear_tile(LinearArgs a) {
  using L = LinT<T>;
  constexpr int VEC = L::VEC, KT = 8 * VEC, NT = WM * WN * 64, ES = sizeof(T);
  constexpr int FM = BM / WM / 32, FN = BN / WN / 32;
  constexpr int PA = BM * 8 / NT, PB = BN * 8 / NT;  // 16-byte pieces of a K-tile per thread
  constexpr int BUF = (BM + BN) * ROW;
  constexpr int PITCH = BN + 4;  // floats of a row of the finished tile
  static_assert(WM * 32 * PITCH * 4 <= NBUF * BUF, "a row block of the finished tile fits where the operands were");
  __shared__ __attribute__((aligned(1024))) char lds[NBUF * BUF];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;

  // consecutive tiles on one XCD, in groups of 8 tile rows, so that its L2 serves a
  // block of tiles whose operands it holds
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
  const int id = xcd_remap(blockIdx.x, gridDim.x);
  const int group = id / (8 * tiles_n), in = id - group * 8 * tiles_n;
  const int rows = min(8, tiles_m - group * 8);
  const int m0 = (group * 8 + in % rows) * BM, n0 = in / rows * BN;
  const T* xb = static_cast<const T*>(a.x) + (int64_t)m0 * a.ldx;
  const T* wb = static_cast<const T*>(a.w) + (int64_t)n0 * a.ldw;
  const int steps = (a.K + KT - 1) / KT;

  // thread t, piece p: tile row p NT / 8 + t / 8, physical chunk t % 8; the rows of a
  // thread's pieces share their swizzle (NT / 8 is a multiple of 16)
  static_assert(NT / 8 % 16 == 0, "rows of one swizzle");
  const int prow = tid >> 3, kc = ((tid & 7) ^ swz(prow)) * VEC;
  const __amdgpu_buffer_rsrc_t rx = rsrc(xb, DMA ? (uint32_t)(((min(BM, a.M - m0) - 1) * a.ldx + a.K) * ES) : 0u);
  const __amdgpu_buffer_rsrc_t rw = rsrc(wb, DMA ? (uint32_t)(((min(BN, a.N - n0) - 1) * a.ldw + a.K) * ES) : 0u);
  uint32_t off[PA + PB];  // bytes from the tile's first row
  u32x4 reg[PA + PB];    // not DMA: a K-tile on its way
#pragma unroll
  for (int p = 0; p < PA + PB; ++p) {
    // rows that do not exist read the last one: they enter only outputs that do not exist
    const int r = prow + (p < PA ? p : p - PA) * (NT / 8), last = (p < PA ? a.M - m0 : a.N - n0) - 1;
    off[p] = (uint32_t)((min(r, last) * (p < PA ? a.ldx : a.ldw) + (DMA ? kc : 0)) * ES);
  }
  // the offset of K-tile s; behind the reduction's end out of range: zeros, by the same number of loads
  auto tile_off = [&](int s) { return s * KT + kc < a.K ? (uint32_t)(s * KT * ES) : OOB; };
  auto fetch_piece = [&](auto p, uint32_t kb, int at) {  // at: a buffer's offset
    load_lds(p < PA ? rx : rw, lds + at + (p * NT + wave * 64) * 16, off[p] + kb);
  };
  // K-tile s into registers, and from there into a buffer
  auto fetch = [&](int s) {
    const int k0 = s * KT;
    auto row = [&](int p) { return reinterpret_cast<const T*>(reinterpret_cast<const char*>(p < PA ? xb : wb) + off[p]); };
    if (k0 + KT <= a.K) {  // the same for the whole workgroup
#pragma unroll
      for (int p = 0; p < PA + PB; ++p) reg[p] = *reinterpret_cast<const u32x4_at2*>(row(p) + k0 + kc);
    } else {
#pragma unroll
      for (int p = 0; p < PA + PB; ++p) reg[p] = piece(row(p), k0 + kc, a.K);
    }
  };
  auto store = [&](int at) {
#pragma unroll
    for (int p = 0; p < PA + PB; ++p) *reinterpret_cast<u32x4*>(lds + at + (p * NT + tid) * 16) = reg[p];
  };

  floatx16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  const int fr = lane & 31, fq = lane >> 5, sw = swz(fr);
  const char* const A = lds + (wm * FM * 32 + fr) * ROW;
  const char* const B = lds + (BM + wn * FN * 32 + fr) * ROW;
  auto operand = [&](const char* base, int at, int ks, int block) {
    return *reinterpret_cast<const u32x4*>(base + block * 32 * ROW + at + (((ks * 2 + fq) ^ sw) << 4));
  };
  auto meet = [&] {
    __asm__ __volatile__("" ::: "memory");
    wait_lgkm0();  // the operands read last are in registers
    wg_barrier();
  };

  static_assert(DMA ? FM % 2 == 0 : NBUF == 2, "two halves, or two buffers");
  if constexpr (DMA) {
    // Two halves per K-tile, of the upper and the lower half of the wave's row blocks.
    // The first runs on x0 and w, the second on x1 and w; during the first x1 is
    // read, during the second the next K-tile's x0 and w (a step's w once its MFMAs
    // have it).  So LDS is free for K-tile s + NBUF early, x0 and w when the first half
    // begins, x1 when the second does, and every load has NBUF - 1/2 K-tiles of time.
    // A half waits for the loads whose operands are read in it, all but the LATE issued
    // last, after its first step, whose operands are in registers by then.  Reads and
    // loads are issued between MFMAs, in their shadow (all of a half's before its MFMAs:
    // 272 us against 224 for 4096 x 8192 x 4096).
    constexpr int H = FM / 2, PH = H * 32 / (NT / 8);  // row blocks of a half; its pieces per wave row
    static_assert(H * 32 % (NT / 8) == 0 && PA == 2 * WM * PH, "pieces and halves");
    constexpr int N_LOW = PA / 2, N_UP = PA / 2 + PB, N_ALL = PA + PB;
    u32x4 x0[4][H], x1[4][H], w[4][FN];
    // the n-th piece of the lower half's rows, of the upper half's and w
    auto low = [&](auto n, uint32_t kb, int at) {
      fetch_piece(std::integral_constant<int, (n / PH * 2 + 1) * PH + n % PH>{}, kb, at);
    };
    auto up = [&](auto n, uint32_t kb, int at) {
      if constexpr (n < PA / 2) fetch_piece(std::integral_constant<int, n / PH * 2 * PH + n % PH>{}, kb, at);
      else fetch_piece(std::integral_constant<int, PA / 2 + n>{}, kb, at);
    };
    // the MFMAs of a step on rows of block base + i, and the L items that fall between them
    auto step = [&](auto base, const u32x4 (&x)[H], const u32x4 (&v)[FN], auto L_items, auto&& item) {
      constexpr int Q = H * FN, LI = L_items;
      static_for<0, Q>([&](auto q) {
        acc[base + q / FN][q % FN] = L::mma32(v[q % FN], x[q / FN], acc[base + q / FN][q % FN]);
        static_for<(q * LI + Q - 1) / Q, ((q + 1) * LI + Q - 1) / Q>([&](auto n) { item(n); });
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, H> second{};
    auto none = [](auto) {};
    for (int t = 0; t < NBUF; ++t) {
      const uint32_t kb = tile_off(t);
      static_for<0, N_UP>([&](auto n) { up(n, kb, t * BUF); });
      static_for<0, N_LOW>([&](auto n) { low(n, kb, t * BUF); });
    }
    constexpr int LATE = (NBUF - 1) * N_ALL;
    wait_vmcnt<N_LOW + LATE>();
    wg_barrier();
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
      for (int i = 0; i < H; ++i) x0[ks][i] = operand(A, 0, ks, i);
#pragma unroll
      for (int j = 0; j < FN; ++j) w[ks][j] = operand(B, 0, ks, j);
    }
    int at = 0;
    for (int s = 0; s < steps; ++s) {
      const int then = at + BUF == NBUF * BUF ? 0 : at + BUF;
      const uint32_t kb = tile_off(s + NBUF);
      constexpr int U1 = (N_UP + 2) / 3, U2 = (N_UP - U1 + 1) / 2, U3 = N_UP - U1 - U2;
      __builtin_amdgcn_sched_barrier(0);
      step(first, x0[0], w[0], std::integral_constant<int, 0>{}, none);
      wait_vmcnt<LATE>();
      meet();
      auto read_x1 = [&](auto n) { x1[n / H][n % H] = operand(A, at, n / H, H + n % H); };
      step(first, x0[1], w[1], std::integral_constant<int, 2 * H + U1>{}, [&](auto n) {
        if constexpr (n < 2 * H) read_x1(n);
        else up(std::integral_constant<int, n - 2 * H>{}, kb, at);
      });
      step(first, x0[2], w[2], std::integral_constant<int, 2 * H + U2>{}, [&](auto n) {
        if constexpr (n < 2 * H) read_x1(std::integral_constant<int, 2 * H + n>{});
        else up(std::integral_constant<int, n - 2 * H + U1>{}, kb, at);
      });
      step(first, x0[3], w[3], std::integral_constant<int, U3>{}, [&](auto n) { up(std::integral_constant<int, n + U1 + U2>{}, kb, at); });
      step(second, x1[0], w[0], std::integral_constant<int, 0>{}, none);
      wait_vmcnt<LATE>();
      meet();
      auto read_x0 = [&](auto n) { x0[n / H][n % H] = operand(A, then, n / H, n % H); };
      auto read_w = [&](auto ks, auto n) { w[ks][n] = operand(B, then, ks, n); };
      step(second, x1[1], w[1], std::integral_constant<int, 2 * H + FN + N_LOW>{}, [&](auto n) {
        if constexpr (n < 2 * H) read_x0(n);
        else if constexpr (n < 2 * H + FN) read_w(std::integral_constant<int, 0>{}, std::integral_constant<int, n - 2 * H>{});
        else low(std::integral_constant<int, n - 2 * H - FN>{}, kb, at);
      });
      step(second, x1[2], w[2], std::integral_constant<int, 2 * H + FN>{}, [&](auto n) {
        if constexpr (n < 2 * H) read_x0(std::integral_constant<int, 2 * H + n>{});
        else read_w(std::integral_constant<int, 1>{}, std::integral_constant<int, n - 2 * H>{});
      });
      step(second, x1[3], w[3], std::integral_constant<int, FN>{}, [&](auto n) { read_w(std::integral_constant<int, 2>{}, n); });
      static_for<0, FN>([&](auto n) { read_w(std::integral_constant<int, 3>{}, n); });
      at = then;
    }
    wait_vmcnt<0>();
    meet();
  } else if (steps > 0) {
    // A step's operands are read during the step before it; the barrier between two
    // K-tiles lies before the last step, whose operands are in registers by then.
    u32x4 xf[2][FM], wf[2][FN];
    auto read = [&](int at, int ks, int set) {
#pragma unroll
      for (int i = 0; i < FM; ++i) xf[set][i] = operand(A, at, ks, i);
#pragma unroll
      for (int j = 0; j < FN; ++j) wf[set][j] = operand(B, at, ks, j);
    };
    auto mma = [&](int set) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = L::mma32(wf[set][j], xf[set][i], acc[i][j]);
    };
    fetch(0);
    store(0);
    meet();
    read(0, 0, 0);
    for (int s = 0; s < steps; ++s) {
      const int at = (s & 1) * BUF;
      const bool more = s + 1 < steps;
      if (more) fetch(s + 1);
#pragma unroll
      for (int ks = 0; ks < 3; ++ks) {
        read(at, ks + 1, (ks + 1) & 1);
        __builtin_amdgcn_sched_barrier(0);  // the reads are under way before the MFMAs
        mma(ks & 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (more) {
        store(at ^ BUF);
        meet();  // every wave's part of the next K-tile is in LDS, and all are done with this one
        read(at ^ BUF, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      mma(1);
    }
  }

  // The finished tile through LDS, a block of 32 rows per wave row at a time, so that
  // whole rows are written.  Block (i, j): lane l holds row l % 32 and
  // features 8 g + 4 (l / 32) .. of g = 0 .. 3.  On the way out a thread keeps its 4
  // features and walks the rows, whose residuals are loaded before the block is put down.
  float* const out = reinterpret_cast<float*>(lds);
  constexpr int TR = NT / (BN / 4), PASSES = WM * 32 / TR;  // rows per pass
  const int n = n0 + tid % (BN / 4) * 4, r0 = tid / (BN / 4);
  const Bias4 bias(a, n);
  // row of pass p in block i: m0 + 32 i + r0 + a number that p alone gives
  static_assert(32 % TR == 0, "a pass lies in one wave row's block");
  auto rel = [](int pass) { return pass * TR / 32 * FM * 32 + pass * TR % 32; };
  auto put_down = [&](int i) {
    __syncthreads();
#pragma unroll
    for (int ii = 0; ii < FM; ++ii)
      if (ii == i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<floatx4*>(out + (wm * 32 + fr) * PITCH + (wn * FN + j) * 32 + 8 * g + 4 * fq) =
                floatx4{acc[ii][j][4 * g], acc[ii][j][4 * g + 1], acc[ii][j][4 * g + 2], acc[ii][j][4 * g + 3]};
    __syncthreads();
  };
  auto sums = [&](int pass) { return *reinterpret_cast<const floatx4*>(out + (pass * TR + r0) * PITCH + n - n0); };
  auto whole = [&](auto f32) {  // a tile without an edge
    using O = Out4<f32>;
    for (int i = 0; i < FM; ++i) {
      const int64_t m = m0 + 32 * i + r0;
      typename O::Raw res[PASSES];
      if (a.res)
#pragma unroll
        for (int pass = 0; pass < PASSES; ++pass) res[pass] = O::load(a.res, m * a.ldres + n + rel(pass) * a.ldres);
      put_down(i);
#pragma unroll
      for (int pass = 0; pass < PASSES; ++pass)
        O::store(a.y, m * a.ldy + n + rel(pass) * a.ldy,
                 epilogue<f32>(a, sums(pass), bias.v, a.res ? O::wide(res[pass]) : floatx4{0.f, 0.f, 0.f, 0.f}));
    }
  };
  if (m0 + BM <= a.M && n0 + BN <= a.N) {
    if (a.out_f32) whole(std::true_type{});
    else whole(std::false_type{});
    return;
  }
  for (int i = 0; i < FM; ++i) {
    put_down(i);
#pragma unroll 1
    for (int pass = 0; pass < PASSES; ++pass) {
      const int m = m0 + 32 * i + r0 + rel(pass);
      finish4(a, m, n, sums(pass), bias, residual4(a, m, n));
    }
  }
}

// Whether rows of bf16 lie between two words.
template <class T>
bool odd_rows(const LinearArgs& a) {
  return sizeof(T) == 2 && (((a.ldx | a.ldw) & 1) || ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w)) & 2));
}

template <class T, int FM, int FN, int NW, int U>
void few(const LinearArgs& a, hipStream_t s) {
  const dim3 tiles((unsigned)(((a.N + 16 * FN - 1) / (16 * FN)) * ((int64_t)(a.M + 16 * FM - 1) / (16 * FM))));
  if (sizeof(T) == 2 && odd_rows<T>(a)) hipLaunchKernelGGL((k_linear_few<T, FM, FN, NW, U, sizeof(T) == 2>), tiles, dim3(NW * 64), 0, s, a);
  else hipLaunchKernelGGL((k_linear_few<T, FM, FN, NW, U, false>), tiles, dim3(NW * 64), 0, s, a);
}

template <class T, int FM, int NW, int S>
void stream(const LinearArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_linear_stream<T, FM, NW, S>), dim3((unsigned)((a.N + 15) / 16)), dim3(NW * 64), 0, s, a);
}

template <int FM, int FN, int NW, int D>
void waves(const LinearArgs& a, hipStream_t s) {
  const int64_t tiles = (int64_t)((a.N + 16 * FN - 1) / (16 * FN)) * ((a.M + 16 * FM - 1) / (16 * FM));
  hipLaunchKernelGGL((k_linear_wave<FM, FN, NW, D>), dim3((unsigned)tiles), dim3(NW * 64), 0, s, a);
}

template <int FM, int FN, int G, int D>
void mid(const LinearArgs& a, hipStream_t s) {
  const int64_t tiles = (int64_t)((a.N + 32 * FN - 1) / (32 * FN)) * ((a.M + 32 * FM - 1) / (32 * FM));
  hipLaunchKernelGGL((k_linear_mid<FM, FN, G, D>), dim3((unsigned)tiles), dim3(G * 256), 0, s, a);
}

template <class T, int BM, int BN, int WM, int WN, bool DMA, int NBUF>
void tile(const LinearArgs& a, hipStream_t s) {
  const int64_t tiles = (int64_t)((a.N + BN - 1) / BN) * ((a.M + BM - 1) / BM);
  hipLaunchKernelGGL((k_linear_tile<T, BM, BN, WM, WN, DMA, NBUF>), dim3((unsigned)tiles), dim3(WM * WN * 64), 0, s, a);
}

// The other kernels for bf16, and what a K-tile (128 bytes of a row) costs
// one workgroup of each, in us: one / `fit` of them on a CU, measured at 128 to 4096
// rows, 4096 features and K = 4096, and what a round of workgroups costs besides.
// One row per kernel, by how the loads go.
enum Kernel { FEW_16x16, FEW_32x16, FEW_32x32, FEW_64x32, TILE_64x64, TILE_64x128, TILE_128x128, TILE_256x128, TILE_256x256, KERNELS };
struct Cost {
  int bm, bn, fit;
  float alone, full, round;
};
// Where a kernel is not built, its cost is 0.
enum Loads { ODD, REGISTERS, LDS };
constexpr Cost COSTS[3][KERNELS] = {
    // loads through registers, some rows between two words
    {{16, 16, 2, .242f, .419f, 3.5f}, {32, 16, 2, .352f, .603f, 3.5f}, {32, 32, 2, .45f, .77f, 2.5f}, {64, 32, 2, .60f, 1.07f, 2.5f}, {64, 64, 4, 1.02f, 1.65f, 3.f}, {}, {128, 128, 2, 1.72f, 1.74f, 6.f}, {}, {256, 256, 1, 3.1f, 3.1f, 16.f}},
    // loads through registers
    {{16, 16, 2, .145f, .255f, 3.5f}, {32, 16, 2, .219f, .395f, 3.5f}, {32, 32, 2, .303f, .517f, 2.5f}, {64, 32, 2, .41f, .766f, 2.5f}, {64, 64, 4, .89f, 1.33f, 3.f}, {}, {128, 128, 2, 1.58f, 1.66f, 6.f}, {}, {256, 256, 1, 2.8f, 2.8f, 16.f}},
    // loads into LDS
    {{16, 16, 2, .103f, .205f, 3.5f}, {32, 16, 2, .157f, .328f, 3.5f}, {32, 32, 2, .245f, .456f, 2.5f}, {64, 32, 2, .345f, .67f, 2.5f}, {64, 64, 2, .33f, .50f, 3.f}, {64, 128, 2, .44f, .74f, 4.f}, {128, 128, 2, .62f, 1.03f, 7.f}, {256, 128, 1, .94f, .94f, 9.f}, {256, 256, 1, 1.48f, 1.48f, 16.f}},
};

// The kernel with the least time by those costs: whole rounds of the chip and the
// rest.  (K = 4096: 512 x 4096 outputs 64 x 128 32 us against 36 for 64 x 64 and
// 44 for 128 x 128; 1024 x 4096 128 x 128 45 against 66 and, 256 x 256, 86; 2048 x 4096
// 256 x 128 69 against 75 and 91; 4096 x 4096 256 x 256 114 against 134 for 256 x 128; 41 x
// 58, K = 18939, 16 x 16 89 before and 54 after shifting odd rows, 32 x 32 177.)
Kernel pick(const LinearArgs& a, Loads loads, bool near, double* us) {
  const int64_t steps = ((int64_t)a.K * 2 + ROW - 1) / ROW;
  Kernel best = FEW_16x16;
  double least = 0;
  for (int k = 0; k < (near ? KERNELS : TILE_64x64); ++k) {
    const Cost& c = COSTS[loads][k];
    if (!c.bm) continue;
    const int64_t n = ((a.M + c.bm - 1) / c.bm) * (int64_t)((a.N + c.bn - 1) / c.bn), round = 256 * c.fit;
    const int64_t whole = n / round, rest = n % round;
    // more than one on some CUs: the slowest CU's time, or, for the two kernels bound by L2, a share of all
    double last = rest <= 256 ? c.alone : c.full;
    if ((k == FEW_32x32 || k == FEW_64x32) && rest > 256) last = c.alone + (c.full - c.alone) * (double)(rest - 256) / (double)(round - 256);
    const double t = whole * (steps * (double)c.full + c.round) + (rest ? steps * last + c.round : 0);
    if (k == 0 || t < least) {
      least = t;
      best = Kernel(k);
    }
  }
  *us = least;
  return best;
}

// The kernels for fp32: what a K-tile costs a workgroup alone on its CU and two of them, and
// what an output tile costs besides 2.5 us of the launch, in us, measured with 16 to 2048
// workgroups at K = 4096 and 512.  `pairs`: two fit a CU, and one behind a pair takes as long
// as a pair.  No less than the operands' way from L2 takes, at 11.5 TB/s (376 x 768 outputs, K = 11136,
// 16 x 16 143 us, 32 x 32 109).
struct F32Cost {
  int bm, bn;
  float alone, two, tile;
  bool pairs, dma;
  void (*run)(const LinearArgs&, hipStream_t);
};
const F32Cost F32_COSTS[] = {
    {16, 16, .06f, .112f, .9f, false, false, waves<1, 1, 12, 2>},   {16, 32, .105f, .2f, .95f, false, false, waves<1, 2, 8, 2>},
    {32, 16, .107f, .2f, .95f, false, false, waves<2, 1, 8, 2>},    {32, 32, .178f, .305f, 1.6f, false, false, mid<1, 1, 4, 2>},
    {32, 64, .308f, .555f, 2.f, false, false, mid<1, 2, 2, 4>},    {64, 32, .308f, .555f, 2.f, false, false, mid<2, 1, 2, 4>},
    {64, 64, .536f, 1.075f, 3.f, false, false, mid<2, 2, 2, 2>},   {64, 64, .634f, 1.03f, 1.45f, true, false, mid<2, 2, 1, 4>},
    {64, 96, .912f, 1.43f, 3.f, true, false, mid<2, 3, 1, 4>},      {96, 64, .912f, 1.43f, 3.f, true, false, mid<3, 2, 1, 4>},
    {96, 96, 1.3f, 2.11f, 4.5f, true, false, mid<3, 3, 1, 4>},      {64, 128, 1.18f, 1.885f, 4.5f, true, false, mid<2, 4, 1, 4>},
    {128, 64, 1.18f, 1.885f, 4.5f, true, false, mid<4, 2, 1, 4>},   {128, 128, 2.1f, 3.72f, 7.f, true, true, tile<float, 128, 128, 2, 2, true, 2>},
    {256, 256, 7.28f, 14.56f, 24.f, false, true, tile<float, 256, 256, 2, 4, true, 2>},
};

// The one with the least time by those costs; of 240 products of the operator's range it takes 2 %
// more than the best of them on average.  (580 x 1891 outputs, K = 4785, 32 x 32 130 us
// against 155 for 64 x 64; 975 x 2986, K = 10274, 64 x 96 474 against 530 for 96 x 96 and 550 for 32 x 64; 1089 x
// 1216, K = 4096, 32 x 64 111 against 121 for 96 x 64; 54 x 832, K = 5760, 16 x 16 14 against 18 for
// 16 x 32 and 32 for 32 x 32; 642 x 128, K = 13312, 16 x 32 45 against 48 for 32 x 16 and 68 for 16 x 16;
// 4096 x 4096, K = 4096, 256 x 256 955, 64 x 128 1010, 64 x 64 1115.)
const F32Cost& pick_f32(const LinearArgs& a, bool dma, double* us) {
  const F32Cost* best = nullptr;
  for (const F32Cost& c : F32_COSTS) {
    if (c.dma && !dma) continue;
    const int64_t n = ((a.M + c.bm - 1) / c.bm) * (int64_t)((a.N + c.bn - 1) / c.bn), steps = ((int64_t)a.K + 31) / 32;
    if (n >= 1 << 22) continue;          // of up to 1024 threads each: fewer than 2^32
    const int64_t cu = (n + 255) / 256;  // of the CU with the most
    const double sums = steps * (cu == 1 ? (double)c.alone : (c.pairs ? (cu + 1) / 2 * 2 : cu) * .5 * c.two);
    const double t = 2.5 + cu * (double)c.tile + std::max(sums, n * (double)(c.bm + c.bn) * a.K * 4 / 11.5e6);
    if (!best || t < *us) {
      best = &c;
      *us = t;
    }
  }
  return *best;
}

// What k_linear_stream takes for blocks of 16 rows, in us: the workgroups bring 12 TB/s from L2,
// one of them up to 95 GB/s of bf16 and, of fp32, 97, 83 or 56 GB/s for one, two or more blocks; the chip
// 5.5 TB/s of weights from memory.  (4096 features, K = 4096, bf16: 16 rows 9.1 us,
// k_linear_few 10.1; 32 rows 10.9 and 14.3; 48 rows 12.7 and 17.5; 64 rows 14.3 and 18.3.
// K = 25088: 32 rows 51 and 72, 64 rows 71 and 93.  48 x 64, K = 11136: 17 and 22.  fp32: 32 x 4096, K =
// 4096, 20 and, k_linear_wave, 22; 64 x 4096, K = 25088, 180 and, k_linear_mid, 150; 64 x 1000, K = 4096, 25 and 16.)
double stream_us(const LinearArgs& a, int blocks, int es) {
  const double row = (double)a.K * es, one = es == 2 ? 95e3 : blocks == 1 ? 97e3 : blocks == 2 ? 83e3 : 56e3;
  const int groups = (a.N + 15) / 16, rounds = (groups + 255) / 256;
  return 2. + std::max(rounds * (16. + 16. * blocks) * row / std::min(one, 12e6 / std::min(groups, 256)), a.N * row / 5.5e6);
}

template <class T>
void launch_t(const LinearArgs& a, hipStream_t s) {
  constexpr int VEC = LinT<T>::VEC;
  constexpr bool F = sizeof(T) == 4;
  // the loads that write LDS move 16 aligned bytes
  const bool dma = a.K % VEC == 0 && a.ldx % VEC == 0 && a.ldw % VEC == 0 && reinterpret_cast<uintptr_t>(a.x) % 16 == 0 &&
                   reinterpret_cast<uintptr_t>(a.w) % 16 == 0;
  // a tile of 256 rows is addressed by 31-bit offsets from its first one
  const bool near = (255 * std::max(a.ldx, a.ldw) + a.K) * (int64_t)sizeof(T) < (int64_t(1) << 31);
  // up to 8 rows the weights are all there is to read.  k_linear_stream reads them for up to
  // 2048 features and for rows of 32 KB and more (one row, bf16: 1000 features, K = 25088,
  // 22 us against 30 with k_linear_few; 64 features 14 against 29; 4096 features 36 against 37; 8
  // rows, fp32, 1000 features, K = 4096, 9.6 against 14.5), fp32 that it cannot take goes by costs up
  // to 2048 features and for rows of 16 KB and more (rows 3 elements apart: one row of 1000, K = 25088, 53
  // against 67, 8 of 5000, K = 4096, 24 against 30, but one of 16384, K = 1024, 18 against 15), and
  // 16 features a workgroup of 16 waves take the rest (one row, bf16: 4096 features, K = 4096, 7.9
  // against 8.4; 16384 features, K = 2048, 13.0 against 17.8; with 8 waves 4096 features, K = 25088, 42)
  if (a.M <= 8) {
    const int64_t row = a.K * (int64_t)sizeof(T);
    if (near && dma && (a.N <= 2048 || row >= 32768)) return stream<T, 1, 8, 3>(a, s);
    if (!F || !near || dma || (a.N > 2048 && row < 16384)) return few<T, 1, 1, 16, 2>(a, s);
  }
  double us;
  const F32Cost* f = nullptr;
  Kernel k = FEW_64x32;  // fp32 rows that are far apart
  if (!F) k = pick(a, dma ? LDS : odd_rows<T>(a) ? ODD : REGISTERS, near, &us);
  else if (near) f = &pick_f32(a, dma, &us);
  if (a.M <= 64 && dma && near) {
    const int blocks = (a.M + 15) / 16;
    if (stream_us(a, blocks, sizeof(T)) < us) {
      if (blocks == 1) return stream<T, 1, 8, 3>(a, s);
      if (blocks == 2) return stream<T, 2, 8, 2>(a, s);
      if (blocks == 3) return stream<T, 3, 6, 3>(a, s);
      return stream<T, 4, 4, 3>(a, s);
    }
  }
  if (f) return f->run(a, s);
  if constexpr (F) {
    few<T, 4, 2, 8, 1>(a, s);
  } else {
    switch (k) {
      case FEW_16x16: return few<T, 1, 1, 16, 2>(a, s);
      case FEW_32x16: return few<T, 2, 1, 16, 2>(a, s);
      case FEW_32x32: return few<T, 2, 2, 8, 2>(a, s);
      case FEW_64x32: return few<T, 4, 2, 8, 1>(a, s);
      case TILE_64x64: return dma ? tile<T, 64, 64, 1, 2, true, 4>(a, s) : tile<T, 64, 64, 2, 2, false, 2>(a, s);
      case TILE_64x128: return tile<T, 64, 128, 1, 4, true, 3>(a, s);
      case TILE_128x128: return dma ? tile<T, 128, 128, 2, 2, true, 2>(a, s) : tile<T, 128, 128, 2, 2, false, 2>(a, s);
      case TILE_256x128: return tile<T, 256, 128, 2, 4, true, 3>(a, s);
      default: return dma ? tile<T, 256, 256, 2, 4, true, 2>(a, s) : tile<T, 256, 256, 2, 4, false, 2>(a, s);
    }
  }
}

}  // namespace

void launch_linear(const LinearArgs& a, Prec p, hipStream_t s) {
  // A launch has fewer than 2^32 threads, of which k_linear_few gives 64 to a feature or
  // one to two outputs: products beyond go in slices (of at most 2^32 outputs, so that the larger
  // of F32_COSTS have fewer than 2^22 tiles).
  constexpr int FEATURES = 1 << 24;
  const int64_t rows = (int64_t(1) << 32) / std::min(a.N, FEATURES) / 256 * 256;
  const int64_t ei = p == BF16 ? 2 : 4, eo = a.out_f32 ? 4 : 2;
  for (int64_t n = 0; n < a.N; n += FEATURES)
    for (int64_t m = 0; m < a.M; m += rows) {
      LinearArgs b = a;
      b.x = static_cast<const char*>(a.x) + m * a.ldx * ei;
      b.w = static_cast<const char*>(a.w) + n * a.ldw * ei;
      if (a.bias) b.bias = a.bias + n;
      if (a.res) b.res = static_cast<const char*>(a.res) + (m * a.ldres + n) * eo;
      b.y = static_cast<char*>(a.y) + (m * a.ldy + n) * eo;
      b.M = (int)std::min<int64_t>(rows, a.M - m);
      b.N = (int)std::min<int64_t>(FEATURES, a.N - n);
      if (p == BF16) launch_t<uint16_t>(b, s);
      else launch_t<float>(b, s);
    }
}

}  // namespace fs
