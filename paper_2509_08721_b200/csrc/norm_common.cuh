// What the kernels of the norm and of the 8-bit checkpoints share: arguments, conversions, paired fp32
// arithmetic, sums over warps, the quantiser.
#pragma once

#include <cuda_bf16.h>
#include <math.h>

#include <type_traits>

#include "common.cuh"
#include "paired.cuh"

namespace sapo {

constexpr int Q8_GROUP = 128;            // columns that share one checkpoint scale
constexpr int NORM_MAX_H = 16384;
constexpr int NORM_THREADS = 256;
constexpr int NORM_MAX_THREADS = 512;
constexpr int SMEM_MAX = 220 * 1024;     // shared memory a block may take for its rows
// A group whose largest magnitude is below this is stored as zeros: 127 (1 / amax) would overflow.
constexpr float Q8_TINY = 1.5046328e-36f;   // 2^-119

enum { KIND_LAYER = SAPO_NORM_LAYER, KIND_RMS = SAPO_NORM_RMS };

// a matrix of fp32 or bf16 rows whose type is known at run time
struct Mat { void* p; int64_t ld; int32_t dtype; };
struct Q8Mat { int8_t* p; float* scale; int64_t ld, ld_scale; };

struct NormFwdArgs {
  Mat x, y; Q8Mat q; const void* gamma; const void* beta; int32_t w_dtype, kind; float eps;
  float* mean; float* rstd; int64_t T; int32_t H; int32_t* status;
};
struct NormBwdArgs {
  Mat dy, x, dx; Q8Mat q; const void* gamma; int32_t w_dtype, kind; const float* mean; const float* rstd;
  int64_t T; int32_t H; float* part; float* dgamma; float* dbeta; int32_t accumulate;
};
struct Ckpt8Args { Mat x; Q8Mat q; int64_t T; int32_t H; int32_t* status; };

// ---------------------------------------------------------------------------- 8 neighbouring columns
__device__ __forceinline__ void unpack8(uint4 u, float2 (&x)[4]) {       // bf16 to fp32: the upper half of the word
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  #pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
}
// int8 to fp32: the byte, its sign flipped, as the last bits of 2^23; exact
__device__ __forceinline__ void unpack8(uint2 u, float2 (&x)[4]) {
  const uint32_t w[2] = {u.x ^ 0x80808080u, u.y ^ 0x80808080u};
  const float2 back = both(-8388736.f);                                   // -(2^23 + 128)
  #pragma unroll
  for (int h = 0; h < 2; ++h) {
    x[2 * h] = add2(make_float2(__uint_as_float(__byte_perm(w[h], 0x4b000000u, 0x7440)),
                                __uint_as_float(__byte_perm(w[h], 0x4b000000u, 0x7441))), back);
    x[2 * h + 1] = add2(make_float2(__uint_as_float(__byte_perm(w[h], 0x4b000000u, 0x7442)),
                                    __uint_as_float(__byte_perm(w[h], 0x4b000000u, 0x7443))), back);
  }
}
__device__ __forceinline__ void load8(const float* p, float2 (&x)[4]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = make_float2(a.x, a.y); x[1] = make_float2(a.z, a.w); x[2] = make_float2(b.x, b.y); x[3] = make_float2(b.z, b.w);
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float2 (&x)[4]) { unpack8(*reinterpret_cast<const uint4*>(p), x); }
__device__ __forceinline__ void load8(const int8_t* p, float2 (&x)[4]) { unpack8(*reinterpret_cast<const uint2*>(p), x); }
__device__ __forceinline__ void load_weight8(const void* w, int32_t dtype, int col, float2 (&x)[4]) {
  if (dtype == SAPO_DTYPE_F32) load8(static_cast<const float*>(w) + col, x);
  else load8(static_cast<const __nv_bfloat16*>(w) + col, x);
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&b);
}
// 8 columns to p (fp32 or bf16 as YF says)
template <bool YF>
__device__ __forceinline__ void put8(void* p, int64_t at, const float2 (&x)[4]) {
  if (YF) {
    float* f = static_cast<float*>(p) + at;
    *reinterpret_cast<float4*>(f) = make_float4(x[0].x, x[0].y, x[1].x, x[1].y);
    *reinterpret_cast<float4*>(f + 4) = make_float4(x[2].x, x[2].y, x[3].x, x[3].y);
  } else {
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p) + at) =
        make_uint4(pack_bf16x2(x[0].x, x[0].y), pack_bf16x2(x[1].x, x[1].y), pack_bf16x2(x[2].x, x[2].y), pack_bf16x2(x[3].x, x[3].y));
  }
}


// ---------------------------------------------------------------------------- several reductions at once
// N values (1, 2, 4 or 8) per lane, each reduced over WIDTH >= N lanes (a power of two): an exchange halves how many values a lane
// still carries, so that the lanes end with one value each, lane i of the WIDTH with value i >> SHIFT, after
// N - 1 + log2(WIDTH / N) shuffles, not N log2(WIDTH).
template <int N, int WIDTH> struct Slots {
  static constexpr int LOG = N == 1 ? 0 : (N == 2 ? 1 : (N == 4 ? 2 : 3));
  static constexpr int LOG_WIDTH = WIDTH == 32 ? 5 : (WIDTH == 16 ? 4 : (WIDTH == 8 ? 3 : 2));
  static constexpr int SHIFT = LOG_WIDTH - LOG;
  static_assert(N == (1 << LOG) && WIDTH == (1 << LOG_WIDTH) && N <= WIDTH, "powers of two");
  __device__ static __forceinline__ int slot() { return (int)(threadIdx.x & (WIDTH - 1)) >> SHIFT; }
  // whether this lane is the first that holds its slot's value
  __device__ static __forceinline__ bool first() { return (threadIdx.x & ((1 << SHIFT) - 1)) == 0; }
  template <class Op>
  __device__ static __forceinline__ float reduce(float (&a)[N], Op op) {
    int d = WIDTH / 2;
    #pragma unroll
    for (int half = N / 2; half >= 1; half >>= 1) {
      const bool upper = (threadIdx.x & d) != 0;
      #pragma unroll
      for (int k = 0; k < half; ++k) {
        const float other = __shfl_xor_sync(0xffffffffu, upper ? a[k] : a[k + half], d);
        a[k] = op(upper ? a[k + half] : a[k], other);
      }
      d >>= 1;
    }
    float x = a[0];
    #pragma unroll
    for (int e = WIDTH >> (LOG + 1); e > 0; e >>= 1) x = op(x, __shfl_xor_sync(0xffffffffu, x, e));
    return x;
  }
  // slot v's value, for all lanes
  __device__ static __forceinline__ float get(float x, int v) {
    return N == 1 ? x : __shfl_sync(0xffffffffu, x, (threadIdx.x & 31 & ~(WIDTH - 1)) | (v << SHIFT));
  }
};
struct AddOp { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct MaxOp { __device__ __forceinline__ float operator()(float a, float b) const { return max_nan(a, b); } };

// ---------------------------------------------------------------------------- the quantiser
// N groups of Q8_GROUP columns at once, WIDTH lanes holding PAIRS pairs of each.  Their maxima are reduced together; the
// lanes of a slot compute its group's scale and reciprocal (once, not once per lane) and hand the reciprocal back.
// The rounding to an integer adds 1.5 2^23 (to nearest even, the integer in the last bits); the product before it is
// rounded by itself, in pairs, and the sum is scalar: a pair of both is compiled to one fma.
// bytes[v][j]: pair j of group v, in the lowest byte of each half.  scale, bad: of the lane's slot.
template <int N> struct PowerOfTwo { static constexpr int value = N == 1 ? 1 : (N == 2 ? 2 : (N <= 4 ? 4 : 8)); };
template <int N, int WIDTH, int PAIRS>
__device__ __forceinline__ void quantise(const float2 (&x)[N][PAIRS], uint2 (&bytes)[N][PAIRS], float& scale, bool& bad) {
  static_assert(N <= 8, "up to 8 groups");
  constexpr int P = PowerOfTwo<N>::value;
  using S = Slots<P, WIDTH>;
  float a[P];
  #pragma unroll
  for (int v = 0; v < P; ++v) {
    a[v] = 0.f;
    if (v >= N) continue;
    #pragma unroll
    for (int j = 0; j < PAIRS; ++j) a[v] = max_nan(a[v], max_nan(fabsf(x[v < N ? v : 0][j].x), fabsf(x[v < N ? v : 0][j].y)));
  }
  const float top = S::reduce(a, MaxOp{});
  bad = !(top < INFINITY);
  const bool some = top >= Q8_TINY && !bad;
  const float inv = some ? 127.f * __frcp_rn(top) : 0.f;
  // a group with a value that is not finite keeps no values: its scale says so wherever it is read
  scale = bad ? __int_as_float(0x7fc00000) : (some ? top * (1.f / 127.f) : 0.f);
  #pragma unroll
  for (int v = 0; v < N; ++v) {
    const float2 i2 = both(S::get(inv, v));
    #pragma unroll
    for (int j = 0; j < PAIRS; ++j) {
      const float2 p = mul2(x[v][j], i2);
      bytes[v][j] = make_uint2(__float_as_uint(__fadd_rn(p.x, 12582912.f)), __float_as_uint(__fadd_rn(p.y, 12582912.f)));
    }
  }
  if (__any_sync(0xffffffffu, bad)) {
    #pragma unroll
    for (int v = 0; v < N; ++v)
      if (S::get(bad ? 1.f : 0.f, v) != 0.f) {
        #pragma unroll
        for (int j = 0; j < PAIRS; ++j) bytes[v][j] = make_uint2(0u, 0u);
      }
  }
}
// 8 neighbouring columns' bytes as the 8-bit row holds them
__device__ __forceinline__ uint2 pack_bytes(const uint2 (&b)[4]) {
  return make_uint2(__byte_perm(__byte_perm(b[0].x, b[0].y, 0x0040), __byte_perm(b[1].x, b[1].y, 0x0040), 0x5410),
                    __byte_perm(__byte_perm(b[2].x, b[2].y, 0x0040), __byte_perm(b[3].x, b[3].y, 0x0040), 0x5410));
}

// ---------------------------------------------------------------------------- sums over the warps of a row
__device__ __forceinline__ void group_barrier(int id, int n_threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n_threads) : "memory");
}
// Sums of one or two values over a group of warps.  Each group has SLOTS places for its warps' sums, zeros in
// those that have no warp, twice: `turn` alternates, so that one barrier a sum is enough.
template <int SLOTS>
__device__ __forceinline__ float group_sum(float a, int wpr, int w, int group, float* red, int turn) {
  #pragma unroll
  for (int d = 16; d > 0; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
  if (wpr == 1) return a;
  float* r = red + (2 * group + turn) * SLOTS;
  if ((threadIdx.x & 31) == 0) r[w] = a;
  group_barrier(1 + group, wpr * 32);
  float t = 0.f;
  #pragma unroll
  for (int i = 0; i < SLOTS; i += 4) {
    const float4 o = *reinterpret_cast<const float4*>(r + i);
    t += (o.x + o.y) + (o.z + o.w);
  }
  return t;
}
// (after the first exchange half of the lanes carry one value and half the other: 6 shuffles, not 10)
template <int SLOTS>
__device__ __forceinline__ float2 group_sum2(float a, float b, int wpr, int w, int group, float2* red, int turn) {
  const bool upper = (threadIdx.x & 16) != 0;
  const float other = __shfl_xor_sync(0xffffffffu, upper ? a : b, 16);
  float x = (upper ? b : a) + other;
  #pragma unroll
  for (int d = 8; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  if (wpr == 1) {
    const float y = __shfl_xor_sync(0xffffffffu, x, 16);
    return upper ? make_float2(y, x) : make_float2(x, y);
  }
  float2* r = red + (2 * group + turn) * SLOTS;
  if ((threadIdx.x & 15) == 0) reinterpret_cast<float*>(r + w)[upper] = x;
  group_barrier(1 + group, wpr * 32);
  float2 t = make_float2(0.f, 0.f);
  #pragma unroll
  for (int i = 0; i < SLOTS; i += 2) {
    const float4 o = *reinterpret_cast<const float4*>(r + i);
    t = add2(t, add2(make_float2(o.x, o.y), make_float2(o.z, o.w)));
  }
  return t;
}

// The end of a backward block.  acc holds the sums over the rows of each of the block's groups of warps,
// [groups][2][pitch] with dgamma's columns first; they are added up in the groups' order, W columns a thread at a time, and
// become the outputs, or with several blocks the block's part of them, [2][part_pitch(H)].
__host__ __device__ constexpr int32_t part_pitch(int32_t H) { return (H + 3) & ~3; }
template <int W>
__device__ __forceinline__ void finish_columns(const NormBwdArgs& a, const float* acc, int groups, int pitch) {
  const int n = a.H / W, first = a.dgamma != nullptr ? 0 : n, last = a.dbeta != nullptr ? 2 * n : n;
  for (int i = first + threadIdx.x; i < last; i += blockDim.x) {
    const bool beta = i >= n;
    const int c = (beta ? i - n : i) * W;
    const float* from = acc + (beta ? pitch : 0) + c;
    float s[W];
    for (int k = 0; k < groups; ++k, from += 2 * pitch) {
      float x[W];
      if constexpr (W == 4) *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(from); else x[0] = *from;
      #pragma unroll
      for (int j = 0; j < W; ++j) s[j] = k == 0 ? x[j] : s[j] + x[j];
    }
    if (gridDim.x > 1) {
      float* out = a.part + ((int64_t)blockIdx.x * 2 + beta) * part_pitch(a.H) + c;
      if constexpr (W == 4) *reinterpret_cast<float4*>(out) = *reinterpret_cast<const float4*>(s); else *out = s[0];
    } else {
      float* out = (beta ? a.dbeta : a.dgamma) + c;
      #pragma unroll
      for (int j = 0; j < W; ++j) out[j] = a.accumulate ? out[j] + s[j] : s[j];
    }
  }
}

}  // namespace sapo
