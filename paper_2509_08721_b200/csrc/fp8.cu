// sapo_fp8_store: a matrix in 8-bit floating point (e4m3), one fp32 scale per row and 128 columns (activations) or per
// 128 x 128 block (weights).  With a = the largest magnitude of a group, scale = a (1/448) and q = x (448 (1/a)) rounded to
// the nearest code: the group's largest value uses the type's largest.
// HBM-bound (3 bytes an element from bf16): rows are taken in pieces of 256 columns by warps, half a warp per group, four
// pieces in flight; blocks of 128 x 128 stay in a block's registers between the search for a and the conversion.
// Measured: 151936 x 896 bf16 by blocks 62 us (6.5 TB/s, the copy rate), 16527 x 3584 by rows 38.5 us (4.7 TB/s; a warp's loads
// wait for its stores: more, smaller or shorter-lived blocks and 2 or 8 pieces were each slower, 40 to 43 us).
#include <cuda_bf16.h>

#include "common.cuh"
#include "float8.cuh"
#include "paired.cuh"

namespace sapo {

constexpr int F8S_THREADS = 256;
constexpr int F8S_PIECES = 4;       // pieces of 256 columns a warp has in flight

struct Fp8StoreArgs {
  const void* x; int64_t R; int32_t C; int64_t ld_x;
  uint8_t* q; float* scale; int64_t ld, ld_scale;
  int32_t vec_x, vec_q;             // rows start where eight values can be read, eight codes written, at once
  int32_t* status;
};

// Eight neighbouring values as they are in memory: bf16 takes four registers until it is converted.
template <class T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
  uint32_t w[4];
  __device__ __forceinline__ float at(int i) const { return __uint_as_float((i & 1) ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16); }
};
template <> struct Eight<float> {
  uint32_t w[8];
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(w[i]); }
};
template <class T>
__device__ __forceinline__ void load8(Eight<T>& e, const T* p, int left, bool vec) {      // left: columns up to the row's end
  if (vec && left >= 8) {
    #pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
      const uint4 a = reinterpret_cast<const uint4*>(p)[h];
      e.w[4 * h] = a.x; e.w[4 * h + 1] = a.y; e.w[4 * h + 2] = a.z; e.w[4 * h + 3] = a.w;
    }
    return;
  }
  #pragma unroll
  for (int i = 0; i < 2 * (int)sizeof(T); ++i) e.w[i] = 0;
  #pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i >= left) continue;
    if (sizeof(T) == 4) e.w[i % (2 * sizeof(T))] = reinterpret_cast<const uint32_t*>(p)[i];
    else e.w[i >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << (16 * (i & 1));
  }
}
// largest magnitude, as an unsigned integer: a NaN is above infinity
template <class T>
__device__ __forceinline__ uint32_t largest(const Eight<T>& e) {
  if constexpr (sizeof(T) == 2) {
    const __nv_bfloat162* b = reinterpret_cast<const __nv_bfloat162*>(e.w);
    const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(__habs2(b[0]), __habs2(b[1])), __hmax2_nan(__habs2(b[2]), __habs2(b[3])));
    const uint32_t w = *reinterpret_cast<const uint32_t*>(&m);
    return max(w << 16, w & 0xFFFF0000u);
  } else {
    uint32_t m = 0;
    #pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, e.w[i] & 0x7FFFFFFFu);
    return m;
  }
}
// codes of eight values; a group that holds no number below infinity, or only tiny ones, has inv 0 and gets zeros
template <class T>
__device__ __forceinline__ void store8(uint8_t* p, int left, bool vec, const Eight<T>& e, float inv) {
  float2 x[4];
  #pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = mul2(make_float2(e.at(2 * i), e.at(2 * i + 1)), both(inv));
  uint2 q = make_uint2(f8_pack4(x[0].x, x[0].y, x[1].x, x[1].y), f8_pack4(x[2].x, x[2].y, x[3].x, x[3].y));
  if (inv == 0.f) q = make_uint2(0, 0);
  if (vec && left >= 8) *reinterpret_cast<uint2*>(p) = q;
  else {
    #pragma unroll
    for (int i = 0; i < 8; ++i) if (i < left) p[i] = (uint8_t)((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
  }
}

// WHOLE: rows of whole pieces on boundaries for vectors, no bounds to look at.
template <class T, bool WHOLE>
__global__ void __launch_bounds__(F8S_THREADS) fp8_rows_kernel(const Fp8StoreArgs a) {
  wait_for_previous();
  const int lane = threadIdx.x & 31;
  const int64_t warp = ((int64_t)blockIdx.x * F8S_THREADS + threadIdx.x) >> 5, warps = (int64_t)gridDim.x * F8S_THREADS / 32;
  const uint32_t per_row = (uint32_t)(a.C + 255) / 256;
  const int64_t pieces = a.R * per_row;
  bool bad = false;
  for (int64_t first = warp * F8S_PIECES; first < pieces; first += warps * F8S_PIECES) {
    Eight<T> e[F8S_PIECES];
    int64_t row = first / per_row;
    int col = (int)(first - row * per_row) * 256 + lane * 8;
    const int64_t row_first = row;
    const int col_first = col;
    #pragma unroll
    for (int u = 0; u < F8S_PIECES; ++u) {
      load8(e[u], static_cast<const T*>(a.x) + row * a.ld_x + col, first + u >= pieces ? 0 : (WHOLE ? 8 : a.C - col), WHOLE || a.vec_x);
      if ((col += 256) >= (int)per_row * 256) { col -= (int)per_row * 256; ++row; }
    }
    // largest magnitudes of the pieces' groups (16 lanes each); lane j of the 16 works out the scale of piece j
    uint32_t m[F8S_PIECES], mine = 0;
    #pragma unroll
    for (int u = 0; u < F8S_PIECES; ++u) {
      m[u] = largest(e[u]);
      #pragma unroll
      for (int d = 8; d > 0; d >>= 1) m[u] = max(m[u], __shfl_xor_sync(0xFFFFFFFFu, m[u], d));
      bad |= m[u] >= 0x7F800000u;
      if ((lane & 15) == u) mine = m[u];
    }
    float scale, inv;
    f8_group(__uint_as_float(mine), scale, inv);
    row = row_first; col = col_first;
    #pragma unroll
    for (int u = 0; u < F8S_PIECES; ++u) {
      const float inv_u = __shfl_sync(0xFFFFFFFFu, inv, (lane & 16) + u);
      const int left = first + u >= pieces ? 0 : (WHOLE ? 8 : a.C - col), group = col >> 7;
      if (left > 0) store8(a.q + row * a.ld + col, left, WHOLE || a.vec_q, e[u], inv_u);
      if ((lane & 15) == u && first + u < pieces && (WHOLE || group * 128 < a.C)) a.scale[row * a.ld_scale + group] = scale;
      if ((col += 256) >= (int)per_row * 256) { col -= (int)per_row * 256; ++row; }
    }
  }
  if (bad) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
}

// One block of 128 x 128: 16 threads a row, 16 rows at a time.
template <class T>
__global__ void __launch_bounds__(F8S_THREADS) fp8_blocks_kernel(const Fp8StoreArgs a) {
  wait_for_previous();
  __shared__ uint32_t warp_max[F8S_THREADS / 32];
  const uint32_t across = (uint32_t)(a.C + 127) / 128;
  const int64_t br = blockIdx.x / across;
  const int bc = (int)(blockIdx.x - br * across);
  const int col = bc * 128 + (threadIdx.x & 15) * 8, left = a.C - col;
  const int64_t row0 = br * 128 + (threadIdx.x >> 4);
  Eight<T> e[8];
  uint32_t m = 0;
  #pragma unroll
  for (int u = 0; u < 8; ++u) load8(e[u], static_cast<const T*>(a.x) + (row0 + 16 * u) * a.ld_x + col, row0 + 16 * u < a.R ? left : 0, a.vec_x);
  #pragma unroll
  for (int u = 0; u < 8; ++u) m = max(m, largest(e[u]));
  m = __reduce_max_sync(0xFFFFFFFFu, m);
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = m;
  __syncthreads();
  #pragma unroll
  for (int w = 0; w < F8S_THREADS / 32; ++w) m = max(m, warp_max[w]);
  float scale, inv;
  f8_group(__uint_as_float(m), scale, inv);
  #pragma unroll
  for (int u = 0; u < 8; ++u)
    if (left > 0 && row0 + 16 * u < a.R) store8(a.q + (row0 + 16 * u) * a.ld + col, left, a.vec_q, e[u], inv);
  if (threadIdx.x == 0) {
    a.scale[br * a.ld_scale + bc] = scale;
    if (m >= 0x7F800000u) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
  }
}

template <class T, bool WHOLE>
static int launch_fp8_rows(const Fp8StoreArgs& a, int sms, cudaStream_t st) {
  static int resident[MAX_DEVICES] = {0};
  const int dev = current_device();
  if (dev < 0) return SAPO_ERR_CUDA;
  if (resident[dev] == 0) resident[dev] = resident_blocks_per_sm(fp8_rows_kernel<T, WHOLE>, F8S_THREADS);
  const int64_t turns = ceil_div<int64_t>(a.R * ceil_div<int64_t>(a.C, 256), F8S_PIECES);
  const int64_t most = (int64_t)sms * resident[dev], need = ceil_div<int64_t>(turns, F8S_THREADS / 32);
  return launch_overlapped(fp8_rows_kernel<T, WHOLE>, dim3((unsigned)(need < most ? need : most)), F8S_THREADS, 0, 0, st, a);
}

template <class T>
static int launch_fp8_store(const Fp8StoreArgs& a, bool blocks, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return SAPO_ERR_CUDA;
  KernelScope scope(SAPO_K_FP8_STORE, st);
  if (blocks) {
    const int64_t n = ceil_div<int64_t>(a.R, 128) * ceil_div<int64_t>(a.C, 128);
    if (n > 0x7FFFFFFF) return SAPO_ERR_UNSUPPORTED_SHAPE;
    return launch_overlapped(fp8_blocks_kernel<T>, dim3((unsigned)n), F8S_THREADS, 0, 0, st, a);
  }
  return a.vec_x && a.vec_q && a.C % 256 == 0 ? launch_fp8_rows<T, true>(a, sms, st) : launch_fp8_rows<T, false>(a, sms, st);
}

}  // namespace sapo

extern "C" int sapo_fp8_store(const void* x, int32_t x_dtype, int64_t R, int32_t C, int64_t ld_x, const sapo_fp8* h_out,
                              int32_t* status, void* stream) {
  using namespace sapo;
  if (!h_out || !status || R < 0 || C < 1 || ld_x < C || (x_dtype != SAPO_DTYPE_BF16 && x_dtype != SAPO_DTYPE_F32)) return SAPO_ERR_INVALID_ARG;
  const sapo_fp8& o = *h_out;
  if (o.ld < C || o.ld_scale < ceil_div<int64_t>(C, 128) || (o.blocks != 0 && o.blocks != 1)) return SAPO_ERR_INVALID_ARG;
  if (R == 0) return SAPO_OK;
  if (!x || !o.data || !o.scale) return SAPO_ERR_INVALID_ARG;
  const size_t size = x_dtype == SAPO_DTYPE_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(x) % size || reinterpret_cast<uintptr_t>(o.scale) % 4) return SAPO_ERR_INVALID_ARG;
  const Fp8StoreArgs a{x, R, C, ld_x, static_cast<uint8_t*>(o.data), o.scale, o.ld, o.ld_scale,
                       aligned16(x) && (R == 1 || (ld_x * (int64_t)size) % 16 == 0),
                       (reinterpret_cast<uintptr_t>(o.data) & 7u) == 0 && (R == 1 || o.ld % 8 == 0), status};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return x_dtype == SAPO_DTYPE_BF16 ? launch_fp8_store<__nv_bfloat16>(a, o.blocks != 0, st) : launch_fp8_store<float>(a, o.blocks != 0, st);
}
