// The norm in front of the LM head (layer norm or RMS norm), forward and backward, and activation
// checkpoints in 8 bits: sapo_norm_fwd, sapo_norm_replay, sapo_norm_bwd, sapo_ckpt8_store,
// sapo_ckpt8_restore.  All of them pass over [T, H] once; a row stays in the registers of the
// threads that loaded it.
//
// Layout of a row over threads: a thread owns vectors of 8 consecutive columns, vector i of a row
// belongs to thread i mod tpr (tpr threads per row, a power of two), at most NV_MAX vectors a
// thread.  A group of 128 columns that shares a checkpoint scale is then 16 neighbouring threads.
#include <cuda_bf16.h>
#include <math.h>

#include <type_traits>

#include "common.cuh"

namespace sapo {

constexpr int Q8_GROUP = 128;            // columns that share one checkpoint scale
constexpr int NORM_MAX_H = 16384;
constexpr int NORM_THREADS = 256;
constexpr int NORM_MAX_THREADS = 512;    // one row of NORM_MAX_H columns
constexpr int NV_MAX = 4;
constexpr int SMEM_MAX = 220 * 1024;     // shared memory a block may take for its rows
// A group whose largest magnitude is below this is stored as zeros: 127 (1 / amax) would overflow.
constexpr float Q8_TINY = 1.5046328e-36f;   // 2^-119

enum { KIND_LAYER = SAPO_NORM_LAYER, KIND_RMS = SAPO_NORM_RMS };

// ---------------------------------------------------------------------------- loads and stores of 8 columns
// n: how many of the 8 columns exist (the rest read as zero and are not written).  VEC: rows start on
// 16-byte boundaries and so does every whole vector.
template <bool VEC>
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
  if (VEC && n == 8) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    return;
  }
  #pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : 0.f;
}
template <bool VEC>
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int n, float (&v)[8]) {
  if (VEC && n == 8) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    #pragma unroll
    for (int j = 0; j < 4; ++j) { v[2 * j] = __uint_as_float(w[j] << 16); v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
    return;
  }
  #pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = j < n ? __bfloat162float(p[j]) : 0.f;
}
template <bool VEC>
__device__ __forceinline__ void load8(const int8_t* p, int n, float (&v)[8]) {
  if (VEC && n == 8) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    #pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = (float)(int8_t)(u.x >> (8 * j));
      v[4 + j] = (float)(int8_t)(u.y >> (8 * j));
    }
    return;
  }
  #pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = j < n ? (float)p[j] : 0.f;
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&b);
}
template <bool VEC>
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
  if (VEC && n == 8) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    return;
  }
  #pragma unroll
  for (int j = 0; j < 8; ++j) if (j < n) p[j] = v[j];
}
template <bool VEC>
__device__ __forceinline__ void store8(__nv_bfloat16* p, int n, const float (&v)[8]) {
  if (VEC && n == 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                              pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    return;
  }
  #pragma unroll
  for (int j = 0; j < 8; ++j) if (j < n) p[j] = __float2bfloat16_rn(v[j]);
}
template <bool VEC>
__device__ __forceinline__ void store8(int8_t* p, int n, const int (&q)[8]) {
  if (VEC && n == 8) {
    uint2 u = make_uint2(0u, 0u);
    #pragma unroll
    for (int j = 0; j < 4; ++j) {
      u.x |= (uint32_t)(uint8_t)q[j] << (8 * j);
      u.y |= (uint32_t)(uint8_t)q[4 + j] << (8 * j);
    }
    *reinterpret_cast<uint2*>(p) = u;
    return;
  }
  #pragma unroll
  for (int j = 0; j < 8; ++j) if (j < n) p[j] = (int8_t)q[j];
}

// a matrix of fp32 or bf16 rows whose type is known at run time (the branch is the same for all threads)
struct Mat { void* p; int64_t ld; int32_t dtype; };
template <bool VEC>
__device__ __forceinline__ void load8(const Mat& m, int64_t row, int col, int n, float (&v)[8]) {
  if (m.dtype == SAPO_DTYPE_F32) load8<VEC>(static_cast<const float*>(m.p) + row * m.ld + col, n, v);
  else load8<VEC>(static_cast<const __nv_bfloat16*>(m.p) + row * m.ld + col, n, v);
}
template <bool VEC>
__device__ __forceinline__ void store8(const Mat& m, int64_t row, int col, int n, const float (&v)[8]) {
  if (m.dtype == SAPO_DTYPE_F32) store8<VEC>(static_cast<float*>(m.p) + row * m.ld + col, n, v);
  else store8<VEC>(static_cast<__nv_bfloat16*>(m.p) + row * m.ld + col, n, v);
}
// per-column weights, fp32 or bf16; `vec`: the array starts on a 16-byte boundary
__device__ __forceinline__ void load_weight8(const void* w, int32_t dtype, bool vec, int col, int n, float (&v)[8]) {
  if (dtype == SAPO_DTYPE_F32) {
    if (vec) load8<true>(static_cast<const float*>(w) + col, n, v);
    else load8<false>(static_cast<const float*>(w) + col, n, v);
  } else {
    if (vec) load8<true>(static_cast<const __nv_bfloat16*>(w) + col, n, v);
    else load8<false>(static_cast<const __nv_bfloat16*>(w) + col, n, v);
  }
}

struct Q8Mat { int8_t* p; float* scale; int64_t ld, ld_scale; };

// ---------------------------------------------------------------------------- sums over a row
// A thread's place: row `r` of the block's rows, thread `lane` of the row's tpr threads.
struct Place { int r, lane, tpr, rows_per_block; };
__device__ __forceinline__ Place place_of(int tpr) {
  Place p;
  p.tpr = tpr;
  p.rows_per_block = blockDim.x / tpr;
  p.r = threadIdx.x / tpr;
  p.lane = threadIdx.x - p.r * tpr;
  return p;
}
// Sum of x over the threads of a row; all threads of the block call it together.  sh: one float per
// warp, of its own for each call between two barriers.
__device__ __forceinline__ float row_sum(float x, const Place& p, float* sh) {
  const int w = p.tpr < 32 ? p.tpr : 32;
  for (int d = w >> 1; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  if (p.tpr <= 32) return x;
  const int warps = p.tpr >> 5;
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
  __syncthreads();
  float t = 0.f;
  for (int i = 0; i < warps; ++i) t += sh[p.r * warps + i];
  return t;
}

// ---------------------------------------------------------------------------- 8-bit groups
// Quantise 8 columns of a group of Q8_GROUP: the 16 threads (fewer when the row has fewer vectors) that
// hold the group agree on its largest magnitude.  Called by whole warps.
__device__ __forceinline__ void quantise8(const float (&v)[8], int width, int (&q)[8], float& scale, bool& bad) {
  float a = 0.f;
  bool nan = false;
  #pragma unroll
  for (int j = 0; j < 8; ++j) { a = fmaxf(a, fabsf(v[j])); nan |= v[j] != v[j]; }
  if (nan) a = INFINITY;                       // fmaxf drops a NaN
  for (int d = width >> 1; d > 0; d >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, d));
  bad = !(a < INFINITY);
  const bool some = a >= Q8_TINY && !bad;
  const float inv = some ? 127.f * __frcp_rn(a) : 0.f;
  // a group with a value that is not finite keeps no values: its scale says so wherever it is read
  scale = bad ? __int_as_float(0x7fc00000) : (some ? a * (1.f / 127.f) : 0.f);
  #pragma unroll
  for (int j = 0; j < 8; ++j) q[j] = some ? __float2int_rn(v[j] * inv) : 0;
}

// ---------------------------------------------------------------------------- forward
// x to y (and to an 8-bit checkpoint): mean and variance from the row in registers (two passes
// there, one over memory).  REPLAY: x comes from a checkpoint and mean / rstd are the stored ones.
struct NormFwdArgs {
  Mat x, y; Q8Mat q; const void* gamma; const void* beta; int32_t w_dtype, w_vec, kind; float eps;
  float* mean; float* rstd; int64_t T; int32_t H, tpr; int32_t* status;
};

template <int NV, bool VEC, bool REPLAY>
__global__ void __launch_bounds__(NORM_MAX_THREADS) norm_fwd_kernel(NormFwdArgs a) {
  __shared__ float sh[2][NORM_MAX_THREADS / 32];
  const Place p = place_of(a.tpr);
  const float inv_h = 1.f / (float)a.H;
  const int gw = a.tpr < 16 ? a.tpr : 16;
  for (int64_t base = (int64_t)blockIdx.x * p.rows_per_block; base < a.T; base += (int64_t)gridDim.x * p.rows_per_block) {
    const int64_t row = base + p.r;
    const bool live = row < a.T;
    float v[NV][8];
    #pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * a.tpr + p.lane) * 8;
      const int n = live ? min(8, max(0, a.H - col)) : 0;
      if (REPLAY) {
        load8<VEC>(a.q.p + row * a.q.ld + col, n, v[i]);
        const float s = n > 0 ? a.q.scale[row * a.q.ld_scale + col / Q8_GROUP] : 0.f;
        #pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= s;
      } else {
        load8<VEC>(a.x, row, col, n, v[i]);
      }
    }
    float mean = 0.f, rstd = 0.f;
    if (REPLAY) {
      if (live) { mean = a.kind == KIND_LAYER ? a.mean[row] : 0.f; rstd = a.rstd[row]; }
    } else {
      if (a.kind == KIND_LAYER) {
        float s = 0.f;
        #pragma unroll
        for (int i = 0; i < NV; ++i)
          #pragma unroll
          for (int j = 0; j < 8; ++j) s += v[i][j];
        mean = row_sum(s, p, sh[0]) * inv_h;
      }
      float s2 = 0.f;
      #pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int col = (i * a.tpr + p.lane) * 8;
        #pragma unroll
        for (int j = 0; j < 8; ++j) { const float d = col + j < a.H ? v[i][j] - mean : 0.f; s2 = fmaf(d, d, s2); }
      }
      const float var = row_sum(s2, p, sh[1]) * inv_h;
      rstd = 1.f / sqrtf(var + a.eps);
      if (a.tpr > 32) __syncthreads();             // the next row writes sh again
      if (live && p.lane == 0) {
        if (a.mean != nullptr && a.kind == KIND_LAYER) a.mean[row] = mean;
        if (a.rstd != nullptr) a.rstd[row] = rstd;
      }
    }
    #pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * a.tpr + p.lane) * 8;
      const int n = live ? min(8, max(0, a.H - col)) : 0;
      if (!REPLAY && a.q.p != nullptr) {
        int q[8]; float scale; bool bad;
        quantise8(v[i], gw, q, scale, bad);
        if (n > 0) {
          store8<VEC>(a.q.p + row * a.q.ld + col, n, q);
          if (col % Q8_GROUP == 0) {
            a.q.scale[row * a.q.ld_scale + col / Q8_GROUP] = scale;
            if (bad) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
          }
        }
      }
      if (n > 0) {
        float g[8], b[8];
        #pragma unroll
        for (int j = 0; j < 8; ++j) { g[j] = 1.f; b[j] = 0.f; }
        if (a.gamma != nullptr) load_weight8(a.gamma, a.w_dtype, a.w_vec, col, n, g);
        if (a.beta != nullptr) load_weight8(a.beta, a.w_dtype, a.w_vec, col, n, b);
        #pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = fmaf((v[i][j] - mean) * rstd, g[j], b[j]);
        store8<VEC>(a.y, row, col, n, v[i]);
      }
    }
  }
}

// ---------------------------------------------------------------------------- checkpoint alone
struct Ckpt8Args { Mat x; Q8Mat q; int64_t T; int32_t H, nvec, vec_log2; int32_t* status; };

// One vector of 8 columns per thread, rows cut into a power of two of vectors so that a group's 16
// threads are neighbours in a warp.
template <bool VEC, bool RESTORE>
__global__ void __launch_bounds__(256) ckpt8_kernel(Ckpt8Args a) {
  const int gw = min(16, 1 << a.vec_log2);
  const int64_t total = a.T << a.vec_log2;
  const int64_t padded = round_up<int64_t>(total, 32);       // whole warps take part in the shuffles
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < padded; i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t row = i >> a.vec_log2;
    const int col = (int)(i & ((1 << a.vec_log2) - 1)) * 8;
    const int n = row < a.T ? min(8, max(0, a.H - col)) : 0;
    float v[8];
    if (RESTORE) {
      if (n == 0) continue;
      load8<VEC>(a.q.p + row * a.q.ld + col, n, v);
      const float s = a.q.scale[row * a.q.ld_scale + col / Q8_GROUP];
      #pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= s;
      store8<VEC>(a.x, row, col, n, v);
    } else {
      load8<VEC>(a.x, row, col, n, v);
      int q[8]; float scale; bool bad;
      quantise8(v, gw, q, scale, bad);
      if (n == 0) continue;
      store8<VEC>(a.q.p + row * a.q.ld + col, n, q);
      if (col % Q8_GROUP == 0) {
        a.q.scale[row * a.q.ld_scale + col / Q8_GROUP] = scale;
        if (bad) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
      }
    }
  }
}

// ---------------------------------------------------------------------------- backward
// Per row, with xh = (x - mean) rstd and g = dy gamma:
//   dx = rstd (g - [layer] mean(g) - xh mean(g xh)),
// and over the rows dgamma = sum dy xh, dbeta = sum dy.  A thread keeps the sums of its columns in
// registers over all rows of its block; the blocks' sums go to `part` ([blocks][2][H]) and
// norm_reduce_kernel adds them up in block order, so that the result does not depend on timing.
struct NormBwdArgs {
  Mat dy, x, dx; Q8Mat q; const void* gamma; int32_t w_dtype, w_vec, kind; const float* mean; const float* rstd;
  int64_t T; int32_t H, tpr; float* part; float* dgamma; float* dbeta; int32_t accumulate;
};

template <int NV, bool VEC, bool FROM_Q8>
__global__ void __launch_bounds__(NORM_MAX_THREADS) norm_bwd_kernel(NormBwdArgs a) {
  __shared__ float sh[2][NORM_MAX_THREADS / 32];
  extern __shared__ float cols[];                  // [2][H], when the block holds several rows
  const Place p = place_of(a.tpr);
  const float inv_h = 1.f / (float)a.H;
  float gam[NV][8], dg[NV][8], db[NV][8];
  #pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = (i * a.tpr + p.lane) * 8;
    const int n = min(8, max(0, a.H - col));
    #pragma unroll
    for (int j = 0; j < 8; ++j) { gam[i][j] = 1.f; dg[i][j] = 0.f; db[i][j] = 0.f; }
    if (a.gamma != nullptr) load_weight8(a.gamma, a.w_dtype, a.w_vec, col, n, gam[i]);
  }
  for (int64_t base = (int64_t)blockIdx.x * p.rows_per_block; base < a.T; base += (int64_t)gridDim.x * p.rows_per_block) {
    const int64_t row = base + p.r;
    const bool live = row < a.T;
    float xh[NV][8], dy[NV][8];
    #pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * a.tpr + p.lane) * 8;
      const int n = live ? min(8, max(0, a.H - col)) : 0;
      load8<VEC>(a.dy, row, col, n, dy[i]);
      if (FROM_Q8) {
        load8<VEC>(a.q.p + row * a.q.ld + col, n, xh[i]);
        const float s = n > 0 ? a.q.scale[row * a.q.ld_scale + col / Q8_GROUP] : 0.f;
        #pragma unroll
        for (int j = 0; j < 8; ++j) xh[i][j] *= s;
      } else {
        load8<VEC>(a.x, row, col, n, xh[i]);
      }
    }
    const float mean = live && a.kind == KIND_LAYER ? a.mean[row] : 0.f;
    const float rstd = live ? a.rstd[row] : 0.f;
    float s1 = 0.f, s2 = 0.f;
    #pragma unroll
    for (int i = 0; i < NV; ++i) {
      #pragma unroll
      for (int j = 0; j < 8; ++j) {
        xh[i][j] = (xh[i][j] - mean) * rstd;        // columns past H: dy is zero there
        const float g = dy[i][j] * gam[i][j];
        s1 += g;
        s2 = fmaf(g, xh[i][j], s2);
        dg[i][j] = fmaf(dy[i][j], xh[i][j], dg[i][j]);
        db[i][j] += dy[i][j];
      }
    }
    const float c1 = a.kind == KIND_LAYER ? row_sum(s1, p, sh[0]) * inv_h : 0.f;
    const float c2 = row_sum(s2, p, sh[1]) * inv_h;
    if (a.tpr > 32) __syncthreads();               // the next row writes sh again
    #pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * a.tpr + p.lane) * 8;
      const int n = live ? min(8, max(0, a.H - col)) : 0;
      if (n > 0) {
        #pragma unroll
        for (int j = 0; j < 8; ++j) dy[i][j] = rstd * (dy[i][j] * gam[i][j] - c1 - xh[i][j] * c2);
        store8<VEC>(a.dx, row, col, n, dy[i]);
      }
    }
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (a.dgamma == nullptr && a.dbeta == nullptr) return;
  // the rows of a warp, then the warps' rows one after the other
  for (int d = 16; d >= a.tpr; d >>= 1) {
    #pragma unroll
    for (int i = 0; i < NV; ++i)
      #pragma unroll
      for (int j = 0; j < 8; ++j) {
        dg[i][j] += __shfl_xor_sync(0xffffffffu, dg[i][j], d);
        db[i][j] += __shfl_xor_sync(0xffffffffu, db[i][j], d);
      }
  }
  const int share = a.tpr < 32 ? 32 : a.tpr;         // threads that hold one copy of the columns
  const int copies = blockDim.x / share;
  const int c = threadIdx.x / share;
  const bool holds = (threadIdx.x & (share - 1)) < a.tpr;
  const int64_t H = a.H;
  for (int k = 0; k < copies; ++k) {
    if (k == c && holds) {
      #pragma unroll
      for (int i = 0; i < NV; ++i)
        #pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int col = (i * a.tpr + p.lane) * 8 + j;
          if (col >= a.H) continue;
          float g = dg[i][j], b = db[i][j];
          if (k > 0) { g += cols[col]; b += cols[H + col]; }
          if (k + 1 < copies) { cols[col] = g; cols[H + col] = b; continue; }
          if (gridDim.x > 1) {
            float* out = a.part + (int64_t)blockIdx.x * 2 * H;
            out[col] = g; out[H + col] = b;
          } else {
            if (a.dgamma != nullptr) a.dgamma[col] = a.accumulate ? a.dgamma[col] + g : g;
            if (a.dbeta != nullptr) a.dbeta[col] = a.accumulate ? a.dbeta[col] + b : b;
          }
        }
    }
    __syncthreads();
  }
}

// dgamma (blockIdx.y 0) and dbeta (1): the sum over the blocks' parts, 32 columns per block, one warp
// for every 32nd part.
__global__ void __launch_bounds__(1024)
norm_reduce_kernel(const float* __restrict__ part, int n_parts, int32_t H, float* dgamma, float* dbeta, int accumulate) {
  __shared__ float sh[32][33];
  float* out = blockIdx.y == 0 ? dgamma : dbeta;
  if (out == nullptr) { asm volatile("griddepcontrol.wait;" ::: "memory"); return; }
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + lane;
  float s = 0.f;
  asm volatile("griddepcontrol.wait;" ::: "memory");      // launched while the backward's last blocks still run
  if (col < H)
    for (int b = w; b < n_parts; b += 32) s += part[((int64_t)b * 2 + blockIdx.y) * H + col];
  sh[w][lane] = s;
  __syncthreads();
  // transposed: warp w now holds the 32 sums of column w
  float t = sh[lane][w];
  #pragma unroll
  for (int d = 16; d > 0; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
  const int c = blockIdx.x * 32 + w;
  if (lane == 0 && c < H) out[c] = accumulate ? out[c] + t : t;
}

// ---------------------------------------------------------------------------- rows through shared memory
// The kernels for rows of more than 128 columns, a multiple of 8, that start on 16-byte boundaries.
// A row belongs to the `wpr` warps of a group; warp w of them owns VPL * 256 consecutive columns, lane l
// of it the vectors of 8 columns (w VPL + v) 32 + l, v < VPL.  Each warp streams its part of the group's
// next STAGES - 1 rows into shared memory with asynchronous copies while it works on the current one, so
// the bytes in flight do not depend on registers or on how long a row's sums take.  Only lanes of the
// same warp read what a lane copied: the wait for a row is one __syncwarp.
// What then bounds a row kernel is instruction issue (at the copy bandwidth an SM has to finish 4 to 6
// columns per clock), so the arithmetic is done in pairs (fma.rn.f32x2 and its kin, each half rounded
// like the scalar operation) and every vector is whole.
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
// (predicated, not branched around: a lane whose columns do not exist copies nothing)
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool exists) {
  if constexpr (BYTES == 16)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}"
                 ::"r"(dst), "l"(src), "r"((uint32_t)exists) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p cp.async.ca.shared.global [%0], [%1], %3;\n\t}"
                 ::"r"(dst), "l"(src), "r"((uint32_t)exists), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void group_barrier(int id, int n_threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n_threads) : "memory");
}

#define SAPO_F32X2(name, ptx)                                                                             \
  __device__ __forceinline__ float2 name(float2 a, float2 b) {                                            \
    float2 d;                                                                                             \
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t" ptx                 \
        " d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"                                                          \
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));                                 \
    return d;                                                                                             \
  }
SAPO_F32X2(add2, "add.rn.f32x2")
SAPO_F32X2(mul2, "mul.rn.f32x2")
#undef SAPO_F32X2
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

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
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
// Quantises N groups whose 16 threads (half a warp) hold whole vectors x[v], v < N; called by whole warps.
// The maxima are reduced together: each exchange halves how many groups a lane still carries, so that at the
// end lane (v << shift) of the half warp has group v's, computes its scale and reciprocal (once, not once per lane)
// and hands the reciprocal back.  The rounding to an integer adds 1.5 2^23 (to nearest even, the integer in
// the last bits); the product before it is rounded by itself, in pairs, and the sum is scalar: a pair of both
// is compiled to one fma.
// scale, bad: of group `slot` = (lane & 15) >> shift, in all lanes (a slot may be N or more: then 0 and false).
template <int N>
__device__ __forceinline__ void quantise(const float2 (&x)[N][4], uint2 (&q)[N], int& slot, float& scale, bool& bad) {
  constexpr int P = N == 1 ? 1 : (N == 2 ? 2 : (N <= 4 ? 4 : 8));           // N rounded up to a power of two
  constexpr int SHIFT = P == 1 ? 4 : (P == 2 ? 3 : (P == 4 ? 2 : 1));
  static_assert(N <= 8, "a half warp reduces up to 8 groups");
  const int lane = threadIdx.x & 31;
  float a[P];
  #pragma unroll
  for (int v = 0; v < P; ++v)
    a[v] = v >= N ? 0.f
                  : max_nan(max_nan(max_nan(fabsf(x[v < N ? v : 0][0].x), fabsf(x[v < N ? v : 0][0].y)),
                                    max_nan(fabsf(x[v < N ? v : 0][1].x), fabsf(x[v < N ? v : 0][1].y))),
                            max_nan(max_nan(fabsf(x[v < N ? v : 0][2].x), fabsf(x[v < N ? v : 0][2].y)),
                                    max_nan(fabsf(x[v < N ? v : 0][3].x), fabsf(x[v < N ? v : 0][3].y))));
  int d = 8;
  #pragma unroll
  for (int half = P / 2; half >= 1; half >>= 1) {
    const bool upper = (lane & d) != 0;
    #pragma unroll
    for (int k = 0; k < half; ++k) {
      const float other = __shfl_xor_sync(0xffffffffu, upper ? a[k] : a[k + half], d);
      a[k] = max_nan(upper ? a[k + half] : a[k], other);
    }
    d >>= 1;
  }
  for (; d > 0; d >>= 1) a[0] = max_nan(a[0], __shfl_xor_sync(0xffffffffu, a[0], d));
  slot = (lane & 15) >> SHIFT;
  bad = !(a[0] < INFINITY);
  const bool some = a[0] >= Q8_TINY && !bad;
  const float inv = some ? 127.f * __frcp_rn(a[0]) : 0.f;
  // a group with a value that is not finite keeps no values: its scale says so wherever it is read
  scale = bad ? __int_as_float(0x7fc00000) : (some ? a[0] * (1.f / 127.f) : 0.f);
  #pragma unroll
  for (int v = 0; v < N; ++v) {
    const float2 i2 = both(P == 1 ? inv : __shfl_sync(0xffffffffu, inv, (lane & 16) | (v << SHIFT)));
    uint32_t n[8];
    #pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 p = mul2(x[v][j], i2);
      n[2 * j] = __float_as_uint(__fadd_rn(p.x, 12582912.f));
      n[2 * j + 1] = __float_as_uint(__fadd_rn(p.y, 12582912.f));
    }
    q[v] = make_uint2(__byte_perm(__byte_perm(n[0], n[1], 0x0040), __byte_perm(n[2], n[3], 0x0040), 0x5410),
                      __byte_perm(__byte_perm(n[4], n[5], 0x0040), __byte_perm(n[6], n[7], 0x0040), 0x5410));
  }
  if (__any_sync(0xffffffffu, bad)) {
    #pragma unroll
    for (int v = 0; v < N; ++v)
      if (__shfl_sync(0xffffffffu, (int)bad, (lane & 16) | (v << SHIFT))) q[v] = make_uint2(0u, 0u);
  }
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

// Checkpoints alone, whole vectors: half a warp takes a group of 128 columns, CKPT_GROUPS of them with all
// loads before the first use.  Row and group of a half-warp's next group follow from those of its last one.
constexpr int CKPT_GROUPS = 4;
template <class TX, bool RESTORE>
__global__ void __launch_bounds__(256) ckpt8_vec_kernel(Ckpt8Args a, int64_t step_rows, int32_t step_groups) {
  const int32_t groups = ceil_div(a.H, Q8_GROUP);
  const int64_t id = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 4;
  const int col_in = (threadIdx.x & 15) * 8;
  int64_t row = id / groups;
  int32_t g = (int32_t)(id - row * groups);
  auto next = [&] { row += step_rows; g += step_groups; if (g >= groups) { g -= groups; ++row; } };
  TX* x = static_cast<TX*>(a.x.p);
  // (both halves of a warp stay as long as one of them has rows: they agree on shuffles)
  while (__any_sync(0xffffffffu, row < a.T)) {
    int64_t rows[CKPT_GROUPS]; int32_t cols[CKPT_GROUPS]; bool live[CKPT_GROUPS];
    float2 v[CKPT_GROUPS][4]; float s[CKPT_GROUPS];
    #pragma unroll
    for (int k = 0; k < CKPT_GROUPS; ++k) {
      rows[k] = row; cols[k] = g * Q8_GROUP + col_in;
      live[k] = row < a.T && cols[k] < a.H;
      s[k] = 0.f;
      #pragma unroll
      for (int j = 0; j < 4; ++j) v[k][j] = both(0.f);
      if (live[k]) {
        if (RESTORE) { load8(a.q.p + row * a.q.ld + cols[k], v[k]); s[k] = a.q.scale[row * a.q.ld_scale + g]; }
        else load8(x + row * a.x.ld + cols[k], v[k]);
      }
      next();
    }
    if (RESTORE) {
      #pragma unroll
      for (int k = 0; k < CKPT_GROUPS; ++k) {
        #pragma unroll
        for (int j = 0; j < 4; ++j) v[k][j] = mul2(v[k][j], both(s[k]));
        if (live[k]) put8<sizeof(TX) == 4>(x, rows[k] * a.x.ld + cols[k], v[k]);
      }
    } else {
      uint2 q[CKPT_GROUPS];
      int slot; float scale; bool bad;
      quantise<CKPT_GROUPS>(v, q, slot, scale, bad);
      #pragma unroll
      for (int k = 0; k < CKPT_GROUPS; ++k) {
        if (live[k]) *reinterpret_cast<uint2*>(a.q.p + rows[k] * a.q.ld + cols[k]) = q[k];
        if (slot == k && (threadIdx.x & 3) == 0 && rows[k] < a.T) {     // (that lane's own columns may be past the row)
          a.q.scale[rows[k] * a.q.ld_scale + cols[k] / Q8_GROUP] = scale;
          if (bad) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
        }
      }
    }
  }
}

// One warp's part of a row of TX in shared memory: VPL * 256 elements.
template <class TX, int VPL>
struct WarpRow {
  static constexpr int BYTES = VPL * 256 * (int)sizeof(TX);
  // Where lane `lane` of the warp copies from in the warp's part of a row, and to.
  static constexpr int LANE = sizeof(TX) == 4 ? 4 : 8, PER_V = sizeof(TX) == 4 ? 2 : 1;
  __device__ static __forceinline__ int lane_dst(int lane) {
    return sizeof(TX) == 4 ? (lane ^ ((lane >> 3) & 1)) * 16 : lane * 8 * (int)sizeof(TX);
  }
  // dst, src: with the lane's offsets; cols: how many of the warp's columns exist (a multiple of 8)
  __device__ static __forceinline__ void copy(uint32_t dst, const TX* src, int cols, int lane) {
    // fp32: neighbouring lanes copy neighbouring 16 bytes; a lane then reads two of them in a row, so pieces
    // are stored with the lowest bit of their index flipped in every other eight: no bank conflicts
    constexpr int B = LANE * (int)sizeof(TX);
    #pragma unroll
    for (int v = 0; v < PER_V * VPL; ++v)
      copy_async<B>(dst + v * 32 * B, src + v * 32 * LANE, v * 32 * LANE + lane * LANE < cols);
  }
  // the lane's vector v
  __device__ static __forceinline__ void read(const uint8_t* at, int v, int lane, float2 (&x)[4]) {
    if constexpr (sizeof(TX) == 4) {
      const int f = (lane >> 2) & 1;
      const float4 a = *reinterpret_cast<const float4*>(at + v * 1024 + (2 * lane + f) * 16);
      const float4 b = *reinterpret_cast<const float4*>(at + v * 1024 + (2 * lane + 1 - f) * 16);
      x[0] = make_float2(a.x, a.y); x[1] = make_float2(a.z, a.w); x[2] = make_float2(b.x, b.y); x[3] = make_float2(b.z, b.w);
    } else {
      load8(reinterpret_cast<const TX*>(at) + (v * 32 + lane) * 8, x);
    }
  }
};

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

template <class TX, int VPL> struct FwdRing {
  static constexpr int STAGE_BYTES = NORM_THREADS / 32 * WarpRow<TX, VPL>::BYTES;
  static constexpr int STAGES = STAGE_BYTES <= 16384 ? 4 : (STAGE_BYTES <= 26624 ? 3 : 2);
  static int smem(int H) { return STAGES * STAGE_BYTES + 2 * H * (int)sizeof(float); }   // and the weights
};

// Zeros where the warp's columns do not exist: nothing is ever copied there, and zeros add nothing to sums.
__device__ __forceinline__ void clear_stages(uint8_t* mine, int bytes, int stages, int stage_bytes, int lane) {
  for (int s = 0; s < stages; ++s)
    for (int i = lane * 16; i < bytes; i += 512) *reinterpret_cast<uint4*>(mine + s * stage_bytes + i) = make_uint4(0u, 0u, 0u, 0u);
  __syncwarp();
}
// TX int8_t: replay from a checkpoint (a.q), statistics given.
template <class TX, int VPL>
__global__ void __launch_bounds__(NORM_THREADS, 2) norm_fwd_ring_kernel(NormFwdArgs a, int wpr) {
  constexpr bool REPLAY = sizeof(TX) == 1;
  constexpr int S = FwdRing<TX, VPL>::STAGES, WARPS = NORM_THREADS / 32;
  using Row = WarpRow<TX, VPL>;
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ __align__(16) float red[2 * WARPS * WARPS];   // [group][turn][slots]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int group = warp / wpr, w = warp - group * wpr;
  const int64_t step = (int64_t)gridDim.x * (WARPS / wpr);
  const int64_t row0 = (int64_t)blockIdx.x * (WARPS / wpr) + group;
  const int col0 = w * VPL * 256 + lane * 8;            // the lane's first column, and
  const int left = a.H - col0;                          // what is left of the row there: vector v exists if 256 v < left
  const int cols = a.H - w * VPL * 256;
  const int64_t ld = REPLAY ? a.q.ld : a.x.ld;
  const TX* src = (REPLAY ? reinterpret_cast<const TX*>(a.q.p) : static_cast<const TX*>(a.x.p)) +
                  row0 * ld + w * VPL * 256 + lane * Row::LANE;
  constexpr int STAGE_BYTES = WARPS * Row::BYTES;
  uint8_t* mine = ring + warp * Row::BYTES;
  for (int i = threadIdx.x; i < 2 * WARPS * WARPS; i += NORM_THREADS) red[i] = 0.f;
  if (cols < VPL * 256) clear_stages(mine, Row::BYTES, S, STAGE_BYTES, lane);
  const uint32_t dst = smem_addr(mine) + Row::lane_dst(lane);
  constexpr int LANES_PER_SLOT = VPL == 1 ? 16 : (VPL == 2 ? 8 : (VPL <= 4 ? 4 : 2));
  const bool first_of_slot = (lane & (LANES_PER_SLOT - 1)) == 0;
  const float inv_h = 1.f / (float)a.H;
  const int ysz = a.y.dtype == SAPO_DTYPE_F32 ? 4 : 2;
  int64_t ahead = row0;                                 // the next row to fetch, `src` its address
  auto fetch = [&](int stage) {
    if (ahead < a.T) Row::copy(dst + stage * STAGE_BYTES, src, cols, lane);
    copy_commit();
    ahead += step;
    src += step * ld;
  };
  #pragma unroll
  for (int s = 0; s < S - 1; ++s) fetch(s);
  // the weights in fp32, once per block: read from global memory for every row they miss L1 one time in five,
  // and the wait for them is longer than the rest of the row's work.  In 16-byte pieces in WarpRow's order.
  float* gs = reinterpret_cast<float*>(ring + S * STAGE_BYTES);
  float* bs = gs + a.H;
  for (int i = threadIdx.x * 8; i < a.H; i += NORM_THREADS * 8) {
    float2 u[4];
    const int f = (i >> 5) & 1, lo = i + 4 * f, hi = i + 4 - 4 * f;
    if (a.gamma != nullptr) {
      load_weight8(a.gamma, a.w_dtype, i, u);
      *reinterpret_cast<float4*>(gs + lo) = make_float4(u[0].x, u[0].y, u[1].x, u[1].y);
      *reinterpret_cast<float4*>(gs + hi) = make_float4(u[2].x, u[2].y, u[3].x, u[3].y);
    }
    if (a.beta != nullptr) {
      load_weight8(a.beta, a.w_dtype, i, u);
      *reinterpret_cast<float4*>(bs + lo) = make_float4(u[0].x, u[0].y, u[1].x, u[1].y);
      *reinterpret_cast<float4*>(bs + hi) = make_float4(u[2].x, u[2].y, u[3].x, u[3].y);
    }
  }
  __syncthreads();
  int stage = 0, turn = 0;
  for (int64_t row = row0; row < a.T; row += step) {
    copy_wait<S - 2>();
    __syncwarp();
    fetch(stage == 0 ? S - 1 : stage - 1);
    const uint8_t* at = mine + stage * STAGE_BYTES;
    stage = stage + 1 == S ? 0 : stage + 1;
    float2 x[VPL][4];
    #pragma unroll
    for (int v = 0; v < VPL; ++v) {
      Row::read(at, v, lane, x[v]);
      if (REPLAY) {
        const float2 s = both(256 * v < left ? a.q.scale[row * a.q.ld_scale + (col0 + 256 * v) / Q8_GROUP] : 0.f);
        #pragma unroll
        for (int j = 0; j < 4; ++j) x[v][j] = mul2(x[v][j], s);
      }
    }
    float mean = 0.f, rstd;
    if (REPLAY) {
      mean = a.kind == KIND_LAYER ? a.mean[row] : 0.f;
      rstd = a.rstd[row];
    } else {
      if (a.kind == KIND_LAYER) {
        float2 s = both(0.f), t = both(0.f);
        #pragma unroll
        for (int v = 0; v < VPL; ++v) { s = add2(s, add2(x[v][0], x[v][1])); t = add2(t, add2(x[v][2], x[v][3])); }
        s = add2(s, t);
        mean = group_sum<WARPS>(s.x + s.y, wpr, w, group, red, turn) * inv_h;
        turn ^= 1;
      }
      float2 s2 = both(0.f), t2 = both(0.f);
      #pragma unroll
      for (int v = 0; v < VPL; ++v) {
        const float2 minus = both(256 * v < left ? -mean : 0.f);
        #pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const float2 d = add2(x[v][j], minus), e = add2(x[v][j + 1], minus);
          s2 = fma2(d, d, s2);
          t2 = fma2(e, e, t2);
        }
      }
      s2 = add2(s2, t2);
      rstd = 1.f / sqrtf(group_sum<WARPS>(s2.x + s2.y, wpr, w, group, red, turn) * inv_h + a.eps);
      turn ^= 1;
      if (w == 0 && lane == 0) {
        if (a.mean != nullptr && a.kind == KIND_LAYER) a.mean[row] = mean;
        if (a.rstd != nullptr) a.rstd[row] = rstd;
      }
      if (a.q.p != nullptr) {
        int8_t* q_row = a.q.p + row * a.q.ld + col0;
        uint2 q[VPL];
        int slot; float scale; bool bad;
        quantise<VPL>(x, q, slot, scale, bad);
        #pragma unroll
        for (int v = 0; v < VPL; ++v)
          if (256 * v < left) *reinterpret_cast<uint2*>(q_row + 256 * v) = q[v];
        // one lane per group: half h of the warp has the groups at columns 256 v + 128 h
        const int scale_col = w * VPL * 256 + 256 * slot + 128 * (lane >> 4);
        if (first_of_slot && slot < VPL && scale_col < a.H) {
          a.q.scale[row * a.q.ld_scale + scale_col / Q8_GROUP] = scale;
          if (bad) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
        }
      }
    }
    const float2 minus = both(-mean), r2 = both(rstd);
    void* y_row = static_cast<char*>(a.y.p) + (row * a.y.ld + col0) * ysz;
    auto finish = [&](auto f) {
      #pragma unroll
      for (int v = 0; v < VPL; ++v) {
        if (256 * v >= left) break;
        #pragma unroll
        for (int j = 0; j < 4; ++j) x[v][j] = mul2(add2(x[v][j], minus), r2);
        float2 u[4];
        if (a.gamma != nullptr) {
          WarpRow<float, VPL>::read(reinterpret_cast<const uint8_t*>(gs + w * VPL * 256), v, lane, u);
          #pragma unroll
          for (int j = 0; j < 4; ++j) x[v][j] = mul2(x[v][j], u[j]);
        }
        if (a.beta != nullptr) {
          WarpRow<float, VPL>::read(reinterpret_cast<const uint8_t*>(bs + w * VPL * 256), v, lane, u);
          #pragma unroll
          for (int j = 0; j < 4; ++j) x[v][j] = add2(x[v][j], u[j]);
        }
        put8<decltype(f)::value>(y_row, 256 * v, x[v]);
      }
    };
    if (a.y.dtype == SAPO_DTYPE_F32) finish(std::true_type{}); else finish(std::false_type{});
  }
}

// Warps of a row and rows of a block in the backward: the sums of a thread's columns over all rows of its
// block are 16 registers a vector, so a thread owns few of them and a row is spread over more warps.
template <class TX, class TDY, int VPL, int MAX_THREADS> struct BwdRing {
  static constexpr int WARP_BYTES = WarpRow<TX, VPL>::BYTES + WarpRow<TDY, VPL>::BYTES + 64 + (sizeof(TX) == 1 ? VPL * 128 : 0);
  static constexpr int FULL = MAX_THREADS / 32 * WARP_BYTES;         // one row of the widest block
  static constexpr int STAGES = 4 * FULL <= SMEM_MAX ? 4 : (3 * FULL <= SMEM_MAX ? 3 : 2);
  static constexpr bool FITS = STAGES * FULL <= SMEM_MAX;            // else norm_bwd_kernel takes it
  // whether a row stays in registers between the sums and dx; a thread with many columns reads it again
  static constexpr bool HOLD = VPL <= 2;
};

template <class TX, class TDY, int VPL, int MAX_THREADS, int SLOTS>
__global__ void __launch_bounds__(MAX_THREADS, MAX_THREADS == 256 ? 2 : 1) norm_bwd_ring_kernel(NormBwdArgs a, int wpr) {
  constexpr bool FROM_Q8 = sizeof(TX) == 1;
  using Ring = BwdRing<TX, TDY, VPL, MAX_THREADS>;
  constexpr int S = Ring::STAGES;
  constexpr bool HOLD = Ring::HOLD;
  extern __shared__ __align__(16) uint8_t ring[];
  // [group][turn][slots]: wpr <= SLOTS, and only groups of two warps and more use them
  constexpr int RED = MAX_THREADS / 32 / 2 * 2 * SLOTS;
  __shared__ __align__(16) float2 red[RED];
  using RowX = WarpRow<TX, VPL>;
  using RowD = WarpRow<TDY, VPL>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, groups = warps / wpr;
  const int group = warp / wpr, w = warp - group * wpr;
  const int64_t step = (int64_t)gridDim.x * groups;
  const int64_t row0 = (int64_t)blockIdx.x * groups + group;
  const int warp_col = w * VPL * 256, cols = a.H - warp_col;
  const int col0 = warp_col + lane * 8, left = a.H - col0;          // vector v of the lane exists if 256 v < left
  uint8_t* mine = ring + warp * Ring::WARP_BYTES;
  const int stage_bytes = warps * Ring::WARP_BYTES;
  for (int i = threadIdx.x; i < RED; i += blockDim.x) red[i] = make_float2(0.f, 0.f);
  __syncthreads();
  if (cols < VPL * 256) clear_stages(mine, Ring::WARP_BYTES, S, stage_bytes, lane);
  const int64_t ldx = FROM_Q8 ? a.q.ld : a.x.ld;
  const TX* xp = (FROM_Q8 ? reinterpret_cast<const TX*>(a.q.p) : static_cast<const TX*>(a.x.p)) + row0 * ldx + warp_col + lane * RowX::LANE;
  const TDY* dyp = static_cast<const TDY*>(a.dy.p) + row0 * a.dy.ld + warp_col + lane * RowD::LANE;
  const float* sp = FROM_Q8 ? a.q.scale + row0 * a.q.ld_scale + col0 / Q8_GROUP : nullptr;
  constexpr int DY_AT = RowX::BYTES, ST_AT = DY_AT + RowD::BYTES, SC_AT = ST_AT + 64;
  const float inv_h = 1.f / (float)a.H;
  const bool layer = a.kind == KIND_LAYER;
  const uint32_t base = smem_addr(mine);
  const uint32_t dst_x = base + RowX::lane_dst(lane), dst_d = base + DY_AT + RowD::lane_dst(lane);
  // lane 0 copies rstd, lane 1 the mean
  const float* stat = lane == 0 ? a.rstd : a.mean;
  const bool copies_stat = lane == 0 || (lane == 1 && layer);
  int64_t ahead = row0;
  auto fetch = [&](int stage) {
    if (ahead < a.T) {
      const uint32_t off = stage * stage_bytes;
      RowX::copy(dst_x + off, xp, cols, lane);
      RowD::copy(dst_d + off, dyp, cols, lane);
      copy_async<4>(base + off + ST_AT + lane * 4, stat + ahead, copies_stat);
      if (FROM_Q8) {
        #pragma unroll
        for (int v = 0; v < VPL; ++v) copy_async<4>(base + off + SC_AT + (v * 32 + lane) * 4, sp + 2 * v, 256 * v < left);
      }
    }
    copy_commit();
    ahead += step;
    xp += step * ldx;
    dyp += step * a.dy.ld;
    if (FROM_Q8) sp += step * a.q.ld_scale;
  };
  #pragma unroll
  for (int s = 0; s < S - 1; ++s) fetch(s);
  float2 gam[HOLD ? VPL : 1][4], dg[VPL][4], db[VPL][4];
  auto weights = [&](int v, float2 (&g)[4]) {
    #pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = both(1.f);
    if (a.gamma != nullptr && 256 * v < left) load_weight8(a.gamma, a.w_dtype, col0 + 256 * v, g);
  };
  #pragma unroll
  for (int v = 0; v < VPL; ++v) {
    #pragma unroll
    for (int j = 0; j < 4; ++j) { dg[v][j] = both(0.f); db[v][j] = both(0.f); }
    if (HOLD) weights(v, gam[v]);
  }
  const int dxsz = a.dx.dtype == SAPO_DTYPE_F32 ? 4 : 2;
  int stage = 0, turn = 0;
  for (int64_t row = row0; row < a.T; row += step) {
    copy_wait<S - 2>();
    __syncwarp();
    fetch(stage == 0 ? S - 1 : stage - 1);
    const uint8_t* at = mine + stage * stage_bytes;
    stage = stage + 1 == S ? 0 : stage + 1;
    const float rstd = *reinterpret_cast<const float*>(at + ST_AT);
    const float mean = layer ? *reinterpret_cast<const float*>(at + ST_AT + 4) : 0.f;
    const float2 minus = both(-mean), r2 = both(rstd);
    float2 xh[HOLD ? VPL : 1][4], g[HOLD ? VPL : 1][4];
    // vector v of the row: xh and dy
    auto take = [&](int v, float2 (&x)[4], float2 (&d)[4]) {
      RowX::read(at, v, lane, x);
      RowD::read(at + DY_AT, v, lane, d);
      const float2 s = both(FROM_Q8 ? *reinterpret_cast<const float*>(at + SC_AT + (v * 32 + lane) * 4) : 1.f);
      #pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = mul2(add2(FROM_Q8 ? mul2(x[j], s) : x[j], minus), r2);
    };
    // (where a vector does not exist dy is zero: it adds nothing to the sums)
    float2 s1 = both(0.f), s2 = both(0.f);
    #pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int k = HOLD ? v : 0;
      take(v, xh[k], g[k]);
      if (!HOLD) weights(v, gam[0]);
      #pragma unroll
      for (int j = 0; j < 4; ++j) {
        dg[v][j] = fma2(g[k][j], xh[k][j], dg[v][j]);
        db[v][j] = add2(db[v][j], g[k][j]);
        g[k][j] = mul2(g[k][j], gam[k][j]);          // dy becomes g = dy gamma
        s1 = add2(s1, g[k][j]);
        s2 = fma2(g[k][j], xh[k][j], s2);
      }
    }
    const float2 sums = group_sum2<SLOTS>(s1.x + s1.y, s2.x + s2.y, wpr, w, group, red, turn);
    turn ^= 1;
    const float2 c1 = both(layer ? -sums.x * inv_h : 0.f), c2 = both(-sums.y * inv_h);
    void* dx_row = static_cast<char*>(a.dx.p) + (row * a.dx.ld + col0) * dxsz;
    auto finish = [&](auto f) {
      #pragma unroll
      for (int v = 0; v < VPL; ++v) {
        const int k = HOLD ? v : 0;
        if (!HOLD) {
          take(v, xh[0], g[0]);
          weights(v, gam[0]);
          #pragma unroll
          for (int j = 0; j < 4; ++j) g[0][j] = mul2(g[0][j], gam[0][j]);
        }
        #pragma unroll
        for (int j = 0; j < 4; ++j) g[k][j] = mul2(r2, fma2(xh[k][j], c2, add2(g[k][j], c1)));
        if (256 * v < left) put8<decltype(f)::value>(dx_row, 256 * v, g[k]);
      }
    };
    if (a.dx.dtype == SAPO_DTYPE_F32) finish(std::true_type{}); else finish(std::false_type{});
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (a.dgamma == nullptr && a.dbeta == nullptr) return;
  // the groups' sums one after the other, through the ring (no copy is in flight any more)
  copy_wait<0>();
  __syncthreads();
  float* acc = reinterpret_cast<float*>(ring);           // [2][H]
  for (int k = 0; k < groups; ++k) {
    if (k == group) {
      #pragma unroll
      for (int v = 0; v < VPL; ++v) {
        const int col = col0 + 256 * v;
        if (col >= a.H) continue;
        #pragma unroll
        for (int j = 0; j < 4; ++j) {
          float2* pg = reinterpret_cast<float2*>(acc + col + 2 * j);
          float2* pb = reinterpret_cast<float2*>(acc + a.H + col + 2 * j);
          if (k > 0) { dg[v][j] = add2(dg[v][j], *pg); db[v][j] = add2(db[v][j], *pb); }
          if (k + 1 < groups) { *pg = dg[v][j]; *pb = db[v][j]; continue; }
          if (gridDim.x > 1) {
            float* out = a.part + (int64_t)blockIdx.x * 2 * a.H + col + 2 * j;
            *reinterpret_cast<float2*>(out) = dg[v][j];
            *reinterpret_cast<float2*>(out + a.H) = db[v][j];
          } else {
            const int c = col + 2 * j;
            if (a.dgamma != nullptr) {
              a.dgamma[c] = a.accumulate ? a.dgamma[c] + dg[v][j].x : dg[v][j].x;
              a.dgamma[c + 1] = a.accumulate ? a.dgamma[c + 1] + dg[v][j].y : dg[v][j].y;
            }
            if (a.dbeta != nullptr) {
              a.dbeta[c] = a.accumulate ? a.dbeta[c] + db[v][j].x : db[v][j].x;
              a.dbeta[c + 1] = a.accumulate ? a.dbeta[c + 1] + db[v][j].y : db[v][j].y;
            }
          }
        }
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------- host side
struct RowPlan { int tpr, nv, threads; };
static RowPlan row_plan(int32_t H) {
  const int nvec = ceil_div(H, 8);
  int tpr = 1;
  while (tpr < nvec && tpr < 16) tpr <<= 1;            // a whole group of 16 vectors, or the whole row
  while (tpr * NV_MAX < nvec) tpr <<= 1;
  RowPlan p;
  p.tpr = tpr;
  p.nv = ceil_div(nvec, tpr);
  p.threads = tpr > NORM_THREADS ? tpr : NORM_THREADS;
  return p;
}
// Rows through shared memory: whole vectors of 8 columns, more of them than one 16-thread group has, rows
// (and weights) on 16-byte boundaries.
static bool ring_ok(int32_t H, bool vec, bool w_vec) { return vec && w_vec && H > Q8_GROUP && H % 8 == 0; }
struct RingPlan { int wpr, vpl, threads, rows_per_block; };
static RingPlan fwd_ring_plan(int32_t H) {
  const int nvec = ceil_div(H, 8);
  RingPlan p;
  p.wpr = 1;
  while (p.wpr * 256 < nvec) p.wpr <<= 1;
  p.vpl = ceil_div(nvec, p.wpr * 32);
  p.threads = NORM_THREADS;
  p.rows_per_block = NORM_THREADS / 32 / p.wpr;
  return p;
}
// Two blocks of 8 warps an SM, or one of 16: whichever leaves fewer warps of the 16 unused, 3 and 5 warps a row
// being those that do not divide 8 well (12 and 10 of 16 warps against 15).
static RingPlan bwd_ring_plan(int32_t H) {
  const int nvec = ceil_div(H, 8);
  RingPlan p;
  p.vpl = nvec <= 32 ? 1 : (H <= 8192 ? 2 : 4);
  p.wpr = ceil_div(nvec, p.vpl * 32);
  const int two = p.wpr > 8 ? 0 : 2 * (8 / p.wpr) * p.wpr, one = 16 / p.wpr * p.wpr;
  p.rows_per_block = two >= one ? 8 / p.wpr : 16 / p.wpr;
  p.threads = p.wpr * p.rows_per_block * 32;
  return p;
}
static int64_t bwd_blocks(int64_t T, int rows_per_block, int per_sm, int sms) {
  const int64_t want = ceil_div<int64_t>(T, rows_per_block);
  const int64_t most = (int64_t)sms * per_sm;
  return want < most ? want : most;
}

static bool type_ok(int32_t dtype) { return dtype == SAPO_DTYPE_BF16 || dtype == SAPO_DTYPE_F32; }
static int esize(int32_t dtype) { return dtype == SAPO_DTYPE_F32 ? 4 : 2; }
// whether rows of a matrix start on 16-byte boundaries
static bool vec_ok(const Mat& m) { return aligned16(m.p) && (m.ld * esize(m.dtype)) % 16 == 0; }
static bool vec_ok(const Q8Mat& q) { return (reinterpret_cast<uintptr_t>(q.p) & 7u) == 0 && q.ld % 8 == 0; }
static bool natural(const Mat& m) { return (reinterpret_cast<uintptr_t>(m.p) & (esize(m.dtype) - 1)) == 0; }

static int mat_check(const Mat& m, int64_t T, int32_t H) {
  if (!type_ok(m.dtype)) return SAPO_ERR_INVALID_ARG;
  if (T > 0 && (!m.p || !natural(m))) return SAPO_ERR_INVALID_ARG;
  return m.ld < H ? SAPO_ERR_INVALID_ARG : SAPO_OK;
}
static int ckpt_check(const sapo_ckpt8* c, int64_t T, int32_t H) {
  if (!c) return SAPO_ERR_INVALID_ARG;
  if (T > 0 && (!c->data || !c->scale || (reinterpret_cast<uintptr_t>(c->scale) & 3u))) return SAPO_ERR_INVALID_ARG;
  return c->ld < H || c->ld_scale < ceil_div(H, Q8_GROUP) ? SAPO_ERR_INVALID_ARG : SAPO_OK;
}
static int dims_check(int64_t T, int32_t H) {
  if (T < 0 || H < 1) return SAPO_ERR_INVALID_ARG;
  return H > NORM_MAX_H || T > 0x7fffff00LL ? SAPO_ERR_UNSUPPORTED_SHAPE : SAPO_OK;
}
static int cfg_check(const sapo_norm_cfg* c, const void* gamma, const void* beta) {
  if (!c || (c->kind != SAPO_NORM_LAYER && c->kind != SAPO_NORM_RMS) || !type_ok(c->w_dtype)) return SAPO_ERR_INVALID_ARG;
  const uintptr_t m = (uintptr_t)esize(c->w_dtype) - 1;
  return (reinterpret_cast<uintptr_t>(gamma) & m) || (reinterpret_cast<uintptr_t>(beta) & m) ? SAPO_ERR_INVALID_ARG : SAPO_OK;
}
static Q8Mat q8_of(const sapo_ckpt8* c) { return c ? Q8Mat{c->data, c->scale, c->ld, c->ld_scale} : Q8Mat{nullptr, nullptr, 0, 0}; }

// Blocks of a kernel that an SM holds, looked up once per kernel and device; opts in to the shared memory.
template <class Kernel>
static int resident_blocks(Kernel kernel, int threads, size_t smem, int* cache) {
  const int dev = current_device();
  if (dev < 0) return 0;
  if (cache[dev] == 0) {
    int n = 0;
    if (smem > 40 * 1024 &&
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_MAX) != cudaSuccess) return 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) != cudaSuccess || n < 1) return 0;
    cache[dev] = n;
  }
  return cache[dev];
}

constexpr int RING_TOO_WIDE = 1;         // rows and weights do not fit: norm_fwd_kernel takes them
template <class TX, int VPL>
static int launch_fwd_ring_vpl(const NormFwdArgs& a, const RingPlan& p, int sms, cudaStream_t st) {
  // (by the width of the row in 256 columns, which the weights' share of shared memory follows)
  static int cache[NORM_MAX_H / 256 + 1][MAX_DEVICES] = {{0}};
  auto kernel = norm_fwd_ring_kernel<TX, VPL>;
  const int steps = ceil_div(a.H, 256);
  const size_t smem = FwdRing<TX, VPL>::smem(steps * 256);
  if (smem > SMEM_MAX) return RING_TOO_WIDE;
  const int per_sm = resident_blocks(kernel, p.threads, smem, cache[steps]);
  if (per_sm == 0) return SAPO_ERR_CUDA;
  int64_t blocks = ceil_div<int64_t>(a.T, p.rows_per_block);
  if (blocks > (int64_t)sms * per_sm) blocks = (int64_t)sms * per_sm;
  KernelScope scope(SAPO_K_NORM_FWD, st);
  kernel<<<(int)blocks, p.threads, smem, st>>>(a, p.wpr);
  return check_launch();
}
template <class TX>
static int launch_fwd_ring(const NormFwdArgs& a, int sms, cudaStream_t st) {
  const RingPlan p = fwd_ring_plan(a.H);
  switch (p.vpl) {
    case 1: return launch_fwd_ring_vpl<TX, 1>(a, p, sms, st);
    case 2: return launch_fwd_ring_vpl<TX, 2>(a, p, sms, st);
    case 3: return launch_fwd_ring_vpl<TX, 3>(a, p, sms, st);
    case 4: return launch_fwd_ring_vpl<TX, 4>(a, p, sms, st);
    case 5: return launch_fwd_ring_vpl<TX, 5>(a, p, sms, st);
    case 6: return launch_fwd_ring_vpl<TX, 6>(a, p, sms, st);
    case 7: return launch_fwd_ring_vpl<TX, 7>(a, p, sms, st);
    default: return launch_fwd_ring_vpl<TX, 8>(a, p, sms, st);
  }
}

// launch == false: only how many blocks of the plan an SM holds (0: this form does not exist)
template <class TX, class TDY, int VPL, int MAX_THREADS, int SLOTS>
static int bwd_ring_vpl(const NormBwdArgs& a, const RingPlan& p, int blocks, bool launch, cudaStream_t st) {
  using Ring = BwdRing<TX, TDY, VPL, MAX_THREADS>;
  if constexpr (!Ring::FITS) {
    return launch ? SAPO_ERR_CUDA : 0;
  } else {
    static int cache[33][MAX_DEVICES] = {{0}};                       // by warps of the block
    auto kernel = norm_bwd_ring_kernel<TX, TDY, VPL, MAX_THREADS, SLOTS>;
    // the ring, or the columns' sums that take its place at the end
    size_t smem = (size_t)Ring::STAGES * (p.threads / 32) * Ring::WARP_BYTES;
    if (p.rows_per_block > 1 && smem < (size_t)2 * a.H * sizeof(float)) smem = (size_t)2 * a.H * sizeof(float);
    if (!launch) return resident_blocks(kernel, p.threads, smem, cache[p.threads / 32]);
    KernelScope scope(SAPO_K_NORM_BWD, st);
    kernel<<<blocks, p.threads, smem, st>>>(a, p.wpr);
    return check_launch();
  }
}
template <class TX, class TDY>
static int bwd_ring_dy(const NormBwdArgs& a, const RingPlan& p, int blocks, bool launch, cudaStream_t st) {
  if (p.vpl == 1) return bwd_ring_vpl<TX, TDY, 1, 256, 2>(a, p, blocks, launch, st);
  if (p.vpl == 2 && p.threads <= 256)
    return p.wpr <= 4 ? bwd_ring_vpl<TX, TDY, 2, 256, 4>(a, p, blocks, launch, st) : bwd_ring_vpl<TX, TDY, 2, 256, 8>(a, p, blocks, launch, st);
  if (p.vpl == 2)
    return p.wpr <= 8 ? bwd_ring_vpl<TX, TDY, 2, 512, 8>(a, p, blocks, launch, st) : bwd_ring_vpl<TX, TDY, 2, 512, 16>(a, p, blocks, launch, st);
  return bwd_ring_vpl<TX, TDY, 4, 512, 16>(a, p, blocks, launch, st);
}
static int bwd_ring(const NormBwdArgs& a, const RingPlan& p, int blocks, bool launch, cudaStream_t st) {
  const bool f = a.dy.dtype == SAPO_DTYPE_F32;
  if (a.q.p != nullptr) return f ? bwd_ring_dy<int8_t, float>(a, p, blocks, launch, st) : bwd_ring_dy<int8_t, __nv_bfloat16>(a, p, blocks, launch, st);
  if (a.x.dtype == SAPO_DTYPE_F32) return f ? bwd_ring_dy<float, float>(a, p, blocks, launch, st) : bwd_ring_dy<float, __nv_bfloat16>(a, p, blocks, launch, st);
  return f ? bwd_ring_dy<__nv_bfloat16, float>(a, p, blocks, launch, st) : bwd_ring_dy<__nv_bfloat16, __nv_bfloat16>(a, p, blocks, launch, st);
}

template <int NV, bool REPLAY>
static int launch_fwd_nv(const NormFwdArgs& a, bool vec, const RowPlan& p, int sms, cudaStream_t st) {
  auto kernel = vec ? norm_fwd_kernel<NV, true, REPLAY> : norm_fwd_kernel<NV, false, REPLAY>;
  static int cache[2][2][MAX_DEVICES] = {{{0}}};
  const int per_sm = resident_blocks(kernel, p.threads, 0, cache[vec][p.threads > NORM_THREADS]);
  if (per_sm == 0) return SAPO_ERR_CUDA;
  int64_t blocks = ceil_div<int64_t>(a.T, p.threads / p.tpr);
  if (blocks > (int64_t)sms * per_sm) blocks = (int64_t)sms * per_sm;
  KernelScope scope(SAPO_K_NORM_FWD, st);
  kernel<<<(int)blocks, p.threads, 0, st>>>(a);
  return check_launch();
}
template <bool REPLAY>
static int launch_fwd(NormFwdArgs a, cudaStream_t st) {
  if (a.T == 0) return SAPO_OK;
  const int sms = sm_count();
  if (sms <= 0) return SAPO_ERR_CUDA;
  const RowPlan p = row_plan(a.H);
  a.tpr = p.tpr;
  const bool vec = (REPLAY || vec_ok(a.x)) && vec_ok(a.y) && (a.q.p == nullptr || vec_ok(a.q));
  if (ring_ok(a.H, vec, a.w_vec != 0)) {
    const int rc = REPLAY ? launch_fwd_ring<int8_t>(a, sms, st)
                          : (a.x.dtype == SAPO_DTYPE_F32 ? launch_fwd_ring<float>(a, sms, st) : launch_fwd_ring<__nv_bfloat16>(a, sms, st));
    if (rc != RING_TOO_WIDE) return rc;
  }
  switch (p.nv) {
    case 1: return launch_fwd_nv<1, REPLAY>(a, vec, p, sms, st);
    case 2: return launch_fwd_nv<2, REPLAY>(a, vec, p, sms, st);
    case 3: return launch_fwd_nv<3, REPLAY>(a, vec, p, sms, st);
    default: return launch_fwd_nv<4, REPLAY>(a, vec, p, sms, st);
  }
}

template <int NV, bool Q8>
static int launch_bwd_nv(const NormBwdArgs& a, bool vec, const RowPlan& p, int blocks, cudaStream_t st) {
  auto kernel = vec ? norm_bwd_kernel<NV, true, Q8> : norm_bwd_kernel<NV, false, Q8>;
  const size_t smem = (size_t)2 * a.H * sizeof(float) * (p.threads > (p.tpr < 32 ? 32 : p.tpr) ? 1 : 0);
  KernelScope scope(SAPO_K_NORM_BWD, st);
  kernel<<<blocks, p.threads, smem, st>>>(a);
  return check_launch();
}
template <bool Q8>
static int launch_bwd(const NormBwdArgs& a, bool vec, const RowPlan& p, int blocks, cudaStream_t st) {
  switch (p.nv) {
    case 1: return launch_bwd_nv<1, Q8>(a, vec, p, blocks, st);
    case 2: return launch_bwd_nv<2, Q8>(a, vec, p, blocks, st);
    case 3: return launch_bwd_nv<3, Q8>(a, vec, p, blocks, st);
    default: return launch_bwd_nv<4, Q8>(a, vec, p, blocks, st);
  }
}

template <class TX, bool RESTORE>
static int launch_ckpt8_vec(const Ckpt8Args& a, int sms, cudaStream_t st) {
  static int cache[MAX_DEVICES] = {0};
  auto kernel = ckpt8_vec_kernel<TX, RESTORE>;
  const int per_sm = resident_blocks(kernel, 256, 0, cache);
  if (per_sm == 0) return SAPO_ERR_CUDA;
  const int32_t groups = ceil_div(a.H, Q8_GROUP);
  int64_t blocks = ceil_div<int64_t>(a.T * groups, 16 * CKPT_GROUPS);
  if (blocks > (int64_t)sms * per_sm) blocks = (int64_t)sms * per_sm;
  const int64_t halves = blocks * 16;
  KernelScope scope(SAPO_K_CKPT8, st);
  kernel<<<(int)blocks, 256, 0, st>>>(a, halves / groups, (int32_t)(halves % groups));
  return check_launch();
}

static int launch_ckpt8(const Mat& x, const Q8Mat& q, int64_t T, int32_t H, bool restore, int32_t* status, cudaStream_t st) {
  if (T == 0) return SAPO_OK;
  const int sms = sm_count();
  if (sms <= 0) return SAPO_ERR_CUDA;
  Ckpt8Args a{x, q, T, H, ceil_div(H, 8), 0, status};
  const bool vec = vec_ok(x) && vec_ok(q);
  if (vec && H % 8 == 0) {
    if (x.dtype == SAPO_DTYPE_F32) return restore ? launch_ckpt8_vec<float, true>(a, sms, st) : launch_ckpt8_vec<float, false>(a, sms, st);
    return restore ? launch_ckpt8_vec<__nv_bfloat16, true>(a, sms, st) : launch_ckpt8_vec<__nv_bfloat16, false>(a, sms, st);
  }
  while ((1 << a.vec_log2) < a.nvec) ++a.vec_log2;
  static int cache[4][MAX_DEVICES] = {{0}};
  auto kernel = restore ? (vec ? ckpt8_kernel<true, true> : ckpt8_kernel<false, true>)
                        : (vec ? ckpt8_kernel<true, false> : ckpt8_kernel<false, false>);
  const int per_sm = resident_blocks(kernel, 256, 0, cache[2 * restore + vec]);
  if (per_sm == 0) return SAPO_ERR_CUDA;
  int64_t blocks = ceil_div<int64_t>(T << a.vec_log2, 256);
  if (blocks > (int64_t)sms * per_sm) blocks = (int64_t)sms * per_sm;
  KernelScope scope(SAPO_K_CKPT8, st);
  kernel<<<(int)blocks, 256, 0, st>>>(a);
  return check_launch();
}

}  // namespace sapo

// =============================================================================== C ABI
extern "C" int sapo_norm_fwd(const void* x, int32_t x_dtype, int64_t T, int32_t H, int64_t ld_x,
                             const void* gamma, const void* beta, const sapo_norm_cfg* h_cfg,
                             void* y, int32_t y_dtype, int64_t ld_y, float* mean, float* rstd,
                             const sapo_ckpt8* h_ckpt, int32_t* status, void* stream) {
  using namespace sapo;
  int rc = cfg_check(h_cfg, gamma, beta);
  if (rc != SAPO_OK || !(h_cfg->eps >= 0.f)) return SAPO_ERR_INVALID_ARG;
  if ((rc = dims_check(T, H)) != SAPO_OK) return rc;
  const Mat mx{const_cast<void*>(x), ld_x, x_dtype}, my{y, ld_y, y_dtype};
  if ((rc = mat_check(mx, T, H)) != SAPO_OK || (rc = mat_check(my, T, H)) != SAPO_OK) return rc;
  if (h_ckpt && ((rc = ckpt_check(h_ckpt, T, H)) != SAPO_OK || !status)) return SAPO_ERR_INVALID_ARG;
  return launch_fwd<false>(NormFwdArgs{mx, my, q8_of(h_ckpt), gamma, beta, h_cfg->w_dtype,
                                       aligned16(gamma) && aligned16(beta), h_cfg->kind, h_cfg->eps,
                                       mean, rstd, T, H, 0, status}, static_cast<cudaStream_t>(stream));
}

extern "C" int sapo_norm_replay(const sapo_ckpt8* h_x, int64_t T, int32_t H, const void* gamma, const void* beta,
                                const sapo_norm_cfg* h_cfg, const float* mean, const float* rstd,
                                void* y, int32_t y_dtype, int64_t ld_y, void* stream) {
  using namespace sapo;
  int rc = cfg_check(h_cfg, gamma, beta);
  if (rc != SAPO_OK) return rc;
  if ((rc = dims_check(T, H)) != SAPO_OK) return rc;
  const Mat my{y, ld_y, y_dtype};
  if ((rc = ckpt_check(h_x, T, H)) != SAPO_OK || (rc = mat_check(my, T, H)) != SAPO_OK) return rc;
  if (T > 0 && (!rstd || (h_cfg->kind == SAPO_NORM_LAYER && !mean))) return SAPO_ERR_INVALID_ARG;
  return launch_fwd<true>(NormFwdArgs{Mat{nullptr, 0, SAPO_DTYPE_BF16}, my, q8_of(h_x), gamma, beta, h_cfg->w_dtype,
                                      aligned16(gamma) && aligned16(beta), h_cfg->kind, 0.f, const_cast<float*>(mean), const_cast<float*>(rstd), T, H, 0,
                                      nullptr}, static_cast<cudaStream_t>(stream));
}

extern "C" size_t sapo_norm_workspace_bytes(int64_t T, int32_t H) {
  using namespace sapo;
  if (dims_check(T, H) != SAPO_OK) return 0;
  int sms = sm_count();
  if (sms <= 0) sms = 148;
  // the larger of what the two forms of the kernel take, whatever the alignment of the rows will be
  const RowPlan p = row_plan(H);
  int64_t blocks = bwd_blocks(T > 0 ? T : 1, p.threads / p.tpr, 2, sms);
  const int64_t ring = bwd_blocks(T > 0 ? T : 1, bwd_ring_plan(H).rows_per_block, 2, sms);
  if (ring > blocks) blocks = ring;
  return round_up<size_t>((size_t)blocks * 2 * H * sizeof(float), 256);
}

extern "C" int sapo_norm_bwd(const void* dy, int32_t dy_dtype, int64_t ld_dy,
                             const void* x, int32_t x_dtype, int64_t ld_x, const sapo_ckpt8* h_ckpt,
                             int64_t T, int32_t H, const void* gamma, const sapo_norm_cfg* h_cfg,
                             const float* mean, const float* rstd, void* dx, int32_t dx_dtype, int64_t ld_dx,
                             float* dgamma, float* dbeta, int32_t accumulate,
                             void* workspace, size_t workspace_bytes, void* stream) {
  using namespace sapo;
  int rc = cfg_check(h_cfg, gamma, nullptr);
  if (rc != SAPO_OK) return rc;
  if ((rc = dims_check(T, H)) != SAPO_OK) return rc;
  const Mat mdy{const_cast<void*>(dy), ld_dy, dy_dtype}, mdx{dx, ld_dx, dx_dtype};
  Mat mx{const_cast<void*>(x), ld_x, x_dtype};
  if ((rc = mat_check(mdy, T, H)) != SAPO_OK || (rc = mat_check(mdx, T, H)) != SAPO_OK) return rc;
  if ((x != nullptr) == (h_ckpt != nullptr) && (T > 0 || x != nullptr)) return SAPO_ERR_INVALID_ARG;
  if (h_ckpt) { if ((rc = ckpt_check(h_ckpt, T, H)) != SAPO_OK) return rc; mx = Mat{nullptr, 0, SAPO_DTYPE_BF16}; }
  else if ((rc = mat_check(mx, T, H)) != SAPO_OK) return rc;
  if (T > 0 && (!rstd || (h_cfg->kind == SAPO_NORM_LAYER && !mean))) return SAPO_ERR_INVALID_ARG;
  const bool reduce = dgamma != nullptr || dbeta != nullptr;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (T == 0) {
    if (!accumulate && ((dgamma && cudaMemsetAsync(dgamma, 0, (size_t)H * 4, st) != cudaSuccess) ||
                        (dbeta && cudaMemsetAsync(dbeta, 0, (size_t)H * 4, st) != cudaSuccess)))
      return SAPO_ERR_CUDA;
    return SAPO_OK;
  }
  const int sms = sm_count();
  if (sms <= 0) return SAPO_ERR_CUDA;
  const bool vec = vec_ok(mdy) && vec_ok(mdx) && (h_ckpt ? vec_ok(q8_of(h_ckpt)) : vec_ok(mx));
  NormBwdArgs a{mdy, mx, mdx, q8_of(h_ckpt), gamma, h_cfg->w_dtype, aligned16(gamma), h_cfg->kind, mean, rstd, T, H, 0,
                static_cast<float*>(workspace), dgamma, dbeta, accumulate};
  const RowPlan p = row_plan(H);
  const RingPlan rp = bwd_ring_plan(H);
  const int resident = ring_ok(H, vec, aligned16(gamma)) ? bwd_ring(a, rp, 0, false, st) : 0;
  const bool ring = resident > 0;
  const int blocks = (int)bwd_blocks(T, ring ? rp.rows_per_block : p.threads / p.tpr, ring && resident < 2 ? resident : 2, sms);
  a.tpr = p.tpr;
  if (reduce && blocks > 1) {
    if (!workspace || !aligned16(workspace)) return SAPO_ERR_INVALID_ARG;
    if (workspace_bytes < (size_t)blocks * 2 * H * sizeof(float)) return SAPO_ERR_WORKSPACE_TOO_SMALL;
  }
  if (ring) rc = bwd_ring(a, rp, blocks, true, st);
  else rc = h_ckpt ? launch_bwd<true>(a, vec, p, blocks, st) : launch_bwd<false>(a, vec, p, blocks, st);
  if (rc != SAPO_OK || !reduce || blocks == 1) return rc;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(ceil_div(H, 32), 2);
  cfg.blockDim = dim3(1024);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  KernelScope scope(SAPO_K_NORM_REDUCE, st);
  return cudaLaunchKernelEx(&cfg, norm_reduce_kernel, (const float*)a.part, blocks, H, dgamma, dbeta, (int)accumulate) == cudaSuccess
             ? SAPO_OK : SAPO_ERR_CUDA;
}

extern "C" int sapo_ckpt8_store(const void* x, int32_t x_dtype, int64_t T, int32_t H, int64_t ld_x,
                                const sapo_ckpt8* h_out, int32_t* status, void* stream) {
  using namespace sapo;
  int rc = dims_check(T, H);
  if (rc != SAPO_OK) return rc;
  const Mat mx{const_cast<void*>(x), ld_x, x_dtype};
  if ((rc = mat_check(mx, T, H)) != SAPO_OK || (rc = ckpt_check(h_out, T, H)) != SAPO_OK) return rc;
  if (!status) return SAPO_ERR_INVALID_ARG;
  return launch_ckpt8(mx, q8_of(h_out), T, H, false, status, static_cast<cudaStream_t>(stream));
}

extern "C" int sapo_ckpt8_restore(const sapo_ckpt8* h_in, int64_t T, int32_t H, void* x, int32_t x_dtype,
                                  int64_t ld_x, void* stream) {
  using namespace sapo;
  int rc = dims_check(T, H);
  if (rc != SAPO_OK) return rc;
  const Mat mx{x, ld_x, x_dtype};
  if ((rc = mat_check(mx, T, H)) != SAPO_OK || (rc = ckpt_check(h_in, T, H)) != SAPO_OK) return rc;
  return launch_ckpt8(mx, q8_of(h_in), T, H, true, nullptr, static_cast<cudaStream_t>(stream));
}
