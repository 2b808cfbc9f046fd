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

#include "common.cuh"

namespace sapo {

constexpr int Q8_GROUP = 128;            // columns that share one checkpoint scale
constexpr int NORM_MAX_H = 16384;
constexpr int NORM_THREADS = 256;
constexpr int NORM_MAX_THREADS = 512;    // one row of NORM_MAX_H columns
constexpr int NV_MAX = 4;
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
// per-column weights: fp32 or bf16, no alignment asked for
__device__ __forceinline__ void load_weight8(const void* w, int32_t dtype, int col, int n, float (&v)[8]) {
  if (dtype == SAPO_DTYPE_F32) load8<false>(static_cast<const float*>(w) + col, n, v);
  else load8<false>(static_cast<const __nv_bfloat16*>(w) + col, n, v);
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
  Mat x, y; Q8Mat q; const void* gamma; const void* beta; int32_t w_dtype, kind; float eps;
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
        if (a.gamma != nullptr) load_weight8(a.gamma, a.w_dtype, col, n, g);
        if (a.beta != nullptr) load_weight8(a.beta, a.w_dtype, col, n, b);
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
  Mat dy, x, dx; Q8Mat q; const void* gamma; int32_t w_dtype, kind; const float* mean; const float* rstd;
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
    if (a.gamma != nullptr) load_weight8(a.gamma, a.w_dtype, col, n, gam[i]);
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
  if (out == nullptr) return;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + lane;
  float s = 0.f;
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
static int64_t bwd_blocks(int64_t T, const RowPlan& p, int sms) {
  const int64_t want = ceil_div<int64_t>(T, p.threads / p.tpr);
  const int64_t most = (int64_t)sms * 2;
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

template <int NV, bool REPLAY>
static int launch_fwd_nv(const NormFwdArgs& a, bool vec, const RowPlan& p, int sms, cudaStream_t st) {
  auto kernel = vec ? norm_fwd_kernel<NV, true, REPLAY> : norm_fwd_kernel<NV, false, REPLAY>;
  int64_t blocks = ceil_div<int64_t>(a.T, p.threads / p.tpr);
  const int64_t most = (int64_t)sms * resident_blocks_per_sm(kernel, p.threads);
  if (blocks > most) blocks = most;
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

static int launch_ckpt8(const Mat& x, const Q8Mat& q, int64_t T, int32_t H, bool restore, int32_t* status, cudaStream_t st) {
  if (T == 0) return SAPO_OK;
  const int sms = sm_count();
  if (sms <= 0) return SAPO_ERR_CUDA;
  Ckpt8Args a{x, q, T, H, ceil_div(H, 8), 0, status};
  while ((1 << a.vec_log2) < a.nvec) ++a.vec_log2;
  const bool vec = vec_ok(x) && vec_ok(q);
  auto kernel = restore ? (vec ? ckpt8_kernel<true, true> : ckpt8_kernel<false, true>)
                        : (vec ? ckpt8_kernel<true, false> : ckpt8_kernel<false, false>);
  int64_t blocks = ceil_div<int64_t>(T << a.vec_log2, 256);
  const int64_t most = (int64_t)sms * resident_blocks_per_sm(kernel, 256);
  if (blocks > most) blocks = most;
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
  return launch_fwd<false>(NormFwdArgs{mx, my, q8_of(h_ckpt), gamma, beta, h_cfg->w_dtype, h_cfg->kind, h_cfg->eps,
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
                                      h_cfg->kind, 0.f, const_cast<float*>(mean), const_cast<float*>(rstd), T, H, 0,
                                      nullptr}, static_cast<cudaStream_t>(stream));
}

extern "C" size_t sapo_norm_workspace_bytes(int64_t T, int32_t H) {
  using namespace sapo;
  if (dims_check(T, H) != SAPO_OK) return 0;
  int sms = sm_count();
  if (sms <= 0) sms = 148;
  const int64_t blocks = bwd_blocks(T > 0 ? T : 1, row_plan(H), sms);
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
  const RowPlan p = row_plan(H);
  const int blocks = (int)bwd_blocks(T, p, sms);
  if (reduce && blocks > 1) {
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 3u)) return SAPO_ERR_INVALID_ARG;
    if (workspace_bytes < (size_t)blocks * 2 * H * sizeof(float)) return SAPO_ERR_WORKSPACE_TOO_SMALL;
  }
  NormBwdArgs a{mdy, mx, mdx, q8_of(h_ckpt), gamma, h_cfg->w_dtype, h_cfg->kind, mean, rstd, T, H, p.tpr,
                static_cast<float*>(workspace), dgamma, dbeta, accumulate};
  const bool vec = vec_ok(mdy) && vec_ok(mdx) && (h_ckpt ? vec_ok(a.q) : vec_ok(mx));
  rc = h_ckpt ? launch_bwd<true>(a, vec, p, blocks, st) : launch_bwd<false>(a, vec, p, blocks, st);
  if (rc != SAPO_OK || !reduce || blocks == 1) return rc;
  KernelScope scope(SAPO_K_NORM_REDUCE, st);
  norm_reduce_kernel<<<dim3(ceil_div(H, 32), 2), 1024, 0, st>>>(a.part, blocks, H, dgamma, dbeta, accumulate);
  return check_launch();
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
