// Norm forward, replay and backward for rows that can be copied 16 bytes at a time.
#pragma once

#include "norm_common.cuh"

namespace sapo {

// ---------------------------------------------------------------------------- rows through shared memory
// The kernels for rows of more than 128 columns, a multiple of 8, that start on 16-byte boundaries.
// A row belongs to the `wpr` warps of a group; warp w of them owns VPL * 256 consecutive columns, lane l
// of it the vectors of 8 columns (w VPL + v) 32 + l, v < VPL.  Each warp streams its part of the group's
// next STAGES - 1 rows into shared memory with asynchronous copies while it works on the current one, so
// the bytes in flight do not depend on registers or on how long a row's sums take.  Only lanes of the
// same warp read what a lane copied: the wait for a row is one __syncwarp.
// What then bounds a row kernel is instruction issue (at the copy bandwidth an SM has to finish 4 to 6
// columns per clock), so the arithmetic is done in pairs and every vector is whole.
// Measured on long runs of rows, beside a copy (forward) or an addition of two arrays (backward) of the same bytes; 30 calls
// in a row, then 1.5 s of them (boxes and their state move either by up to 10 %):
//   forward    146382 x 1536 bf16  150 and 157 us (copy 143), 500000 x 512  165 and 160 us (copy 160)
//   backward   143347 x 3584 bf16  476 and 514 us (addition 437), 146382 x 1536  237 and 213 us (194), where the fewer
//              warps of a row leave the waits for its sums less covered (45 % of issue slots used, 75 % of the DRAM rate)
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
// (predicated, not branched around: a lane whose columns do not exist copies nothing)
template <int BYTES, bool ALWAYS>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool exists) {
  if constexpr (ALWAYS && BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else if constexpr (ALWAYS)
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
  else if constexpr (BYTES == 16)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}"
                 ::"r"(dst), "l"(src), "r"((uint32_t)exists) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p cp.async.ca.shared.global [%0], [%1], %3;\n\t}"
                 ::"r"(dst), "l"(src), "r"((uint32_t)exists), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

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
  template <bool FULL>
  __device__ static __forceinline__ void copy(uint32_t dst, const TX* src, int cols, int lane) {
    // fp32: neighbouring lanes copy neighbouring 16 bytes; a lane then reads two of them in a row, so pieces
    // are stored with the lowest bit of their index flipped in every other eight: no bank conflicts
    constexpr int B = LANE * (int)sizeof(TX);
    #pragma unroll
    for (int v = 0; v < PER_V * VPL; ++v)
      copy_async<B, FULL>(dst + v * 32 * B, src + v * 32 * LANE, v * 32 * LANE + lane * LANE < cols);
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

template <class TX, int VPL> struct FwdRing {
  static constexpr int STAGE_BYTES = NORM_THREADS / 32 * WarpRow<TX, VPL>::BYTES;
  static constexpr int STAGES = sizeof(TX) == 1 ? 4 : (VPL <= 4 ? 3 : 2);
  static constexpr int smem(int H) { return STAGES * STAGE_BYTES + 2 * H * (int)sizeof(float); }   // and the weights
};

// Zeros where the warp's columns do not exist: nothing is ever copied there, and zeros add nothing to sums.
__device__ __forceinline__ void clear_stages(uint8_t* mine, int bytes, int stages, int stage_bytes, int lane) {
  for (int s = 0; s < stages; ++s)
    for (int i = lane * 16; i < bytes; i += 512) *reinterpret_cast<uint4*>(mine + s * stage_bytes + i) = make_uint4(0u, 0u, 0u, 0u);
  __syncwarp();
}
// y = (x - mean) rstd gamma + beta; the row stays in registers between its mean, its sum of squares about the mean
// and y, so it is read once and nothing is subtracted from a sum of squares.  With a checkpoint the groups of 128
// columns are quantised on the way (146382 x 1536: 150 us for 0.90 GB without, 206 us for 1.13 GB with).
// The weights are kept in shared memory in fp32, in the order in which a warp reads them without bank conflicts.
// TX int8_t: replay from a checkpoint (a.q), statistics given.
template <class TX, int VPL, bool FULL>
__global__ void __launch_bounds__(NORM_THREADS, 2) norm_fwd_ring_kernel(NormFwdArgs a, int wpr) {
  wait_for_previous();
  let_next_start();
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
  if (!FULL && cols < VPL * 256) clear_stages(mine, Row::BYTES, S, STAGE_BYTES, lane);
  const uint32_t dst = smem_addr(mine) + Row::lane_dst(lane);
  const float inv_h = 1.f / (float)a.H;
  const int ysz = a.y.dtype == SAPO_DTYPE_F32 ? 4 : 2;
  char* y_row = static_cast<char*>(a.y.p) + (row0 * a.y.ld + col0) * ysz;
  const int64_t y_step = step * a.y.ld * ysz;
  // rows of this group, and how many of them are still to fetch (`src`: the next one)
  const int n_rows = row0 < a.T ? (int)((a.T - row0 + step - 1) / step) : 0;
  int to_fetch = n_rows;
  auto fetch = [&](int stage) {
    if (to_fetch > 0 && SAPO_IN_BOUNDS(row0 + (n_rows - to_fetch) * step < a.T && stage >= 0 && stage < S))
      Row::template copy<FULL>(dst + stage * STAGE_BYTES, src, cols, lane);
    copy_commit();
    --to_fetch;
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
  int64_t row = row0;
  for (int i = 0; i < n_rows; ++i, row += step) {
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
        const float2 s = both(FULL || 256 * v < left ? a.q.scale[row * a.q.ld_scale + (col0 + 256 * v) / Q8_GROUP] : 0.f);
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
        const float2 minus = both(FULL || 256 * v < left ? -mean : 0.f);
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
        uint2 bytes[VPL][4];
        float scale; bool bad;
        quantise<VPL, 16, 4>(x, bytes, scale, bad);
        #pragma unroll
        for (int v = 0; v < VPL; ++v)
          if (FULL || 256 * v < left) *reinterpret_cast<uint2*>(q_row + 256 * v) = pack_bytes(bytes[v]);
        // one lane per group: half h of the warp has the groups at columns 256 v + 128 h
        using Half = Slots<PowerOfTwo<VPL>::value, 16>;
        const int scale_col = w * VPL * 256 + 256 * Half::slot() + 128 * (lane >> 4);
        if (Half::first() && Half::slot() < VPL && scale_col < a.H) {
          a.q.scale[row * a.q.ld_scale + scale_col / Q8_GROUP] = scale;
          if (bad) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
        }
      }
    }
    const float2 minus = both(-mean), r2 = both(rstd);
    auto finish = [&](auto f) {
      #pragma unroll
      for (int v = 0; v < VPL; ++v) {
        if (!FULL && 256 * v >= left) break;
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
    y_row += y_step;
  }
}

// dx = rstd (g - mean_c(g) - xh mean_c(g xh)) with g = dy gamma: both sums of a row cross its warps together.  dgamma
// and dbeta stay in registers over all rows of a block and leave it once, as the block's part.
// Warps of a row and rows of a block: the sums of a thread's columns are 16 registers a vector, so a thread
// owns few of them and a row is spread over more warps (one vector a thread and half as many registers: 1536 columns
// 240 -> 215 us, but 16527 x 896 23 -> 27 us, as there are more parts to add).
template <class TX, class TDY, int VPL, int MAX_THREADS> struct BwdRing {
  static constexpr int WARP_BYTES = WarpRow<TX, VPL>::BYTES + WarpRow<TDY, VPL>::BYTES + 64 + (sizeof(TX) == 1 ? VPL * 128 : 0);
  static constexpr int FULL = MAX_THREADS / 32 * WARP_BYTES;         // one row of the widest block
  static constexpr int STAGES = 4 * FULL <= SMEM_MAX ? 4 : (3 * FULL <= SMEM_MAX ? 3 : 2);
  static constexpr bool FITS = STAGES * FULL <= SMEM_MAX;            // else norm_bwd_any_kernel takes it
  // whether a row stays in registers between the sums and dx; a thread with many columns reads it again
  static constexpr bool HOLD = VPL <= 2;
};

template <class TX, class TDY, int VPL, int MAX_THREADS, int SLOTS, bool FULL>
__global__ void __launch_bounds__(MAX_THREADS, MAX_THREADS == 256 ? 2 : 1) norm_bwd_ring_kernel(NormBwdArgs a, int wpr) {
  wait_for_previous();
  let_next_start();
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
  if (!FULL && cols < VPL * 256) clear_stages(mine, Ring::WARP_BYTES, S, stage_bytes, lane);
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
  const int n_rows = row0 < a.T ? (int)((a.T - row0 + step - 1) / step) : 0;
  int to_fetch = n_rows;
  stat += row0;
  auto fetch = [&](int stage) {
    if (to_fetch > 0 && SAPO_IN_BOUNDS(row0 + (n_rows - to_fetch) * step < a.T && stage >= 0 && stage < S)) {
      const uint32_t off = stage * stage_bytes;
      RowX::template copy<FULL>(dst_x + off, xp, cols, lane);
      RowD::template copy<FULL>(dst_d + off, dyp, cols, lane);
      copy_async<4, false>(base + off + ST_AT + lane * 4, stat, copies_stat);
      if (FROM_Q8) {
        #pragma unroll
        for (int v = 0; v < VPL; ++v) copy_async<4, FULL>(base + off + SC_AT + (v * 32 + lane) * 4, sp + 2 * v, 256 * v < left);
      }
    }
    copy_commit();
    --to_fetch;
    stat += step;
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
  char* dx_row = static_cast<char*>(a.dx.p) + (row0 * a.dx.ld + col0) * dxsz;
  const int64_t dx_step = step * a.dx.ld * dxsz;
  int stage = 0, turn = 0;
  for (int i = 0; i < n_rows; ++i) {
    copy_wait<S - 2>();
    __syncwarp();
    fetch(stage == 0 ? S - 1 : stage - 1);
    const uint8_t* at = mine + stage * stage_bytes;
    stage = stage + 1 == S ? 0 : stage + 1;
    const float rstd = *reinterpret_cast<const float*>(at + ST_AT);
    const float mean = layer ? *reinterpret_cast<const float*>(at + ST_AT + 4) : 0.f;
    const float2 minus = both(-mean), r2 = both(rstd), shift = both(-mean * rstd);
    float2 xh[HOLD ? VPL : 1][4], g[HOLD ? VPL : 1][4];
    // vector v of the row: xh and dy
    auto take = [&](int v, float2 (&x)[4], float2 (&d)[4]) {
      RowX::read(at, v, lane, x);
      RowD::read(at + DY_AT, v, lane, d);
      if (FROM_Q8) {       // value and (value - mean) rstd in one rounding: the value itself is off by much more
        const float2 s = both(*reinterpret_cast<const float*>(at + SC_AT + (v * 32 + lane) * 4) * rstd);
        #pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = fma2(x[j], s, shift);
      } else {
        #pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = mul2(add2(x[j], minus), r2);
      }
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
    const float2 c1 = both(layer ? -sums.x * inv_h * rstd : 0.f), c2 = both(-sums.y * inv_h * rstd);
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
        for (int j = 0; j < 4; ++j) g[k][j] = fma2(xh[k][j], c2, fma2(g[k][j], r2, c1));
        if (FULL || 256 * v < left) put8<decltype(f)::value>(dx_row, 256 * v, g[k]);
      }
    };
    if (a.dx.dtype == SAPO_DTYPE_F32) finish(std::true_type{}); else finish(std::false_type{});
    dx_row += dx_step;
  }
  if (a.dgamma == nullptr && a.dbeta == nullptr) return;
  // the groups' sums take the ring's place (no copy is in flight any more)
  copy_wait<0>();
  __syncthreads();
  static_assert(S * Ring::WARP_BYTES >= 2 * VPL * 256 * (int)sizeof(float), "a warp's sums in its share of the ring");
  float* acc = reinterpret_cast<float*>(ring);
  const int pitch = wpr * VPL * 256;
  float4* to = reinterpret_cast<float4*>(acc + group * 2 * pitch + col0);
  #pragma unroll
  for (int v = 0; v < VPL; ++v) {
    #pragma unroll
    for (int h = 0; h < 2; ++h) {
      to[64 * v + h] = make_float4(dg[v][2 * h].x, dg[v][2 * h].y, dg[v][2 * h + 1].x, dg[v][2 * h + 1].y);
      to[pitch / 4 + 64 * v + h] = make_float4(db[v][2 * h].x, db[v][2 * h].y, db[v][2 * h + 1].x, db[v][2 * h + 1].y);
    }
  }
  __syncthreads();
  finish_columns<4>(a, acc, groups, pitch);
}

// dgamma and dbeta (blockIdx.y) as the sums of the blocks' parts, 32 columns a block: 8 lanes hold 4 columns each of every
// 64th part, all of a thread's loads before the first use.  What it takes is their latency and a launch's: 2 to 3 us
// behind the main kernel (16527 x 896, 296 parts; with a load per part and turn it was 5).
constexpr int REDUCE_WARPS = 16;
__global__ void __launch_bounds__(REDUCE_WARPS * 32)
norm_reduce_kernel(const float* part, int n_parts, int32_t H, float* dgamma, float* dbeta, int accumulate) {
  constexpr int STEP = REDUCE_WARPS * 4, N = 5;          // 5 * 64 parts: two blocks' of each of up to 160 SMs at a time
  __shared__ __align__(16) float sums[REDUCE_WARPS][32];
  wait_for_previous();
  let_next_start();
  const bool beta = dgamma == nullptr || blockIdx.y != 0;
  float* out = beta ? dbeta : dgamma;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, pitch = part_pitch(H);
  const int col = blockIdx.x * 32 + (lane & 7) * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (col < H) {
    const float* src = part + (beta ? pitch : 0) + col;
    for (int b = w * 4 + (lane >> 3); b < n_parts; b += N * STEP) {
      float4 x[N];
      #pragma unroll
      for (int j = 0; j < N; ++j)
        x[j] = b + j * STEP < n_parts ? __ldcg(reinterpret_cast<const float4*>(src + (int64_t)(b + j * STEP) * 2 * pitch)) : make_float4(0.f, 0.f, 0.f, 0.f);
      #pragma unroll
      for (int j = 0; j < N; ++j) { s.x += x[j].x; s.y += x[j].y; s.z += x[j].z; s.w += x[j].w; }
    }
  }
  #pragma unroll
  for (int d = 16; d >= 8; d >>= 1) {
    s.x += __shfl_xor_sync(0xffffffffu, s.x, d); s.y += __shfl_xor_sync(0xffffffffu, s.y, d);
    s.z += __shfl_xor_sync(0xffffffffu, s.z, d); s.w += __shfl_xor_sync(0xffffffffu, s.w, d);
  }
  if (lane < 8) *reinterpret_cast<float4*>(&sums[w][lane * 4]) = s;
  __syncthreads();
  if (w != 0 || blockIdx.x * 32 + lane >= H) return;
  float t = 0.f;
  #pragma unroll
  for (int k = 0; k < REDUCE_WARPS; ++k) t += sums[k][lane];
  float* to = out + blockIdx.x * 32 + lane;
  *to = accumulate ? *to + t : t;
}

// Checkpoints alone, rows on 16-byte boundaries in whole vectors.  L = 32: a warp takes N * 256 neighbouring columns of a
// row (`segments` of them a row), each lane N vectors 256 columns apart, so that one address serves all of a step.
// L < 32: rows of up to 8 L columns, 32 / L rows a warp at a time and N of those a lane.
// Bound by DRAM, from L2 by the waits for a group's largest value: on long bf16 matrices 90 % (store) and 85 % (restore) of
// the copy bandwidth; 16527 x 896, which L2 holds, stored and restored in 15.6 us for 90 MB.
template <class TX, int L, int N, bool RESTORE>
__global__ void __launch_bounds__(256) ckpt8_rows_kernel(Ckpt8Args a, int32_t segments, int64_t step_rows, int32_t step_segments) {
  wait_for_previous();
  let_next_start();
  constexpr int ROWS = L == 32 ? 1 : N * (32 / L), G = L < 16 ? L : 16;       // rows of a warp's step, lanes of a group
  using S = Slots<PowerOfTwo<N>::value, G>;
  const int lane = threadIdx.x & 31;
  const int64_t id = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  int64_t unit = id / segments;                                               // rows unit * ROWS on
  int32_t seg = (int32_t)(id - unit * segments);
  while (unit * ROWS < a.T) {
    const int64_t row = unit * ROWS + (lane / L) * (L == 32 ? 0 : N);
    const int col = seg * N * 256 * (L == 32) + (lane & (L - 1)) * 8;
    TX* x = static_cast<TX*>(a.x.p) + row * a.x.ld + col;
    int8_t* q = a.q.p + row * a.q.ld + col;
    const int64_t x_next = L == 32 ? 256 : a.x.ld, q_next = L == 32 ? 256 : a.q.ld;
    // vector k of the lane: 256 k columns on (L = 32), or k rows on
    auto exists = [&](int k) { return L == 32 ? col + 256 * k < a.H : row + k < a.T && col < a.H; };
    if (!SAPO_IN_BOUNDS(unit >= 0 && seg >= 0 && seg < segments)) break;
    float2 v[N][4];
    if constexpr (RESTORE) {
      float s[N];
      #pragma unroll
      for (int k = 0; k < N; ++k) {
        s[k] = 0.f;
        #pragma unroll
        for (int j = 0; j < 4; ++j) v[k][j] = both(0.f);
        if (exists(k)) {
          load8(q + k * q_next, v[k]);
          s[k] = a.q.scale[(row + (L == 32 ? 0 : k)) * a.q.ld_scale + (col + (L == 32 ? 256 * k : 0)) / Q8_GROUP];
        }
      }
      #pragma unroll
      for (int k = 0; k < N; ++k) {
        #pragma unroll
        for (int j = 0; j < 4; ++j) v[k][j] = mul2(v[k][j], both(s[k]));
        if (exists(k)) put8<sizeof(TX) == 4>(x + k * x_next, 0, v[k]);
      }
    } else {
      #pragma unroll
      for (int k = 0; k < N; ++k) {
        #pragma unroll
        for (int j = 0; j < 4; ++j) v[k][j] = both(0.f);
        if (exists(k)) load8(x + k * x_next, v[k]);
      }
      uint2 bytes[N][4];
      float scale; bool bad;
      quantise<N, G, 4>(v, bytes, scale, bad);
      #pragma unroll
      for (int k = 0; k < N; ++k)
        if (exists(k)) *reinterpret_cast<uint2*>(q + k * q_next) = pack_bytes(bytes[k]);
      // one lane per group: of vector slot() of the lane's half warp, or of its row
      const int k = S::slot();
      const int group_col = L == 32 ? seg * N * 256 + 256 * k + 128 * (lane >> 4) : 0;
      const int64_t group_row = L == 32 ? row : row + k;
      if (S::first() && k < N && group_col < a.H && group_row < a.T) {
        a.q.scale[group_row * a.q.ld_scale + group_col / Q8_GROUP] = scale;
        if (bad) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
      }
    }
    unit += step_rows; seg += step_segments;
    if (seg >= segments) { seg -= segments; ++unit; }
  }
}

}  // namespace sapo
