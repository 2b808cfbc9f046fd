// Norm forward, replay and backward and the checkpoints for rows of any width, pitch and alignment, and for rows of up
// to 128 columns (256 in the forward), which are too short for the streaming kernels.  Nothing is staged: a row is loaded into registers at
// once, and short rows several at a time; the other warps of the SM cover the wait.  Three ways to own columns:
//   Cols<1, E>   single columns, 32 apart: a warp's accesses are contiguous whatever the row's first byte is
//   Cols<2, E>   pairs of neighbouring columns, where rows start on pair boundaries and H is even
//   Vector<L>    8 neighbouring columns, L lanes a row and 32 / L rows a warp, for rows of up to 8 L columns on 16-byte
//                boundaries
// Measured at 120 million columns, beside the copy bandwidth: rows of 64 bf16 forward 105 us (70 %), backward 144 us (76 %);
// rows of 1001 fp32 94 and 89 %, bounded by DRAM; rows of 1001 bf16 224 and 241 us (33 and 46 %), bounded by the load and
// store unit: a 2-byte access moves 64 bytes a warp, a sixteenth of what whole vectors do.
#pragma once

#include "norm_common.cuh"

namespace sapo {

// E columns of a lane in E / 2 pairs: pair p is columns 64 p and 64 p + 1 (W = 2) or 64 p and 64 p + 32 (W = 1) behind
// the lane's first one.  left: how many columns the row has from the lane's first one on.
template <int W, int E> struct Cols {
  static constexpr int LANES = 32, PAIRS = E / 2;       // lanes of a row (in one warp), pairs of a lane
  static constexpr int GROUP_LANES = 32;                // lanes of a group of 128 columns
  static constexpr int SECOND = W == 2 ? 1 : 32;
  // a group of 128 columns is 2 pairs of all 32 lanes; groups a lane takes part in
  static constexpr int GROUP_PAIRS = 2, GROUPS = E / 4;
  __device__ static __forceinline__ int first_col(int lane) { return lane * W; }
  __device__ static __forceinline__ bool has(int p, int half, int left) { return 64 * p + (half ? SECOND : 0) < left; }
  __device__ static __forceinline__ int col_of(int p, int half) { return 64 * p + (half ? SECOND : 0); }
  __device__ static __forceinline__ float to_float(float x) { return x; }
  __device__ static __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
  __device__ static __forceinline__ float to_float(int8_t x) { return (float)x; }
  template <class T>
  __device__ static __forceinline__ void load(const T* at, int left, float2 (&x)[PAIRS]) {
    #pragma unroll
    for (int p = 0; p < PAIRS; ++p) {
      const T* c = at + 64 * p;
      x[p] = both(0.f);
      if constexpr (W == 1) {
        x[p] = make_float2(has(p, 0, left) ? to_float(c[0]) : 0.f, has(p, 1, left) ? to_float(c[32]) : 0.f);
      } else if (has(p, 0, left)) {
        if constexpr (sizeof(T) == 4) {
          x[p] = *reinterpret_cast<const float2*>(c);
        } else if constexpr (sizeof(T) == 2) {
          const uint32_t u = *reinterpret_cast<const uint32_t*>(c);
          x[p] = make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
        } else {
          const char2 u = *reinterpret_cast<const char2*>(c);
          x[p] = make_float2((float)u.x, (float)u.y);
        }
      }
    }
  }
  __device__ static __forceinline__ void store(float* at, int left, const float2 (&x)[PAIRS]) {
    #pragma unroll
    for (int p = 0; p < PAIRS; ++p) {
      if constexpr (W == 2) { if (has(p, 0, left)) *reinterpret_cast<float2*>(at + 64 * p) = x[p]; }
      else { if (has(p, 0, left)) at[64 * p] = x[p].x; if (has(p, 1, left)) at[64 * p + 32] = x[p].y; }
    }
  }
  __device__ static __forceinline__ void store(__nv_bfloat16* at, int left, const float2 (&x)[PAIRS]) {
    #pragma unroll
    for (int p = 0; p < PAIRS; ++p) {
      if constexpr (W == 2) { if (has(p, 0, left)) *reinterpret_cast<uint32_t*>(at + 64 * p) = pack_bf16x2(x[p].x, x[p].y); }
      else {
        if (has(p, 0, left)) at[64 * p] = __float2bfloat16_rn(x[p].x);
        if (has(p, 1, left)) at[64 * p + 32] = __float2bfloat16_rn(x[p].y);
      }
    }
  }
  // the bytes of one group, its first column at `at`
  __device__ static __forceinline__ void store_group(int8_t* at, int left, const uint2 (&b)[GROUP_PAIRS]) {
    #pragma unroll
    for (int p = 0; p < GROUP_PAIRS; ++p) {
      if constexpr (W == 2) { if (has(p, 0, left)) *reinterpret_cast<char2*>(at + 64 * p) = make_char2((int8_t)b[p].x, (int8_t)b[p].y); }
      else { if (has(p, 0, left)) at[64 * p] = (int8_t)b[p].x; if (has(p, 1, left)) at[64 * p + 32] = (int8_t)b[p].y; }
    }
  }
};

template <int L> struct Vector {
  static constexpr int LANES = L, PAIRS = 4, GROUP_PAIRS = 4, GROUPS = 1, GROUP_LANES = L < 16 ? L : 16;
  __device__ static __forceinline__ int first_col(int lane) { return (lane & (L - 1)) * 8; }
  __device__ static __forceinline__ bool has(int, int, int left) { return left > 0; }       // all 8 columns or none
  __device__ static __forceinline__ int col_of(int p, int half) { return 2 * p + half; }
  template <class T>
  __device__ static __forceinline__ void load(const T* at, int left, float2 (&x)[4]) {
    #pragma unroll
    for (int p = 0; p < 4; ++p) x[p] = both(0.f);
    if (left > 0) load8(at, x);
  }
  __device__ static __forceinline__ void store(float* at, int left, const float2 (&x)[4]) { if (left > 0) put8<true>(at, 0, x); }
  __device__ static __forceinline__ void store(__nv_bfloat16* at, int left, const float2 (&x)[4]) { if (left > 0) put8<false>(at, 0, x); }
  __device__ static __forceinline__ void store_group(int8_t* at, int left, const uint2 (&b)[4]) {
    if (left > 0) *reinterpret_cast<uint2*>(at) = pack_bytes(b);
  }
};

// per-column weights of a lane, `otherwise` where there are none
template <class A>
__device__ __forceinline__ void any_weights(const void* w, int32_t dtype, int col, int left, float otherwise, float2 (&g)[A::PAIRS]) {
  auto get = [&](int p, int half) {
    const int c = col + A::col_of(p, half);
    if (w == nullptr || !A::has(p, half, left)) return otherwise;
    return dtype == SAPO_DTYPE_F32 ? static_cast<const float*>(w)[c] : __bfloat162float(static_cast<const __nv_bfloat16*>(w)[c]);
  };
  #pragma unroll
  for (int p = 0; p < A::PAIRS; ++p) g[p] = make_float2(get(p, 0), get(p, 1));
}

// Where a warp is: `group` of the block's groups of wpr warps, warp w of its row; with U > 1 or fewer than 32 lanes a
// row (wpr = 1) a warp takes U rows per lane, neighbouring lanes' rows U apart.
struct AnyPlace { int group, groups, w; };
__device__ __forceinline__ AnyPlace any_place(int wpr) {
  const int warp = threadIdx.x >> 5;
  return AnyPlace{warp / wpr, (int)(blockDim.x >> 5) / wpr, warp % wpr};
}
constexpr int ANY_SLOTS = 16;                            // warps a row at most
constexpr int ANY_RED = 2 * (NORM_MAX_THREADS / 32 / 2) * ANY_SLOTS;   // groups of two warps and more use them

// U rows a lane at a time: U > 1 with several warps a row is U = 2 (both rows' sums cross the warps together).
// (16 columns and one row a lane: 96 registers, so that two blocks of up to 10 warps fit on an SM)
template <class TX, class A, int U>
__global__ void __maxnreg__((A::PAIRS == 8 && U == 1) ? 96 : 128) norm_fwd_any_kernel(NormFwdArgs a, int wpr) {
  wait_for_previous();
  let_next_start();
  constexpr bool REPLAY = sizeof(TX) == 1;
  constexpr int P = A::PAIRS, G = A::GROUPS, L = A::LANES, PER_WARP = U * (32 / L);
  constexpr bool ONE_WARP = L < 32 || U > 2;            // a row never crosses warps
  using Rows = Slots<U, L>;
  __shared__ __align__(16) float2 red[ANY_RED];
  for (int i = threadIdx.x; i < ANY_RED; i += blockDim.x) red[i] = make_float2(0.f, 0.f);
  __syncthreads();
  const int lane = threadIdx.x & 31;
  const AnyPlace at = any_place(wpr);
  const int col = at.w * 64 * P + A::first_col(lane), left = a.H - col;
  const float inv_h = 1.f / (float)a.H;
  const bool layer = a.kind == KIND_LAYER;
  float2 gam[P], bet[P];
  any_weights<A>(a.gamma, a.w_dtype, col, left, 1.f, gam);
  any_weights<A>(a.beta, a.w_dtype, col, left, 0.f, bet);
  int turn = 0;
  // the sums of U rows over all their columns: in the lanes of the row's slot (ONE_WARP), or in all lanes
  auto row_sums = [&](float (&s)[U], float (&t)[U]) {
    if constexpr (ONE_WARP) {
      const float mine = Rows::reduce(s, AddOp{});
      #pragma unroll
      for (int u = 0; u < U; ++u) t[u] = Rows::get(mine, u);
    } else {
      const float2 x = group_sum2<ANY_SLOTS>(s[0], U == 2 ? s[U - 1] : 0.f, wpr, at.w, at.group, red, turn);
      turn ^= 1;
      t[0] = x.x;
      if (U == 2) t[U - 1] = x.y;
    }
  };
  for (int64_t base = ((int64_t)blockIdx.x * at.groups + at.group) * PER_WARP; base < a.T;
       base += (int64_t)gridDim.x * at.groups * PER_WARP) {
    const int64_t row = base + (lane / L) * U;           // the lane's first row
    float2 x[U][P];
    int n[U];                                            // columns of the row from the lane's first one on
    #pragma unroll
    for (int u = 0; u < U; ++u) {
      n[u] = row + u < a.T ? left : 0;
      A::load((REPLAY ? reinterpret_cast<const TX*>(a.q.p) + (row + u) * a.q.ld : static_cast<const TX*>(a.x.p) + (row + u) * a.x.ld) + col, n[u], x[u]);
    }
    float mean[U], rstd[U];
    if (REPLAY) {
      #pragma unroll
      for (int u = 0; u < U; ++u) {
        mean[u] = row + u < a.T && layer ? a.mean[row + u] : 0.f;
        rstd[u] = row + u < a.T ? a.rstd[row + u] : 0.f;
        #pragma unroll
        for (int k = 0; k < G; ++k) {
          const int g = at.w * G + k + (lane & (L - 1)) / A::GROUP_LANES;
          const float2 s = both(row + u < a.T && g * Q8_GROUP < a.H ? a.q.scale[(row + u) * a.q.ld_scale + g] : 0.f);
          #pragma unroll
          for (int j = 0; j < A::GROUP_PAIRS; ++j) x[u][k * A::GROUP_PAIRS + j] = mul2(x[u][k * A::GROUP_PAIRS + j], s);
        }
      }
    } else {
      float s[U], t[U];
      #pragma unroll
      for (int u = 0; u < U; ++u) mean[u] = 0.f;
      if (layer) {
        #pragma unroll
        for (int u = 0; u < U; ++u) {
          float2 v = both(0.f);
          #pragma unroll
          for (int p = 0; p < P; ++p) v = add2(v, x[u][p]);
          s[u] = v.x + v.y;
        }
        row_sums(s, t);
        #pragma unroll
        for (int u = 0; u < U; ++u) mean[u] = t[u] * inv_h;
      }
      #pragma unroll
      for (int u = 0; u < U; ++u) {
        float2 v = both(0.f);
        #pragma unroll
        for (int p = 0; p < P; ++p) {
          const float2 d = add2(x[u][p], make_float2(A::has(p, 0, left) ? -mean[u] : 0.f, A::has(p, 1, left) ? -mean[u] : 0.f));
          v = fma2(d, d, v);
        }
        s[u] = v.x + v.y;
      }
      row_sums(s, t);
      #pragma unroll
      for (int u = 0; u < U; ++u) {
        rstd[u] = 1.f / sqrtf(t[u] * inv_h + a.eps);
        if (at.w == 0 && (lane & (L - 1)) == 0 && row + u < a.T) {
          if (a.mean != nullptr && layer) a.mean[row + u] = mean[u];
          if (a.rstd != nullptr) a.rstd[row + u] = rstd[u];
        }
      }
      if (a.q.p != nullptr) {
        // the groups of all U rows together: slot u G + k
        constexpr int N = U * G;
        using Q = Slots<N, A::GROUP_LANES>;
        float2 v[N][A::GROUP_PAIRS];
        uint2 bytes[N][A::GROUP_PAIRS];
        float scale; bool bad;
        #pragma unroll
        for (int i = 0; i < N; ++i)
          #pragma unroll
          for (int j = 0; j < A::GROUP_PAIRS; ++j) v[i][j] = x[i / G][(i % G) * A::GROUP_PAIRS + j];
        quantise<N, A::GROUP_LANES, A::GROUP_PAIRS>(v, bytes, scale, bad);
        #pragma unroll
        for (int i = 0; i < N; ++i)
          A::store_group(a.q.p + (row + i / G) * a.q.ld + col + (i % G) * Q8_GROUP, n[i / G] - (i % G) * Q8_GROUP, bytes[i]);
        const int64_t r = row + Q::slot() / G;
        const int g = at.w * G + Q::slot() % G + (lane & (L - 1)) / A::GROUP_LANES;
        if (Q::first() && r < a.T && g * Q8_GROUP < a.H) {
          a.q.scale[r * a.q.ld_scale + g] = scale;
          if (bad) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
        }
      }
    }
    auto finish = [&](auto* y) {
      #pragma unroll
      for (int u = 0; u < U; ++u) {
        #pragma unroll
        for (int p = 0; p < P; ++p) x[u][p] = fma2(mul2(add2(x[u][p], both(-mean[u])), both(rstd[u])), gam[p], bet[p]);
        A::store(y + (row + u) * a.y.ld + col, n[u], x[u]);
      }
    };
    if (a.y.dtype == SAPO_DTYPE_F32) finish(static_cast<float*>(a.y.p)); else finish(static_cast<__nv_bfloat16*>(a.y.p));
  }
}

template <class TX, class A, int U>
__global__ void __launch_bounds__(NORM_MAX_THREADS) norm_bwd_any_kernel(NormBwdArgs a, int wpr) {
  wait_for_previous();
  let_next_start();
  constexpr bool FROM_Q8 = sizeof(TX) == 1;
  constexpr int P = A::PAIRS, G = A::GROUPS, L = A::LANES, PER_WARP = U * (32 / L);
  constexpr bool ONE_WARP = L < 32 || U > 1;
  using Sums = Slots<2 * U, L>;                         // slot 2 u: sum of g, 2 u + 1: sum of g xh, of row u
  extern __shared__ __align__(16) float cols_acc[];     // [groups][2][H], of two groups or more
  __shared__ __align__(16) float2 red[ANY_RED];
  for (int i = threadIdx.x; i < ANY_RED; i += blockDim.x) red[i] = make_float2(0.f, 0.f);
  __syncthreads();
  const int lane = threadIdx.x & 31;
  const AnyPlace at = any_place(wpr);
  const int col = at.w * 64 * P + A::first_col(lane), left = a.H - col;
  const float inv_h = 1.f / (float)a.H;
  const bool layer = a.kind == KIND_LAYER;
  float2 gam[P], dg[P], db[P];
  any_weights<A>(a.gamma, a.w_dtype, col, left, 1.f, gam);
  #pragma unroll
  for (int p = 0; p < P; ++p) { dg[p] = both(0.f); db[p] = both(0.f); }
  int turn = 0;
  for (int64_t base = ((int64_t)blockIdx.x * at.groups + at.group) * PER_WARP; base < a.T;
       base += (int64_t)gridDim.x * at.groups * PER_WARP) {
    const int64_t row = base + (lane / L) * U;           // the lane's first row
    float2 x[U][P], g[U][P];
    float mean[U], rstd[U];
    int n[U];
    #pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool live = row + u < a.T;
      n[u] = live ? left : 0;
      A::load((FROM_Q8 ? reinterpret_cast<const TX*>(a.q.p) + (row + u) * a.q.ld : static_cast<const TX*>(a.x.p) + (row + u) * a.x.ld) + col, n[u], x[u]);
      mean[u] = live && layer ? a.mean[row + u] : 0.f;
      rstd[u] = live ? a.rstd[row + u] : 0.f;
    }
    auto load_dy = [&](const auto* dy) {
      #pragma unroll
      for (int u = 0; u < U; ++u) A::load(dy + (row + u) * a.dy.ld + col, n[u], g[u]);
    };
    if (a.dy.dtype == SAPO_DTYPE_F32) load_dy(static_cast<const float*>(a.dy.p)); else load_dy(static_cast<const __nv_bfloat16*>(a.dy.p));
    if (FROM_Q8) {
      #pragma unroll
      for (int u = 0; u < U; ++u)
        #pragma unroll
        for (int k = 0; k < G; ++k) {
          const int gr = at.w * G + k + (lane & (L - 1)) / A::GROUP_LANES;
          const float2 s = both(row + u < a.T && gr * Q8_GROUP < a.H ? a.q.scale[(row + u) * a.q.ld_scale + gr] : 0.f);
          #pragma unroll
          for (int j = 0; j < A::GROUP_PAIRS; ++j) x[u][k * A::GROUP_PAIRS + j] = mul2(x[u][k * A::GROUP_PAIRS + j], s);
        }
    }
    // (where a column does not exist dy is zero: it adds nothing to the sums)
    float s[2 * U];
    #pragma unroll
    for (int u = 0; u < U; ++u) {
      const float2 r2 = both(rstd[u]), minus = both(-mean[u]);
      float2 s1 = both(0.f), s2 = both(0.f);
      #pragma unroll
      for (int p = 0; p < P; ++p) {
        x[u][p] = mul2(add2(x[u][p], minus), r2);
        dg[p] = fma2(g[u][p], x[u][p], dg[p]);
        db[p] = add2(db[p], g[u][p]);
        g[u][p] = mul2(g[u][p], gam[p]);
        s1 = add2(s1, g[u][p]);
        s2 = fma2(g[u][p], x[u][p], s2);
      }
      s[2 * u] = s1.x + s1.y;
      s[2 * u + 1] = s2.x + s2.y;
    }
    float2 one = both(0.f);
    float slot_sum = 0.f;
    if constexpr (ONE_WARP) slot_sum = Sums::reduce(s, AddOp{});
    else { one = group_sum2<ANY_SLOTS>(s[0], s[1], wpr, at.w, at.group, red, turn); turn ^= 1; }
    auto finish = [&](auto* dx) {
      #pragma unroll
      for (int u = 0; u < U; ++u) {
        const float sum1 = ONE_WARP ? Sums::get(slot_sum, 2 * u) : one.x, sum2 = ONE_WARP ? Sums::get(slot_sum, 2 * u + 1) : one.y;
        const float2 r2 = both(rstd[u]), c1 = both(layer ? -sum1 * inv_h * rstd[u] : 0.f), c2 = both(-sum2 * inv_h * rstd[u]);
        #pragma unroll
        for (int p = 0; p < P; ++p) x[u][p] = fma2(x[u][p], c2, fma2(g[u][p], r2, c1));
        A::store(dx + (row + u) * a.dx.ld + col, n[u], x[u]);
      }
    };
    if (a.dx.dtype == SAPO_DTYPE_F32) finish(static_cast<float*>(a.dx.p)); else finish(static_cast<__nv_bfloat16*>(a.dx.p));
  }
  if (a.dgamma == nullptr && a.dbeta == nullptr) return;
  // the rows that shared a warp, then the groups' sums
  #pragma unroll
  for (int d = 16; d >= L; d >>= 1)
    #pragma unroll
    for (int p = 0; p < P; ++p) {
      dg[p] = add2(dg[p], make_float2(__shfl_xor_sync(0xffffffffu, dg[p].x, d), __shfl_xor_sync(0xffffffffu, dg[p].y, d)));
      db[p] = add2(db[p], make_float2(__shfl_xor_sync(0xffffffffu, db[p].x, d), __shfl_xor_sync(0xffffffffu, db[p].y, d)));
    }
  const bool alone = at.groups == 1;
  float* to = alone ? a.part + (int64_t)blockIdx.x * 2 * part_pitch(a.H) : cols_acc + at.group * 2 * a.H;
  const int second = alone ? part_pitch(a.H) : a.H;
  if (lane < L) {
    #pragma unroll
    for (int p = 0; p < P; ++p)
      #pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (!A::has(p, h, left)) continue;
        const int c = col + A::col_of(p, h);
        const float vg = h ? dg[p].y : dg[p].x, vb = h ? db[p].y : db[p].x;
        if (alone && gridDim.x == 1) {
          if (a.dgamma != nullptr) a.dgamma[c] = a.accumulate ? a.dgamma[c] + vg : vg;
          if (a.dbeta != nullptr) a.dbeta[c] = a.accumulate ? a.dbeta[c] + vb : vb;
        } else {
          to[c] = vg; to[second + c] = vb;
        }
      }
  }
  if (alone) return;
  __syncthreads();
  finish_columns<1>(a, cols_acc, at.groups, a.H);
}

template <bool RESTORE> struct CkptAny { static constexpr int GROUPS = RESTORE ? 4 : 2; };    // groups a warp takes at a time
// Checkpoints alone: a warp takes a group of 128 columns, N of them with all loads before the first use; addresses are
// stepped from group to group.
template <class TX, int W, bool RESTORE>
__global__ void __launch_bounds__(256) ckpt8_any_kernel(Ckpt8Args a, int64_t step_rows, int32_t step_groups) {
  wait_for_previous();
  let_next_start();
  constexpr int N = CkptAny<RESTORE>::GROUPS;
  using A = Cols<W, 4>;
  using S = Slots<N, 32>;
  const int32_t groups = ceil_div(a.H, Q8_GROUP);
  const int64_t id = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  const int col = A::first_col(threadIdx.x & 31);
  int64_t row = id / groups;
  int32_t g = (int32_t)(id - row * groups);
  TX* x = static_cast<TX*>(a.x.p) + row * a.x.ld + g * Q8_GROUP + col;
  int8_t* q = a.q.p + row * a.q.ld + g * Q8_GROUP + col;
  float* s = a.q.scale + row * a.q.ld_scale + g;
  const int64_t x_step = step_rows * a.x.ld + step_groups * Q8_GROUP, x_wrap = a.x.ld - (int64_t)groups * Q8_GROUP;
  const int64_t q_step = step_rows * a.q.ld + step_groups * Q8_GROUP, q_wrap = a.q.ld - (int64_t)groups * Q8_GROUP;
  const int64_t s_step = step_rows * a.q.ld_scale + step_groups, s_wrap = a.q.ld_scale - groups;
  const int32_t last_left = a.H - (groups - 1) * Q8_GROUP - col;       // columns from the lane's first one on, last group
  while (row < a.T) {
    if (!SAPO_IN_BOUNDS(row >= 0 && g >= 0 && g < groups && x - static_cast<TX*>(a.x.p) == row * a.x.ld + g * Q8_GROUP + col &&
                        q - a.q.p == row * a.q.ld + g * Q8_GROUP + col && s - a.q.scale == row * a.q.ld_scale + g))
      break;
    TX* xs[N]; int8_t* qs[N]; float* ss[N];
    int left[N]; bool in[N];
    float2 v[N][2]; float scale_of[N];
    #pragma unroll
    for (int k = 0; k < N; ++k) {
      xs[k] = x; qs[k] = q; ss[k] = s;
      in[k] = row < a.T;
      left[k] = !in[k] ? 0 : (g == groups - 1 ? last_left : Q8_GROUP);
      scale_of[k] = 0.f;
      if constexpr (RESTORE) { A::load((const int8_t*)q, left[k], v[k]); if (in[k]) scale_of[k] = *s; }
      else A::load((const TX*)x, left[k], v[k]);
      row += step_rows; g += step_groups; x += x_step; q += q_step; s += s_step;
      if (g >= groups) { g -= groups; ++row; x += x_wrap; q += q_wrap; s += s_wrap; }
    }
    if constexpr (RESTORE) {
      #pragma unroll
      for (int k = 0; k < N; ++k) {
        v[k][0] = mul2(v[k][0], both(scale_of[k]));
        v[k][1] = mul2(v[k][1], both(scale_of[k]));
        A::store(xs[k], left[k], v[k]);
      }
    } else {
      uint2 bytes[N][2];
      float scale; bool bad;
      quantise<N, 32, 2>(v, bytes, scale, bad);
      #pragma unroll
      for (int k = 0; k < N; ++k) {
        A::store_group(qs[k], left[k], bytes[k]);
        if (S::first() && S::slot() == k && in[k]) {
          *ss[k] = scale;
          if (bad) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
        }
      }
    }
  }
}

}  // namespace sapo
