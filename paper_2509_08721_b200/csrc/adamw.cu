// sapo_adamw_step: one AdamW step (Loshchilov & Hutter: Adam with the decay of the weights outside the moments) over a
// list of tensors in as few launches as their number allows; moments in 32 bits, or in 8 with an fp32 scale per 128.
//
// The 8-bit state holds m and the ROOT of v, which halves v's span of exponents.  m is rounded to the nearest code: its
// average moves by a tenth of a gradient a step, more than half a code.  v moves by a thousandth a step, far less than a
// code: to the nearest it would stand still once about ten gradients are in it, so its root is rounded up or down by a
// random number (16 bits of Philox, counted by element, tensor and step) that makes it right on average, and a root that
// is not zero never becomes zero (its smallest code is 2^-6 / 448 of the group's largest), so that no weight is divided by
// eps alone.
//
// Measured: 136 M weights, 32 bits, bf16 gradients 561 us (6.8 TB/s); 165 M weights in 24 tensors, 8 bits, fp32 gradients
// 470 us in a burst (6.4 TB/s), 565 sustained (80 instructions a weight: the power cap takes the clock to 1.55 GHz).
// HBM-bound: per weight 4 + 4 (master) + 2 or 4 (gradient) + 2 (bf16 copy) + 16 (32 bits) or 4.13 (8 bits) bytes.  A
// warp takes 512 consecutive elements (256 with 8-bit states, which are as much work as memory: more warps hide it better), all
// loads before the first use.
#include <cuda_bf16.h>

#include "common.cuh"
#include "float8.cuh"
#include "paired.cuh"
#include "philox.cuh"

namespace sapo {

constexpr int ADW_THREADS = 256;
// groups of 128 a warp takes at a time, and the elements of a warp and of a block
template <bool BITS8> constexpr int ADW_GROUPS = BITS8 ? 2 : 4;
template <bool BITS8> constexpr int ADW_WARP = ADW_GROUPS<BITS8> * F8_GROUP;
template <bool BITS8> constexpr int ADW_BLOCK = ADW_WARP<BITS8> * ADW_THREADS / 32;
constexpr int ADW_TENSORS = 32;                                     // tensors a launch takes (its parameters hold the list)

struct AdamWEntry {
  const float* master; float* master_out;
  const void* grad;
  const void* m; const void* v; void* m_out; void* v_out;
  const float* m_scale; const float* v_scale; float* m_scale_out; float* v_scale_out;
  __nv_bfloat16* copy;
  int64_t n;
  float lr_factor, decay;
  int32_t first_block;      // blocks of the launch before this tensor's
  int32_t number;           // of the tensor in the caller's list: part of the random counter
  int32_t vectors;          // every array starts on a boundary for vectors of four elements
};

struct AdamWArgs {
  AdamWEntry t[ADW_TENSORS];
  int32_t n_tensors;
  double lr, beta1, beta2;
  const float* lr_dev; const int32_t* step_dev; const float* grad_scale;
  float b1, b2, one_minus_b1, one_minus_b2, eps, inv_bias1, inv_bias2_root;
  uint32_t step, k0, k1;
  int32_t* status;
};

// 1 - b^t in 64 bits
__host__ __device__ inline double one_minus_power(double b, uint32_t t) {
  double p = 1.0;
  for (; t; t >>= 1, b *= b) if (t & 1u) p *= b;
  return 1.0 - p;
}

// Four neighbouring elements from p on, `left` of which exist (WHOLE: all four, on a boundary for one access).
struct Four { float v[4]; };
template <bool WHOLE>
__device__ __forceinline__ Four load4(const float* p, int left) {
  Four f;
  if (WHOLE) { const float4 x = *reinterpret_cast<const float4*>(p); f.v[0] = x.x; f.v[1] = x.y; f.v[2] = x.z; f.v[3] = x.w; }
  else {
    #pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = i < left ? p[i] : 0.f;
  }
  return f;
}
template <bool WHOLE>
__device__ __forceinline__ Four load4(const __nv_bfloat16* p, int left) {
  Four f;
  if (WHOLE) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    f.v[0] = __uint_as_float(x.x << 16); f.v[1] = __uint_as_float(x.x & 0xFFFF0000u);
    f.v[2] = __uint_as_float(x.y << 16); f.v[3] = __uint_as_float(x.y & 0xFFFF0000u);
  } else {
    #pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = i < left ? __bfloat162float(p[i]) : 0.f;
  }
  return f;
}
template <bool WHOLE>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int left) {
  if (WHOLE) return *reinterpret_cast<const uint32_t*>(p);
  uint32_t q = 0;
  #pragma unroll
  for (int i = 0; i < 4; ++i) if (i < left) q |= (uint32_t)p[i] << (8 * i);
  return q;
}
template <bool WHOLE>
__device__ __forceinline__ void store4(float* p, int left, const float (&v)[4]) {
  if (WHOLE) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  else {
    #pragma unroll
    for (int i = 0; i < 4; ++i) if (i < left) p[i] = v[i];
  }
}
template <bool WHOLE>
__device__ __forceinline__ void store4(__nv_bfloat16* p, int left, const float (&v)[4]) {
  if (WHOLE) {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  } else {
    #pragma unroll
    for (int i = 0; i < 4; ++i) if (i < left) p[i] = __float2bfloat16_rn(v[i]);
  }
}
template <bool WHOLE>
__device__ __forceinline__ void store_codes(uint8_t* p, int left, uint32_t q) {
  if (WHOLE) *reinterpret_cast<uint32_t*>(p) = q;
  else {
    #pragma unroll
    for (int i = 0; i < 4; ++i) if (i < left) p[i] = (uint8_t)(q >> (8 * i));
  }
}

// a b rounded by itself: the assembler fuses a paired product and a sum that follows into one rounding, so the products
// whose sum makes the state are not paired
__device__ __forceinline__ float2 product(float2 a, float2 b) { return make_float2(__fmul_rn(a.x, b.x), __fmul_rn(a.y, b.y)); }

// A root in units of its scale, rounded to one of the two codes around it: bits16 is 16 times a number uniform on [0, 65536).
__device__ __forceinline__ float round_root(float t, uint32_t bits16) {
  const uint32_t up = (__float_as_uint(fmaxf(t, 0.015625f)) + (bits16 | 8u)) & 0xFFF00000u;
  return t > 0.f ? __uint_as_float(up) : 0.f;            // (480, one step above the largest code, is stored as that one)
}
__device__ __forceinline__ float rcp_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Square roots of two numbers: an approximation of the inverse root and one step of Newton's method on it, s + (v - s s) / (2 s),
// with the residual exact.  Rounded correctly but for about one in 10^5 (one unit then); of v below the normal numbers 0.
__device__ __forceinline__ float2 root2(float2 v) {
  const float least = 1.17549435e-38f;
  float2 y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(fmaxf(v.x, least)));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(fmaxf(v.y, least)));
  const float2 s = mul2(v, y), r = fma2(fma2(make_float2(-s.x, -s.y), s, v), mul2(y, both(0.5f)), s);
  return make_float2(v.x >= least ? r.x : 0.f, v.y >= least ? r.y : 0.f);
}

// What a step has in common for the elements of a tensor
struct AdamWStep { float minus_lr, shrink, grad_scale, inv_bias1, inv_bias2_root; uint32_t step; };

// 512 elements of tensor t from `base` on.  WHOLE: they all exist, and every array can be read and written four at a time.
template <bool BITS8, class G, bool WHOLE>
__device__ __forceinline__ void adamw_run(const AdamWArgs& a, const AdamWEntry& t, const AdamWStep& c, int64_t base) {
  constexpr uint32_t ALL = 0xFFFFFFFFu;
  constexpr int GROUPS = ADW_GROUPS<BITS8>, WARP = ADW_WARP<BITS8>;
  const int lane = threadIdx.x & 31;
  const int64_t at = base + 4 * lane, group = base >> 7, groups = (t.n + F8_GROUP - 1) >> 7;
  const int left = WHOLE ? WARP : (int)max((int64_t)-WARP, min((int64_t)WARP, t.n - at));      // elements from this lane's first on
  Four g[GROUPS], w[GROUPS], m[GROUPS], v[GROUPS];
  uint32_t qm[GROUPS], qv[GROUPS];
  float sm[GROUPS], sv[GROUPS];
  #pragma unroll
  for (int u = 0; u < GROUPS; ++u) {
    g[u] = load4<WHOLE>(static_cast<const G*>(t.grad) + at + u * F8_GROUP, left - u * F8_GROUP);
    w[u] = load4<WHOLE>(t.master + at + u * F8_GROUP, left - u * F8_GROUP);
    if (BITS8) {
      qm[u] = load_codes<WHOLE>(static_cast<const uint8_t*>(t.m) + at + u * F8_GROUP, left - u * F8_GROUP);
      qv[u] = load_codes<WHOLE>(static_cast<const uint8_t*>(t.v) + at + u * F8_GROUP, left - u * F8_GROUP);
      const bool there = WHOLE || group + u < groups;
      sm[u] = there ? t.m_scale[group + u] : 0.f;
      sv[u] = there ? t.v_scale[group + u] : 0.f;
    } else {
      m[u] = load4<WHOLE>(static_cast<const float*>(t.m) + at + u * F8_GROUP, left - u * F8_GROUP);
      v[u] = load4<WHOLE>(static_cast<const float*>(t.v) + at + u * F8_GROUP, left - u * F8_GROUP);
    }
  }
  // random words: the eight elements of a counter belong to two lanes; each of them makes the counters of every other group
  uint32_t rnd[GROUPS][2];
  if (BITS8) {
    #pragma unroll
    for (int u = 0; u < GROUPS; u += 2) {
      const uint64_t eight = (uint64_t)(base + (u + (lane & 1)) * F8_GROUP + 4 * (lane & ~1)) >> 3;
      const uint4 r = philox4x32_10((uint32_t)eight, (uint32_t)(eight >> 32), (uint32_t)t.number, c.step, a.k0, a.k1);
      const bool odd = lane & 1;
      const uint32_t p = __shfl_xor_sync(ALL, odd ? r.x : r.z, 1), q = __shfl_xor_sync(ALL, odd ? r.y : r.w, 1);
      rnd[u][0] = odd ? p : r.x; rnd[u][1] = odd ? q : r.y;
      rnd[u + 1][0] = odd ? r.z : p; rnd[u + 1][1] = odd ? r.w : q;
    }
  }
  // moments and weights; afterwards m and v hold the new m and (8 bits) the new root
  uint32_t most_m[GROUPS], most_r[GROUPS];      // of the groups
  bool bad = false;
  #pragma unroll
  for (int u = 0; u < GROUPS; ++u) {
    float big = 0.f, mm = 0.f, mr = 0.f;
    float2 x[2], m0[2], v0[2];
    float root[4];
    if (BITS8) { f8_unpack4(qm[u], m[u].v); f8_unpack4(qv[u], root); }
    #pragma unroll
    for (int h = 0; h < 2; ++h) {
      x[h] = mul2(make_float2(g[u].v[2 * h], g[u].v[2 * h + 1]), both(c.grad_scale));
      m0[h] = make_float2(m[u].v[2 * h], m[u].v[2 * h + 1]);
      v0[h] = make_float2(v[u].v[2 * h], v[u].v[2 * h + 1]);
      if (BITS8) {
        m0[h] = mul2(m0[h], both(sm[u]));
        const float2 r = mul2(make_float2(root[2 * h], root[2 * h + 1]), both(sv[u]));
        v0[h] = mul2(r, r);
      }
      big = max_nan(big, max_nan(fabsf(x[h].x), fabsf(x[h].y)));
    }
    // Squares that may leave the fp32 range, and what is not finite, are looked at one by one.  Products and sums are
    // rounded one by one: the state is the same to the bit however a compiler would fuse them.
    const bool plain = __all_sync(ALL, big < 1e18f);
    #pragma unroll
    for (int h = 0; h < 2; ++h) {
      float2 m1 = add2(product(both(a.b1), m0[h]), product(both(a.one_minus_b1), x[h]));
      float2 v1 = add2(product(both(a.b2), v0[h]), product(mul2(both(a.one_minus_b2), x[h]), x[h]));
      const float2 was = make_float2(w[u].v[2 * h], w[u].v[2 * h + 1]);
      bool fine[2] = {true, true};
      if (!plain) {
        fine[0] = fabsf(x[h].x) < __int_as_float(0x7f800000); fine[1] = fabsf(x[h].y) < __int_as_float(0x7f800000);
        bad = bad || !fine[0] || !fine[1];
        m1 = make_float2(fine[0] ? m1.x : m0[h].x, fine[1] ? m1.y : m0[h].y);
        v1 = make_float2(fine[0] ? fminf(v1.x, 3.402823466e38f) : v0[h].x, fine[1] ? fminf(v1.y, 3.402823466e38f) : v0[h].y);
      }
      const float2 r1 = BITS8 ? root2(v1) : make_float2(sqrtf(v1.x), sqrtf(v1.y));
      const float2 above = mul2(m1, both(c.inv_bias1)), below = fma2(r1, both(c.inv_bias2_root), both(a.eps));
      const float2 now = fma2(both(c.minus_lr), mul2(above, make_float2(rcp_fast(below.x), rcp_fast(below.y))), mul2(was, both(c.shrink)));
      w[u].v[2 * h] = fine[0] ? now.x : was.x; w[u].v[2 * h + 1] = fine[1] ? now.y : was.y;
      m[u].v[2 * h] = m1.x; m[u].v[2 * h + 1] = m1.y;
      v[u].v[2 * h] = BITS8 ? r1.x : v1.x; v[u].v[2 * h + 1] = BITS8 ? r1.y : v1.y;
      if (BITS8) { mm = fmaxf(mm, fmaxf(fabsf(m1.x), fabsf(m1.y))); mr = fmaxf(mr, fmaxf(r1.x, r1.y)); }
    }
    store4<WHOLE>(t.master_out + at + u * F8_GROUP, left - u * F8_GROUP, w[u].v);
    if (t.copy != nullptr) store4<WHOLE>(t.copy + at + u * F8_GROUP, left - u * F8_GROUP, w[u].v);
    if (BITS8) {
      most_m[u] = __reduce_max_sync(ALL, __float_as_uint(mm));
      most_r[u] = __reduce_max_sync(ALL, __float_as_uint(mr));
    } else {
      store4<WHOLE>(static_cast<float*>(t.m_out) + at + u * F8_GROUP, left - u * F8_GROUP, m[u].v);
      store4<WHOLE>(static_cast<float*>(t.v_out) + at + u * F8_GROUP, left - u * F8_GROUP, v[u].v);
    }
  }
  if (BITS8) {
    // the divisions of the groups (of m, then of the root) are done by a lane each
    uint32_t mine = 0;
    #pragma unroll
    for (int u = 0; u < GROUPS; ++u) {
      if ((lane & (2 * GROUPS - 1)) == u) mine = most_m[u];
      if ((lane & (2 * GROUPS - 1)) == GROUPS + u) mine = most_r[u];
    }
    float scale, inv;
    f8_group(__uint_as_float(mine), scale, inv);
    const int64_t own = group + (lane & (GROUPS - 1));
    if (lane < 2 * GROUPS && (WHOLE || own < groups)) (lane < GROUPS ? t.m_scale_out : t.v_scale_out)[own] = scale;
    #pragma unroll
    for (int u = 0; u < GROUPS; ++u) {
      const float2 im = both(__shfl_sync(ALL, inv, u)), ir = both(__shfl_sync(ALL, inv, GROUPS + u));
      const float2 x = mul2(make_float2(m[u].v[0], m[u].v[1]), im), y = mul2(make_float2(m[u].v[2], m[u].v[3]), im);
      store_codes<WHOLE>(static_cast<uint8_t*>(t.m_out) + at + u * F8_GROUP, left - u * F8_GROUP, f8_pack4(x.x, x.y, y.x, y.y));
      const float2 p = mul2(make_float2(v[u].v[0], v[u].v[1]), ir), q = mul2(make_float2(v[u].v[2], v[u].v[3]), ir);
      store_codes<WHOLE>(static_cast<uint8_t*>(t.v_out) + at + u * F8_GROUP, left - u * F8_GROUP,
                  f8_pack4(round_root(p.x, (rnd[u][0] << 4) & 0xFFFF0u), round_root(p.y, (rnd[u][0] >> 12) & 0xFFFF0u),
                           round_root(q.x, (rnd[u][1] << 4) & 0xFFFF0u), round_root(q.y, (rnd[u][1] >> 12) & 0xFFFF0u)));
    }
  }
  if (bad) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
}

template <bool BITS8, class G>
__global__ void __launch_bounds__(ADW_THREADS, BITS8 ? 5 : 3) adamw_kernel(const __grid_constant__ AdamWArgs a) {
  wait_for_previous();
  const int warp = threadIdx.x >> 5;
  int lo = 0, hi = a.n_tensors - 1;            // the last tensor whose first block is not behind this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.t[mid].first_block <= (int)blockIdx.x) lo = mid; else hi = mid - 1;
  }
  const AdamWEntry& t = a.t[lo];
  float inv_bias1 = a.inv_bias1, inv_bias2_root = a.inv_bias2_root;
  uint32_t step = a.step;
  if (a.step_dev != nullptr) {
    __shared__ float bias[2];
    step = (uint32_t)max(*a.step_dev, 1);
    if (threadIdx.x == 0) { bias[0] = (float)(1.0 / one_minus_power(a.beta1, step)); bias[1] = (float)(1.0 / sqrt(one_minus_power(a.beta2, step))); }
    __syncthreads();
    inv_bias1 = bias[0]; inv_bias2_root = bias[1];
  }
  const int64_t base = (int64_t)((int)blockIdx.x - t.first_block) * ADW_BLOCK<BITS8> + (int64_t)warp * ADW_WARP<BITS8>;
  if (base >= t.n) return;
  const double lr = (a.lr_dev != nullptr ? (double)*a.lr_dev : a.lr) * (double)t.lr_factor;
  const AdamWStep c{-(float)lr, (float)(1.0 - lr * (double)t.decay), a.grad_scale != nullptr ? *a.grad_scale : 1.f, inv_bias1, inv_bias2_root, step};
  if (t.vectors && base + ADW_WARP<BITS8> <= t.n) adamw_run<BITS8, G, true>(a, t, c, base);
  else                                     adamw_run<BITS8, G, false>(a, t, c, base);
}

static bool multiple_of(const void* p, size_t k) { return reinterpret_cast<uintptr_t>(p) % k == 0; }

// one launch per 32 tensors of the list that are of this kind
template <bool BITS8, class G>
static int launch_adamw(const sapo_adamw_tensor* list, int32_t n, AdamWArgs& a, cudaStream_t st) {
  constexpr int g_dtype = sizeof(G) == 2 ? SAPO_DTYPE_BF16 : SAPO_DTYPE_F32;
  int64_t blocks = 0;
  a.n_tensors = 0;
  const auto launch = [&]() -> int {
    if (a.n_tensors == 0) return SAPO_OK;
    KernelScope scope(SAPO_K_ADAMW, st);
    const int rc = launch_overlapped(adamw_kernel<BITS8, G>, dim3((unsigned)blocks), ADW_THREADS, 0, 0, st, a);
    blocks = 0; a.n_tensors = 0;
    return rc;
  };
  for (int32_t i = 0; i < n; ++i) {
    const sapo_adamw_tensor& t = list[i];
    if (t.n == 0 || (t.state_bits == 8) != BITS8 || t.grad_dtype != g_dtype) continue;
    const int64_t need = ceil_div<int64_t>(t.n, ADW_BLOCK<BITS8>);
    if (a.n_tensors == ADW_TENSORS || blocks + need > 0x7FFFFFFF) {
      const int rc = launch();
      if (rc != SAPO_OK) return rc;
    }
    const size_t state = BITS8 ? 4 : 16;
    const bool vectors = aligned16(t.master) && aligned16(t.master_out) && multiple_of(t.grad, 4 * sizeof(G)) && multiple_of(t.m, state) &&
                         multiple_of(t.v, state) && multiple_of(t.m_out, state) && multiple_of(t.v_out, state) && multiple_of(t.copy_bf16, 8);
    a.t[a.n_tensors++] = AdamWEntry{t.master, t.master_out, t.grad, t.m, t.v, t.m_out, t.v_out, t.m_scale, t.v_scale, t.m_scale_out,
                                    t.v_scale_out, static_cast<__nv_bfloat16*>(t.copy_bf16), t.n, t.lr_factor, t.weight_decay,
                                    (int32_t)blocks, i, vectors ? 1 : 0};
    blocks += need;
  }
  return launch();
}

}  // namespace sapo

extern "C" int sapo_adamw_step(const sapo_adamw_tensor* h_tensors, int32_t n_tensors, const sapo_adamw_cfg* h_cfg, int32_t* status,
                               void* stream) {
  using namespace sapo;
  if (n_tensors < 0 || (n_tensors > 0 && !h_tensors) || !h_cfg || !status) return SAPO_ERR_INVALID_ARG;
  const sapo_adamw_cfg& c = *h_cfg;
  if (!(c.beta1 >= 0. && c.beta1 < 1.) || !(c.beta2 >= 0. && c.beta2 < 1.) || !(c.eps >= 0. && c.eps < 1e30) || !(c.lr - c.lr == 0.)) return SAPO_ERR_INVALID_ARG;
  if (!c.step_dev && c.step < 1) return SAPO_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const sapo_adamw_tensor& t = h_tensors[i];
    if (t.n < 0 || (t.state_bits != 8 && t.state_bits != 32) || (t.grad_dtype != SAPO_DTYPE_BF16 && t.grad_dtype != SAPO_DTYPE_F32))
      return SAPO_ERR_INVALID_ARG;
    if (t.n == 0) continue;
    if (!t.master || !t.master_out || !t.grad || !t.m || !t.v || !t.m_out || !t.v_out) return SAPO_ERR_INVALID_ARG;
    if (t.state_bits == 8 && (!t.m_scale || !t.v_scale || !t.m_scale_out || !t.v_scale_out)) return SAPO_ERR_INVALID_ARG;
    const size_t g = t.grad_dtype == SAPO_DTYPE_BF16 ? 2 : 4, s = t.state_bits == 8 ? 1 : 4;
    if (!multiple_of(t.master, 4) || !multiple_of(t.master_out, 4) || !multiple_of(t.grad, g) || !multiple_of(t.m, s) || !multiple_of(t.v, s) ||
        !multiple_of(t.m_out, s) || !multiple_of(t.v_out, s) || !multiple_of(t.copy_bf16, 2))
      return SAPO_ERR_INVALID_ARG;
    if (!(t.weight_decay - t.weight_decay == 0.f) || !(t.lr_factor - t.lr_factor == 0.f)) return SAPO_ERR_INVALID_ARG;
    if (ceil_div<int64_t>(t.n, ADW_BLOCK<true>) > 0x7FFFFFFF) return SAPO_ERR_UNSUPPORTED_SHAPE;
  }
  if (current_device() < 0) return SAPO_ERR_CUDA;
  AdamWArgs a;
  a.lr = c.lr; a.beta1 = c.beta1; a.beta2 = c.beta2;
  a.lr_dev = c.lr_dev; a.step_dev = c.step_dev; a.grad_scale = c.grad_scale;
  a.b1 = (float)c.beta1; a.b2 = (float)c.beta2;
  a.one_minus_b1 = (float)(1. - c.beta1); a.one_minus_b2 = (float)(1. - c.beta2);
  a.eps = (float)c.eps;
  a.step = (uint32_t)(c.step < 1 ? 1 : c.step);
  a.inv_bias1 = (float)(1. / one_minus_power(c.beta1, a.step));
  a.inv_bias2_root = (float)(1. / sqrt(one_minus_power(c.beta2, a.step)));
  a.k0 = (uint32_t)c.seed; a.k1 = (uint32_t)(c.seed >> 32);
  a.status = status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int rc = launch_adamw<true, __nv_bfloat16>(h_tensors, n_tensors, a, st);
  if (rc == SAPO_OK) rc = launch_adamw<true, float>(h_tensors, n_tensors, a, st);
  if (rc == SAPO_OK) rc = launch_adamw<false, __nv_bfloat16>(h_tensors, n_tensors, a, st);
  if (rc == SAPO_OK) rc = launch_adamw<false, float>(h_tensors, n_tensors, a, st);
  return rc;
}
