// sapo_sample: draws one token of every row of logits, with temperature, top-k, top-p and min-p, from a 64-bit random
// number per row.
//
// The draw is a race of exponentials: token i with weight w_i = exp((z_i - zmax) / T) finishes at e_i / w_i, where e_i is
// a unit exponential made of 32 random bits of (the row's number, i); the first to finish wins, which token i does with
// probability w_i / sum w.  Against a search in the cumulated weights this needs no prefix sums along the vocabulary,
// splits over any number of blocks, and its outcome hangs on two numbers instead of on a long rounded sum.
//
// A cluster of 1 to 8 blocks holds a row in shared memory and walks over it there: the largest logit; the sums of
// weights; with top-k or top-p the place where the sorted row is cut; then the race.  Only a token with
// e_i < L w_i / sum w can win unless nobody does that well (probability exp(-L)), and e_i >= n_i 2^-32, so the race
// compares the upper 16 random bits of a token (eight tokens share one call of the generator) and only the about L
// tokens of a row that pass are worked out, in 64 bits.  Should none do well enough, every token is.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <math_constants.h>

#include "common.cuh"
#include "paired.cuh"
#include "philox.cuh"
#include "umma.cuh"

namespace sapo {
namespace cg = cooperative_groups;
using umma::ex2;

constexpr int SMP_THREADS = 512;
constexpr int SMP_WARPS = SMP_THREADS / 32;
constexpr int SMP_MAX_CLUSTER = 8;
constexpr int SMP_BINS = 2048;
constexpr float SMP_BINS_PER_OCTAVE = 64.f;   // the last bin takes everything below 2^-32 of the largest weight
constexpr int SMP_LIST = 256;                 // candidates a block keeps
constexpr int SMP_SORT = SMP_THREADS;         // tokens that are sorted at once, one a thread
constexpr float SMP_LEAD = 16.f;              // L: no candidate wins with probability 1e-7
constexpr float SMP_LOG2E = 1.4426950408889634f;
constexpr size_t SMP_MAX_PIECE = 180 * 1024;  // bytes of a row a block can hold

struct SampleArgs {
  const void* z; int64_t ld; int32_t B, V, piece;      // piece: tokens a block holds, a multiple of 8
  const int64_t* seeds;
  const float* temperature; const int32_t* top_k; const float* top_p; const float* min_p;    // one a row, or nullptr:
  float temperature_all; int32_t top_k_all; float top_p_all, min_p_all;                      // these
  int32_t* ids; float* logp; int32_t* status;
};

struct Cut { uint32_t bin, before, count, mass_lo, mass_hi, before_lo, before_hi; };   // of a bin, and of the bins in front of it
struct Last { uint32_t key, index, kept_lo, kept_hi; };                                 // the last token that stays, and the mass up to it

struct SampleShared {
  uint32_t slots[2][SMP_MAX_CLUSTER][8];    // what the blocks of the cluster tell one another; two sets, taken in turn
  uint32_t warp[2][SMP_WARPS][4];
  uint32_t scan[SMP_WARPS][4];
  Cut cut;
  Last last;
  uint32_t n_list, n_sort;
  uint32_t list[SMP_LIST];                  // candidates of the race
  uint64_t sort[SMP_SORT];                  // tokens to be put in order: key, and the index from above
  uint32_t count[SMP_BINS], mass_lo[SMP_BINS], mass_hi[SMP_BINS];   // of the tokens in a bin; mass in units of 2^-40
};

// order-preserving map of a float to an unsigned integer (both zeros are equal)
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }
// w (at most 1) in units of 2^-40, to the nearest
__device__ __forceinline__ uint64_t fixed_mass(float w) {
  const float f = w * 1099511627776.f;
  const uint32_t high = (uint32_t)(f * 9.5367431640625e-7f);          // f 2^-20, truncated
  return ((uint64_t)high << 20) + __float2uint_rn(f - (float)high * 1048576.f);
}
__device__ __forceinline__ uint64_t join64(uint32_t lo, uint32_t hi) { return ((uint64_t)hi << 32) | lo; }

template <class T> struct Vec;      // eight tokens of a row
template <> struct Vec<float> {
  static __device__ __forceinline__ void get(const float* p, float (&z)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    z[0] = a.x; z[1] = a.y; z[2] = a.z; z[3] = a.w; z[4] = b.x; z[5] = b.y; z[6] = b.z; z[7] = b.w;
  }
  static __device__ __forceinline__ float most(const float* p) {
    float z[8];
    get(p, z);
    return max_nan(max_nan(max_nan(z[0], z[1]), max_nan(z[2], z[3])), max_nan(max_nan(z[4], z[5]), max_nan(z[6], z[7])));
  }
};
template <> struct Vec<__nv_bfloat16> {
  static __device__ __forceinline__ void get(const __nv_bfloat16* p, float (&z)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
    #pragma unroll
    for (int i = 0; i < 4; ++i) { z[2 * i] = __uint_as_float(w[i] << 16); z[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
  static __device__ __forceinline__ float most(const __nv_bfloat16* p) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const __nv_bfloat162* w = reinterpret_cast<const __nv_bfloat162*>(&a);
    const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(w[0], w[1]), __hmax2_nan(w[2], w[3]));
    return max_nan(__low2float(m), __high2float(m));
  }
};
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }

template <class T>
__global__ void __launch_bounds__(SMP_THREADS, 2) sample_kernel(const SampleArgs a) {
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t C = cluster.num_blocks(), rank = cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  SampleShared& sh = *reinterpret_cast<SampleShared*>(smem_raw);
  T* piece = reinterpret_cast<T*>(smem_raw + ((sizeof(SampleShared) + 15) & ~size_t(15)));
  int turn = 0;

  auto barrier = [&]() { if (C > 1) cluster.sync(); else __syncthreads(); };
  // Tell every block of the cluster W words (of the first threads, the same in each) and wait; returns those of all blocks.
  auto exchange = [&](const uint32_t* v, int W) -> const uint32_t (*)[8] {
    const int t = turn;
    turn ^= 1;
    if (tid < (int)C) {
      uint32_t* to = cluster.map_shared_rank(&sh.slots[t][rank][0], tid);
      for (int i = 0; i < W; ++i) to[i] = v[i];
    }
    barrier();
    return sh.slots[t];
  };
  // Combine the words of every thread of the cluster; op(x, y) folds y into x; all threads get the result.  One warp
  // combines what the warps of a block have, and tells the blocks.
  auto reduce = [&](auto& v, auto op) {
    constexpr int W = sizeof(v) / 4;
    auto fold = [&](int widest) {
      #pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        if (d > widest) continue;
        uint32_t o[W];
        #pragma unroll
        for (int i = 0; i < W; ++i) o[i] = __shfl_xor_sync(0xFFFFFFFFu, v[i], d);
        op(v, o);
      }
    };
    fold(16);
    uint32_t (*each)[4] = sh.warp[turn];
    if (lane == 0)
      for (int i = 0; i < W; ++i) each[warp][i] = v[i];
    __syncthreads();
    if (warp == 0) {
      for (int i = 0; i < W; ++i) v[i] = each[lane & (SMP_WARPS - 1)][i];
      fold(SMP_WARPS / 2);
    }
    const uint32_t (*all)[8] = exchange(v, W);
    for (int i = 0; i < W; ++i) v[i] = all[0][i];
    for (uint32_t r = 1; r < C; ++r) op(v, all[r]);
  };
  auto add = [](uint32_t& x, uint32_t y) { x = __float_as_uint(__uint_as_float(x) + __uint_as_float(y)); };

  cluster.sync();                      // every block's shared memory is there before the first store to it
  wait_for_previous();
  const int row = blockIdx.x / C;
  const uint32_t begin = rank * (uint32_t)a.piece;
  const int n = max(0, min(a.piece, a.V - (int)begin));       // tokens of this block
  const int n_vec = (n + 7) / 8;

  // ---- the row's piece into shared memory: a thread fetches the eights of tokens that it will look at
  {
    const T* from = static_cast<const T*>(a.z) + (int64_t)row * a.ld + begin;
    const bool aligned = (reinterpret_cast<uintptr_t>(from) & 15u) == 0;
    for (int v = tid; v < n_vec; v += SMP_THREADS) {
      if (aligned && 8 * v + 8 <= n) {
        #pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                       ::"r"(umma::smem_u32(reinterpret_cast<uint8_t*>(piece + 8 * v) + 16 * h)),
                         "l"(reinterpret_cast<const uint8_t*>(from + 8 * v) + 16 * h) : "memory");
      } else {
        for (int i = 8 * v; i < 8 * v + 8; ++i) piece[i] = i < n ? from[i] : T(-CUDART_INF_F);   // behind the end: no weight
      }
    }
  }
  const float temperature = a.temperature ? a.temperature[row] : a.temperature_all;
  const float min_p = a.min_p ? a.min_p[row] : a.min_p_all, top_p = a.top_p ? a.top_p[row] : a.top_p_all;
  int32_t top_k = a.top_k ? a.top_k[row] : a.top_k_all;
  if (top_k <= 0 || top_k >= a.V) top_k = 0;
  const uint32_t k0 = (uint32_t)a.seeds[row], k1 = (uint32_t)((uint64_t)a.seeds[row] >> 32);
  const bool greedy = temperature == 0.f || top_k == 1 || top_p <= 0.f;
  const bool by_mass = top_p < 1.f && !greedy, by_count = top_k > 0 && !greedy, cuts = by_mass || by_count;
  if (cuts) for (int i = tid; i < SMP_BINS; i += SMP_THREADS) { sh.count[i] = 0; sh.mass_lo[i] = 0; sh.mass_hi[i] = 0; }
  if (tid == 0) { sh.n_list = 0; sh.n_sort = 0; }
  asm volatile("cp.async.wait_all;" ::: "memory");

  // ---- the largest logit: of the block, and of the row.  Without top-k and top-p the sums below are formed against the
  //      block's and told together with it.
  const bool settings_ok = temperature >= 0.f && temperature < CUDART_INF_F && min_p >= 0.f && top_p == top_p;
  const bool alone = !cuts && settings_ok && !(min_p > 0.f);
  uint32_t top[1];
  {
    float m = -CUDART_INF_F;
    for (int v = tid; v < n_vec; v += SMP_THREADS) m = max_nan(m, Vec<T>::most(piece + 8 * v));
    top[0] = __float_as_uint(m);
    auto larger = [](uint32_t* x, const uint32_t* y) { x[0] = __float_as_uint(max_nan(__uint_as_float(x[0]), __uint_as_float(y[0]))); };
    if (alone) {
      #pragma unroll
      for (int d = 16; d > 0; d >>= 1) { const uint32_t o = __shfl_xor_sync(0xFFFFFFFFu, top[0], d); larger(top, &o); }
      if (lane == 0) sh.scan[warp][0] = top[0];
      __syncthreads();
      top[0] = sh.scan[lane & (SMP_WARPS - 1)][0];
      #pragma unroll
      for (int d = SMP_WARPS / 2; d > 0; d >>= 1) { const uint32_t o = __shfl_xor_sync(0xFFFFFFFFu, top[0], d); larger(top, &o); }
    } else reduce(top, larger);
  }
  float zmax = __uint_as_float(top[0]);
  auto bad_row = [&]() {                              // the same in all blocks, behind a barrier: nothing touches another block any more
    if (zmax < CUDART_INF_F && zmax > -CUDART_INF_F && settings_ok) return false;
    if (rank == 0 && tid == 0) {
      a.ids[row] = -1; a.logp[row] = 0.f;
      if (!settings_ok || zmax != -CUDART_INF_F) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
    }
    return true;
  };
  if (!alone && bad_row()) return;
  // distance of a token from the largest, in octaves of its weight: (zmax - z) scale, never 0 * inf
  const float scale = greedy ? SMP_LOG2E : fminf(SMP_LOG2E / temperature, 1e30f);
  const float floor_octaves = min_p > 0.f && !greedy ? fmaxf(-log2f(min_p), 0.f) : CUDART_INF_F;     // kept up to here
  auto octaves = [&](float z) -> float { return (zmax - z) * scale; };
  auto bin_of = [&](float o) { return (uint32_t)fminf(o * SMP_BINS_PER_OCTAVE, (float)(SMP_BINS - 1)); };
  auto into_bin = [&](uint32_t bin, float o) {
    atomicAdd(&sh.count[bin], 1u);
    if (!by_mass) return;
    const uint64_t m = fixed_mass(ex2(-o));
    const uint32_t lo = (uint32_t)m, was = atomicAdd(&sh.mass_lo[bin], lo), hi = (uint32_t)(m >> 32) + (was + lo < was);
    if (hi) atomicAdd(&sh.mass_hi[bin], hi);
  };

  // ---- sums of the weights at temperature 1 and at the row's, of the tokens that min_p keeps; the first token with the
  //      largest logit; for top-k and top-p a histogram of the octaves, without the tokens of its last bin
  uint32_t sums[4];
  {
    float s1 = 0.f, sT = 0.f, far = 0.f;
    uint32_t first = 0xFFFFFFFFu;
    // (a block of -inf, or with a NaN or +inf, has no largest logit to go by: its sums are 0, or the row is bad)
    const float ref = fabsf(zmax) < CUDART_INF_F ? zmax : 0.f;
    const bool other = !greedy && !cuts && (scale != SMP_LOG2E || floor_octaves < CUDART_INF_F);
    for (int v = tid; v < n_vec; v += SMP_THREADS) {
      float z[8];
      Vec<T>::get(piece + 8 * v, z);
      float p[2] = {0.f, 0.f};
      #pragma unroll
      for (int i = 0; i < 8; ++i) p[i & 1] += ex2((z[i] - ref) * SMP_LOG2E);
      s1 += p[0] + p[1];
      if (cuts) {
        #pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float o = octaves(z[i]);
          if (o < (SMP_BINS - 1) / SMP_BINS_PER_OCTAVE) into_bin(bin_of(o), o);      // (tokens behind the end are infinitely far)
          else if (by_mass) far += ex2(-o);
        }
      } else if (other) {
        #pragma unroll
        for (int i = 0; i < 8; ++i) { const float o = (ref - z[i]) * scale; sT += o <= floor_octaves ? ex2(-o) : 0.f; }
      } else if (greedy) {
        #pragma unroll
        for (int i = 7; i >= 0; --i) if (z[i] == zmax) first = min(first, begin + 8 * v + i);
      }
    }
    sums[0] = __float_as_uint(s1); sums[1] = __float_as_uint(other ? sT : s1); sums[2] = first; sums[3] = __float_as_uint(far);
    if (alone) {
      // words of a block: its largest logit, its sums against that, its first token with it
      uint32_t v[4] = {sums[0], sums[1], first, top[0]};
      #pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        add(v[0], __shfl_xor_sync(0xFFFFFFFFu, v[0], d));
        if (other) add(v[1], __shfl_xor_sync(0xFFFFFFFFu, v[1], d));
        if (greedy) v[2] = min(v[2], __shfl_xor_sync(0xFFFFFFFFu, v[2], d));
      }
      if (lane == 0)
        for (int i = 0; i < 3; ++i) sh.warp[turn][warp][i] = v[i];
      __syncthreads();
      if (warp == 0) {
        for (int i = 0; i < 3; ++i) v[i] = sh.warp[turn][lane & (SMP_WARPS - 1)][i];
        #pragma unroll
        for (int d = SMP_WARPS / 2; d > 0; d >>= 1) {
          add(v[0], __shfl_xor_sync(0xFFFFFFFFu, v[0], d));
          add(v[1], __shfl_xor_sync(0xFFFFFFFFu, v[1], d));
          v[2] = min(v[2], __shfl_xor_sync(0xFFFFFFFFu, v[2], d));
        }
        if (!other) v[1] = v[0];
      }
      const uint32_t (*all)[8] = exchange(v, 4);
      zmax = -CUDART_INF_F;
      for (uint32_t r = 0; r < C; ++r) zmax = max_nan(zmax, __uint_as_float(all[r][3]));
      if (bad_row()) return;
      s1 = 0.f; sT = 0.f; first = 0xFFFFFFFFu;
      for (uint32_t r = 0; r < C; ++r) {
        const float less = zmax - __uint_as_float(all[r][3]);
        s1 += __uint_as_float(all[r][0]) * ex2(-less * SMP_LOG2E);
        sT += __uint_as_float(all[r][1]) * ex2(-less * scale);
        if (less == 0.f) first = min(first, all[r][2]);
      }
      sums[0] = __float_as_uint(s1); sums[1] = __float_as_uint(sT); sums[2] = first;
    } else {
      reduce(sums, [&](uint32_t* x, const uint32_t* y) { add(x[0], y[0]); add(x[1], y[1]); x[2] = min(x[2], y[2]); add(x[3], y[3]); });
    }
  }
  const float log_sum = logf(__uint_as_float(sums[0]));
  if (greedy) {
    if (rank == 0 && tid == 0) { a.ids[row] = (int32_t)sums[2]; a.logp[row] = -log_sum; }
    return;
  }
  float weight = __uint_as_float(sums[1]);       // of the tokens in the race
  // the time at which a token finishes, in 64 bits
  auto finish = [&](uint32_t token, float z) -> double {
    const uint32_t half = token & 7u, s = 16 * (half & 1u);
    uint32_t bits = 0;
    #pragma unroll 1
    for (uint32_t part = 0; part < 2; ++part) {
      const uint4 r = philox4x32_10(token >> 3, part, 0, 0, k0, k1);
      const uint32_t w = half < 2 ? r.x : half < 4 ? r.y : half < 6 ? r.z : r.w;
      bits = (bits << 16) | ((w >> s) & 0xFFFFu);
    }
    const double e = -log1p(-((double)bits + 0.5) * 2.3283064365386963e-10);
    return e * exp(((double)zmax - (double)z) * fmin(1.0 / (double)temperature, 1e30));
  };
  // first to finish, the lower index where two finish together; words: time, index, a flag
  auto earlier = [](uint32_t* x, const uint32_t* y) {
    const double p = __longlong_as_double((long long)join64(x[0], x[1])), q = __longlong_as_double((long long)join64(y[0], y[1]));
    x[3] |= y[3];
    if (q < p || (q == p && y[2] < x[2])) { x[0] = y[0]; x[1] = y[1]; x[2] = y[2]; }
  };
  auto words = [](uint32_t (&v)[4], double t, uint32_t who, uint32_t flag) {
    v[0] = (uint32_t)__double2loint(t); v[1] = (uint32_t)__double2hiint(t); v[2] = who; v[3] = flag;
  };

  // ---- where the row, sorted by logit (equal ones by index), is cut: keys above key_cut stay, and of those equal to it
  //      the ones up to index_cut
  uint32_t key_cut = 0, index_cut = 0xFFFFFFFFu;
  if (cuts) {
    // The bin of the histograms in which the search ends: the one with the target-th token, or the one where the mass
    // reaches `target` (of_total: times the mass of all); beyond the histogram there are far_count tokens of far_mass, in
    // its last bin.  Each block adds up its share of the bins over the cluster.
    auto find = [&](bool mass_wanted, double target, bool of_total, uint32_t before, uint64_t before_mass, bool with_far) {
      const int per_block = SMP_BINS / (int)C, per = max(1, per_block / SMP_THREADS);
      uint32_t c[4]; uint64_t m[4];
      uint32_t c_sum = 0; uint64_t m_sum = 0;
      #pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[i] = 0; m[i] = 0;
        if (i >= per || tid * per >= per_block) continue;
        const int bin = (int)rank * per_block + tid * per + i;
        #pragma unroll 4
        for (uint32_t r = 0; r < C; ++r) {
          c[i] += *cluster.map_shared_rank(&sh.count[bin], r);
          if (by_mass) m[i] += join64(*cluster.map_shared_rank(&sh.mass_lo[bin], r), *cluster.map_shared_rank(&sh.mass_hi[bin], r));
        }
        c_sum += c[i]; m_sum += m[i];
      }
      uint32_t c_in = c_sum; uint64_t m_in = m_sum;               // inclusive sums over the threads
      #pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, c_in, d);
        const uint64_t y = __shfl_up_sync(0xFFFFFFFFu, m_in, d);
        if (lane >= d) { c_in += x; m_in += y; }
      }
      if (lane == 31) { sh.scan[warp][0] = c_in; sh.scan[warp][1] = (uint32_t)m_in; sh.scan[warp][2] = (uint32_t)(m_in >> 32); }
      __syncthreads();
      uint32_t total[3] = {0, 0, 0}, c_base = 0;
      uint64_t m_all = 0, m_base = 0;
      for (int w = 0; w < SMP_WARPS; ++w) {
        if (w == warp) { c_base = total[0]; m_base = m_all; }
        total[0] += sh.scan[w][0]; m_all += join64(sh.scan[w][1], sh.scan[w][2]);
      }
      total[1] = (uint32_t)m_all; total[2] = (uint32_t)(m_all >> 32);
      const uint32_t (*all)[8] = exchange(total, 3);
      uint32_t c_at = before + c_base + c_in - c_sum, c_end = before;
      uint64_t m_at = before_mass + m_base + m_in - m_sum, m_end = before_mass;
      for (uint32_t r = 0; r < C; ++r) {
        if (r == rank) { c_at += c_end - before; m_at += m_end - before_mass; }
        c_end += all[r][0]; m_end += join64(all[r][1], all[r][2]);
      }
      const uint32_t far_count = with_far ? (uint32_t)a.V - c_end : 0;
      const uint64_t far_mass = with_far ? (uint64_t)((double)__uint_as_float(sums[3]) * 1099511627776.0) : 0;
      if (of_total) target *= (double)(m_end + far_mass);
      #pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (c[i] > 0) {
          const bool here = mass_wanted ? (double)m_at < target && (double)(m_at + m[i]) >= target
                                        : (double)c_at < target && (double)(c_at + c[i]) >= target;
          if (here) {
            const Cut cut{(uint32_t)((int)rank * per_block + tid * per + i), c_at, c[i], (uint32_t)m[i], (uint32_t)(m[i] >> 32),
                          (uint32_t)m_at, (uint32_t)(m_at >> 32)};
            for (uint32_t r = 0; r < C; ++r) *cluster.map_shared_rank(&sh.cut, r) = cut;
          }
        }
        c_at += c[i]; m_at += m[i];
      }
      barrier();
      struct Found { Cut cut; double target; uint64_t total; } f{sh.cut, target, m_end + far_mass};
      if (mass_wanted ? (double)m_end < target : (double)c_end < target)
        f.cut = Cut{SMP_BINS - 1, c_end, far_count, (uint32_t)far_mass, (uint32_t)(far_mass >> 32), (uint32_t)m_end, (uint32_t)(m_end >> 32)};
      return f;
    };
    // The tokens that `take` picks (at most SMP_SORT in the cluster), in the first block, in order, one a thread (0: none).
    auto gather_sorted = [&](auto take, uint32_t many) -> uint64_t {
      SampleShared& first = *cluster.map_shared_rank(&sh, 0);
      for (int v = tid; v < n_vec; v += SMP_THREADS) {
        float z[8];
        Vec<T>::get(piece + 8 * v, z);
        #pragma unroll
        for (int i = 0; i < 8; ++i)
          if (take(z[i]) && 8 * v + i < n) {
            const uint32_t at = atomicAdd(&first.n_sort, 1u);
            if (at < SMP_SORT) first.sort[at] = ((uint64_t)order_key(z[i]) << 32) | (0xFFFFFFFFu - (begin + 8 * v + i));
          }
      }
      barrier();
      if (rank != 0) return 0;
      const uint32_t have = min(sh.n_sort, (uint32_t)SMP_SORT);
      uint64_t x = tid < (int)have ? sh.sort[tid] : 0;
      __syncthreads();
      if (tid == 0) sh.n_sort = 0;
      // bitonic, largest first; partners in other warps meet in shared memory
      for (uint32_t size = 2; (size >> 1) < many && size <= SMP_SORT; size <<= 1)
        for (uint32_t d = size >> 1; d > 0; d >>= 1) {
          uint64_t y;
          if (d >= 32) {
            sh.sort[tid] = x;
            __syncthreads();
            y = sh.sort[tid ^ d];
            __syncthreads();
          } else y = __shfl_xor_sync(0xFFFFFFFFu, x, d);
          const bool want_larger = ((tid & d) == 0) == ((tid & size) == 0);
          x = (x > y) == want_larger ? x : y;
        }
      return x;
    };
    // inclusive sum over the block's threads
    auto scan_mass = [&](uint64_t m) -> uint64_t {
      #pragma unroll
      for (int d = 1; d < 32; d <<= 1) { const uint64_t y = __shfl_up_sync(0xFFFFFFFFu, m, d); if (lane >= d) m += y; }
      if (lane == 31) { sh.scan[warp][0] = (uint32_t)m; sh.scan[warp][1] = (uint32_t)(m >> 32); }
      __syncthreads();
      for (int w = 0; w < warp; ++w) m += join64(sh.scan[w][0], sh.scan[w][1]);
      __syncthreads();
      return m;
    };
    auto mass_of = [&](uint64_t x) -> uint64_t { return x ? fixed_mass(ex2(-octaves(key_value((uint32_t)(x >> 32))))) : 0; };

    auto f = by_count ? find(false, (double)top_k, false, 0, 0, true) : find(true, (double)top_p, true, 0, 0, true);
    if (f.cut.before + f.cut.count <= SMP_SORT) {
      // ---- few tokens can stay: the first block sorts them, cuts by all three rules and runs the race
      const uint32_t many = f.cut.before + f.cut.count, bin = f.cut.bin;
      const uint64_t x = gather_sorted([&](float z) { return bin_of(octaves(z)) <= bin; }, many);
      if (rank != 0) return;
      bool in = x != 0 && (!by_count || tid < top_k);
      const float z = key_value((uint32_t)(x >> 32));
      if (by_mass) {
        const uint64_t m = in ? mass_of(x) : 0, incl = scan_mass(m);
        if (tid == SMP_THREADS - 1) { sh.scan[0][2] = (uint32_t)incl; sh.scan[0][3] = (uint32_t)(incl >> 32); }
        __syncthreads();
        const double target = by_count ? (double)top_p * (double)join64(sh.scan[0][2], sh.scan[0][3]) : f.target;
        in = in && (tid == 0 || (double)(incl - m) < target);
      }
      in = in && octaves(z) <= floor_octaves;
      uint32_t win[4];
      const uint32_t token = 0xFFFFFFFFu - (uint32_t)x;
      words(win, in ? finish(token, z) : CUDART_INF, in ? token : 0xFFFFFFFFu, __float_as_uint(0.f));
      #pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        uint32_t o[4];
        #pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __shfl_xor_sync(0xFFFFFFFFu, win[i], d);
        earlier(win, o);
      }
      uint32_t (*each)[4] = sh.warp[turn];
      __syncthreads();
      if (lane == 0)
        for (int i = 0; i < 4; ++i) each[warp][i] = win[i];
      __syncthreads();
      for (int w = 0; w < SMP_WARPS; ++w) earlier(win, each[w]);
      if (in && token == win[2]) { a.ids[row] = (int32_t)token; a.logp[row] = (z - zmax) - log_sum; }
      return;
    }
    // From a bin to the last token that stays.  Returns the mass of what stays.
    auto search = [&](const decltype(f)& found, bool mass_wanted) -> uint64_t {
      Cut cut = found.cut;
      const double target = found.target;
      if (cut.count <= SMP_SORT) {
        const uint64_t x = gather_sorted([&](float z) { return bin_of(octaves(z)) == cut.bin; }, cut.count);
        if (rank == 0) {
          const uint64_t before = join64(cut.before_lo, cut.before_hi), m = by_mass ? mass_of(x) : 0, incl = before + (by_mass ? scan_mass(m) : 0);
          const bool stays = x != 0 && (mass_wanted ? tid == 0 || (double)(incl - m) < target : tid < (int)(top_k - cut.before));
          const int last = __syncthreads_count(stays) - 1;
          if (tid == last) {
            const Last l{(uint32_t)(x >> 32), 0xFFFFFFFFu - (uint32_t)x, (uint32_t)incl, (uint32_t)(incl >> 32)};
            for (uint32_t r = 0; r < C; ++r) *cluster.map_shared_rank(&sh.last, r) = l;
          }
        }
        barrier();
        key_cut = sh.last.key; index_cut = sh.last.index;
        return join64(sh.last.kept_lo, sh.last.kept_hi);
      }
      // Many tokens in one bin: their range of keys is cut into bins again, until a single key is left.
      uint32_t key_low = 0, key_high = 0;
      for (int level = 0; level < 5; ++level) {      // 32 bits of key in steps of 11, and the look that finds one key
        uint32_t range[2] = {0xFFFFFFFFu, 0};
        for (int v = tid; v < n_vec; v += SMP_THREADS) {
          float z[8];
          Vec<T>::get(piece + 8 * v, z);
          #pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (8 * v + i >= n) break;
            const uint32_t key = order_key(z[i]);
            if (level == 0 ? bin_of(octaves(z[i])) == cut.bin : key >= key_low && key <= key_high) { range[0] = min(range[0], key); range[1] = max(range[1], key); }
          }
        }
        reduce(range, [](uint32_t* x, const uint32_t* y) { x[0] = min(x[0], y[0]); x[1] = max(x[1], y[1]); });
        key_low = range[0]; key_high = range[1];
        if (key_low >= key_high) break;
        int shift = 0;
        while (((key_high - key_low) >> shift) >= SMP_BINS) ++shift;
        for (int i = tid; i < SMP_BINS; i += SMP_THREADS) { sh.count[i] = 0; sh.mass_lo[i] = 0; sh.mass_hi[i] = 0; }
        __syncthreads();
        for (int v = tid; v < n_vec; v += SMP_THREADS) {
          float z[8];
          Vec<T>::get(piece + 8 * v, z);
          #pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (8 * v + i >= n) break;
            const uint32_t key = order_key(z[i]);
            if (key >= key_low && key <= key_high) into_bin((key_high - key) >> shift, octaves(z[i]));
          }
        }
        barrier();
        cut = find(mass_wanted, target, false, cut.before, join64(cut.before_lo, cut.before_hi), false).cut;
        if (cut.count == 0) {                        // the mass falls short of the target by rounding: all of them stay
          key_cut = key_low; index_cut = 0xFFFFFFFFu;
          return (uint64_t)target;
        }
        key_high -= cut.bin << shift;
        key_low = max(key_low, key_high - ((1u << shift) - 1));
      }
      // how many of the tokens with this key stay, and up to which index
      const uint64_t before = join64(cut.before_lo, cut.before_hi), mass = by_mass ? fixed_mass(ex2(-octaves(key_value(key_low)))) : 0;
      uint32_t stay = cut.count;
      if (!mass_wanted) stay = (uint32_t)target - cut.before;
      else if (mass > 0) stay = (uint32_t)fmin((double)cut.count, fmax(1.0, ceil((target - (double)before) / (double)mass)));
      key_cut = key_low; index_cut = 0xFFFFFFFFu;
      if (stay < cut.count) {
        // warps hold runs of eights in index order: tokens of this key a warp, then a block has
        const int per_warp = (n_vec + SMP_WARPS - 1) / SMP_WARPS, v0 = warp * per_warp, v1 = min(n_vec, v0 + per_warp);
        uint32_t mine = 0;
        for (int v = v0 + lane; v < v1; v += 32) {
          float z[8];
          Vec<T>::get(piece + 8 * v, z);
          #pragma unroll
          for (int i = 0; i < 8; ++i) mine += 8 * v + i < n && order_key(z[i]) == key_cut;
        }
        mine = __reduce_add_sync(0xFFFFFFFFu, mine);
        __syncthreads();
        if (lane == 0) sh.scan[warp][3] = mine;
        __syncthreads();
        uint32_t all_of_block = 0, at = 0;
        for (int w = 0; w < SMP_WARPS; ++w) { if (w == warp) at = all_of_block; all_of_block += sh.scan[w][3]; }
        const uint32_t (*all)[8] = exchange(&all_of_block, 1);
        for (uint32_t r = 0; r < rank; ++r) at += all[r][0];
        uint32_t who[1] = {0xFFFFFFFFu};
        if (at < stay && at + mine >= stay) {        // the last that stays is one of this warp's
          for (int v = v0; v < v1 && who[0] == 0xFFFFFFFFu; v += 32) {
            uint32_t bits = 0;
            if (v + lane < v1) {
              float z[8];
              Vec<T>::get(piece + 8 * (v + lane), z);
              #pragma unroll
              for (int i = 0; i < 8; ++i) bits |= (uint32_t)(8 * (v + lane) + i < n && order_key(z[i]) == key_cut) << i;
            }
            uint32_t in = __popc(bits);
            #pragma unroll
            for (int d = 1; d < 32; d <<= 1) { const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, in, d); if (lane >= d) in += x; }
            uint32_t at_lane = at + in - __popc(bits), mine_at = 0xFFFFFFFFu;
            for (int i = 0; i < 8; ++i)
              if ((bits >> i) & 1u) { if (++at_lane == stay) mine_at = begin + 8 * (v + lane) + i; }
            who[0] = __reduce_min_sync(0xFFFFFFFFu, mine_at);
            at += __shfl_sync(0xFFFFFFFFu, in, 31);
          }
        }
        reduce(who, [](uint32_t* x, const uint32_t* y) { x[0] = min(x[0], y[0]); });
        index_cut = who[0];
      }
      return before + mass * stay;
    };
    uint64_t stays = search(f, !by_count);
    if (by_count && by_mass) {
      if (f.cut.count > SMP_SORT) {                  // the histogram has been used for keys
        for (int i = tid; i < SMP_BINS; i += SMP_THREADS) { sh.count[i] = 0; sh.mass_lo[i] = 0; sh.mass_hi[i] = 0; }
        __syncthreads();
        for (int v = tid; v < n_vec; v += SMP_THREADS) {
          float z[8];
          Vec<T>::get(piece + 8 * v, z);
          #pragma unroll
          for (int i = 0; i < 8; ++i) { const float o = octaves(z[i]); if (o < (SMP_BINS - 1) / SMP_BINS_PER_OCTAVE) into_bin(bin_of(o), o); }
        }
        barrier();
      }
      const auto g = find(true, (double)top_p * (double)stays, false, 0, 0, true);
      stays = search(g, true);
    }
    weight = (float)((double)stays * 9.094947017729282e-13);      // 2^-40
    if (!by_mass || floor_octaves < CUDART_INF_F) {               // not known from the search, or min_p takes some out
      uint32_t w[1];
      float s = 0.f;
      for (int v = tid; v < n_vec; v += SMP_THREADS) {
        float z[8];
        Vec<T>::get(piece + 8 * v, z);
        #pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t key = order_key(z[i]);
          const float o = octaves(z[i]);
          if ((key > key_cut || (key == key_cut && begin + 8 * v + i <= index_cut)) && o <= floor_octaves) s += ex2(-o);
        }
      }
      w[0] = __float_as_uint(s);
      reduce(w, [&](uint32_t* x, const uint32_t* y) { add(x[0], y[0]); });
      weight = __uint_as_float(w[0]);
    }
  }

  // ---- the race
  auto kept = [&](float z, int i) {
    if (i >= n || octaves(z) > floor_octaves) return false;
    const uint32_t key = order_key(z);
    return key > key_cut || (key == key_cut && begin + i <= index_cut);
  };
  // candidates: upper 16 bits <= 65536 L w / weight (with room for the rounding of w and weight)
  const float reach = SMP_LEAD / weight;
  const float bound = 65536.f * reach * 1.001f;
  for (int v = tid; v < n_vec; v += SMP_THREADS) {
    float z[8];
    Vec<T>::get(piece + 8 * v, z);
    const uint4 r = philox4x32_10((begin >> 3) + v, 0, 0, 0, k0, k1);
    const uint32_t word[4] = {r.x, r.y, r.z, r.w};
    float lead = -1.f;
    #pragma unroll
    for (int i = 0; i < 8; ++i) {                   // 2^23 + bound w + 1 against 2^23 + the upper bits
      const float u = __uint_as_float(__byte_perm(word[i >> 1], 0x4B000000u, (i & 1) ? 0x7632 : 0x7610));
      lead = fmaxf(lead, fmaf(ex2((z[i] - zmax) * scale), bound, 8388609.f) - u);
    }
    if (lead >= 0.f) {
      #pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        const uint32_t w = i < 2 ? r.x : i < 4 ? r.y : i < 6 ? r.z : r.w, upper = (i & 1) ? w >> 16 : w & 0xFFFFu;
        const float zi = as_float(piece[8 * v + i]);
        if (!((float)upper <= fmaf(ex2(-octaves(zi)), bound, 2.f)) || !kept(zi, 8 * v + i)) continue;
        const uint32_t at = atomicAdd(&sh.n_list, 1u);
        if (at < SMP_LIST) sh.list[at] = 8 * v + i;
      }
    }
  }
  __syncthreads();
  uint32_t win[4] = {0, 0, 0, 0};
  double best = CUDART_INF;
  uint32_t who = 0xFFFFFFFFu;
  if (warp == 0) {                                 // the list is short: one warp works it out
    const uint32_t listed = sh.n_list;
    for (uint32_t j = lane; j < min(listed, (uint32_t)SMP_LIST); j += 32) {
      const uint32_t i = sh.list[j];
      const double t = finish(begin + i, as_float(piece[i]));
      if (t < best || (t == best && begin + i < who)) { best = t; who = begin + i; }
    }
    words(win, best, who, listed > SMP_LIST ? 1u : 0u);
    #pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      uint32_t o[4];
      #pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __shfl_xor_sync(0xFFFFFFFFu, win[i], d);
      earlier(win, o);
    }
  }
  {
    const uint32_t (*all)[8] = exchange(win, 4);
    for (int i = 0; i < 4; ++i) win[i] = all[0][i];
    for (uint32_t r = 1; r < C; ++r) earlier(win, all[r]);
  }
  if (win[3] || !(__hiloint2double((int)win[1], (int)win[0]) < 0.99 * (double)reach)) {       // the same in all blocks
    best = CUDART_INF; who = 0xFFFFFFFFu;
    #pragma unroll 1
    for (int v = tid; v < n_vec; v += SMP_THREADS)
      #pragma unroll 1
      for (int i = 8 * v; i < 8 * v + 8; ++i) {
        const float z = as_float(piece[i]);
        if (!kept(z, i)) continue;
        const double t = finish(begin + i, z);
        if (t < best) { best = t; who = begin + i; }
      }
    words(win, best, who, 0);
    reduce(win, earlier);
  }
  const int at = (int)(win[2] - begin);
  if (tid == 0 && win[2] >= begin && at < n) {             // the winner's block
    a.ids[row] = (int32_t)win[2];
    a.logp[row] = (as_float(piece[at]) - zmax) - log_sum;
  }
}

template <class T>
static int launch_sample(const SampleArgs& args, int sms, cudaStream_t st) {
  // A row is cut over as many blocks as leave an SM room for two of them (76 KB of logits each); a batch that would not
  // fill the device is cut finer, down to 2048 tokens a block.
  int C = 1;
  const auto piece_of = [&](int c) { return round_up<int64_t>(ceil_div<int64_t>(args.V, c), 8); };
  while (C < SMP_MAX_CLUSTER && piece_of(C) * (int64_t)sizeof(T) > 76 * 1024) C *= 2;
  while (C < SMP_MAX_CLUSTER && (int64_t)args.B * C * 2 <= 2 * sms && piece_of(C) > 2048) C *= 2;
  SampleArgs a = args;
  a.piece = (int32_t)piece_of(C);
  if (a.piece * sizeof(T) > SMP_MAX_PIECE) return SAPO_ERR_UNSUPPORTED_SHAPE;
  const size_t smem = ((sizeof(SampleShared) + 15) & ~size_t(15)) + a.piece * sizeof(T);
  static size_t allowed[MAX_DEVICES] = {0};
  const int dev = current_device();
  if (dev < 0) return SAPO_ERR_CUDA;
  if (allowed[dev] < smem) {
    const size_t most = ((sizeof(SampleShared) + 15) & ~size_t(15)) + SMP_MAX_PIECE;
    if (cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most) != cudaSuccess) return SAPO_ERR_CUDA;
    allowed[dev] = most;
  }
  KernelScope scope(SAPO_K_SAMPLE, st);
  return launch_overlapped(sample_kernel<T>, dim3((unsigned)(a.B * C)), SMP_THREADS, smem, C, st, a);
}

}  // namespace sapo

extern "C" int sapo_sample(const void* logits, int32_t dtype, int32_t B, int32_t V, int64_t ld, const int64_t* seeds,
                           const sapo_sample_cfg* h_cfg, int32_t* ids, float* logp, int32_t* status, void* stream) {
  using namespace sapo;
  if (!h_cfg || B < 0 || V < 1 || ld < 0 || !status) return SAPO_ERR_INVALID_ARG;
  if (dtype != SAPO_DTYPE_BF16 && dtype != SAPO_DTYPE_F32) return SAPO_ERR_INVALID_ARG;
  if (!h_cfg->temperature_rows && !(h_cfg->temperature >= 0.f && h_cfg->temperature <= 3.4e38f)) return SAPO_ERR_INVALID_ARG;
  if (!h_cfg->min_p_rows && !(h_cfg->min_p >= 0.f)) return SAPO_ERR_INVALID_ARG;
  if (!h_cfg->top_p_rows && h_cfg->top_p != h_cfg->top_p) return SAPO_ERR_INVALID_ARG;
  if (B == 0) return SAPO_OK;
  if (!logits || !seeds || !ids || !logp) return SAPO_ERR_INVALID_ARG;
  const size_t size = dtype == SAPO_DTYPE_BF16 ? 2 : 4;
  if ((int64_t)V * (int64_t)size > (int64_t)SMP_MAX_CLUSTER * (int64_t)SMP_MAX_PIECE - 64 * SMP_MAX_CLUSTER || B > (1 << 24)) return SAPO_ERR_UNSUPPORTED_SHAPE;
  if (reinterpret_cast<uintptr_t>(logits) % size) return SAPO_ERR_INVALID_ARG;
  const int sms = sm_count();
  if (sms <= 0) return SAPO_ERR_CUDA;
  const SampleArgs a{logits, ld, B, V, 0, seeds, h_cfg->temperature_rows, h_cfg->top_k_rows, h_cfg->top_p_rows, h_cfg->min_p_rows,
                     h_cfg->temperature, h_cfg->top_k, h_cfg->top_p, h_cfg->min_p, ids, logp, status};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return dtype == SAPO_DTYPE_BF16 ? launch_sample<__nv_bfloat16>(a, sms, st) : launch_sample<float>(a, sms, st);
}
