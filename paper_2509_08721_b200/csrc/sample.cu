// sapo_sample: draws one token of every row of logits, with temperature, top-k, top-p and min-p, from a 64-bit random
// number per row.
//
// The draw is a race of exponentials: token i with weight w_i = exp((z_i - zmax) / T) finishes at e_i / w_i, where e_i is
// a unit exponential made of 32 random bits of (the row's number, i); the first to finish wins, which token i does with
// probability w_i / sum w.  Against a search in the cumulated weights this needs no prefix sums along the vocabulary,
// splits over any number of blocks, and its outcome hangs on two numbers instead of on a long rounded sum.
//
// A cluster of 1 to 8 blocks holds a row in shared memory (it is read from HBM once) and walks over it there.  Only a token with
// e_i < L w_i / sum w can win unless nobody does that well (probability exp(-L)), and e_i >= n_i 2^-32, so the race
// compares the upper 16 random bits of a token (eight tokens share one call of the generator) with L w_i / sum w, and only the
// about L tokens that pass are worked out: in 32 bits, and where two come within a thousandth in 64.  Should none do
// well enough, the race goes over more of them.  So an id is the one that 64-bit arithmetic gives.
//
// race_kernel (no top-k, no top-p): every block for itself, one exchange at the end.  sample_kernel: top-k up to 256 from the
// threads' largest logits, sorted, which gives a logit that at least k tokens reach, and a sort of the few that do; else a
// histogram of 64 bins an octave of weight (counts and masses as integers: the same whatever the order of additions) to the bin
// in which the row is cut, and a sort of that bin's tokens.
//
// What bounds it: 512 x 151936 bf16 109 us (24 at the copy rate): instructions, 200 for eight tokens, of which the
// generator's 20 wide products occupy the multiplier 80 of 130 issue slots.  One row, top-k and top-p, 14 us: a chain of 6
// cluster barriers and the code's first fetch.  96 x 152064 fp32 with settings of their own 85 us: the same chain, of
// 9 barriers where only top-p is set, two blocks an SM.
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

constexpr int SMP_MAX_CLUSTER = 8;
constexpr int SMP_SORT = 512;                 // tokens that are sorted at once, one a thread
constexpr int SMP_BINS = 2048;
constexpr float SMP_BINS_PER_OCTAVE = 64.f;   // the last bin takes everything below 2^-32 of the largest weight
constexpr int SMP_LIST = 256;                 // candidates a block keeps
constexpr float SMP_LEAD = 16.f;              // L: no candidate wins with probability 1e-7
constexpr float SMP_LOG2E = 1.4426950408889634f;
constexpr size_t SMP_MAX_PIECE = 180 * 1024;  // bytes of a row a block can hold
constexpr int32_t SMP_MAX_TOKENS = (1 << 19) - 1;      // the sums of 13 bits of mass stay below 2^32
constexpr float SMP_TIE = 1.001f;             // times nearer than this are told apart in 64 bits
constexpr int SMP_THREADS = SMP_SORT;

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
  alignas(16) uint32_t slots[2][SMP_MAX_CLUSTER][4];    // what the blocks of the cluster tell one another; two sets, taken in turn
  uint32_t warp[2][32][4];
  uint32_t scan[32][4];
  uint32_t n_list, n_sort;
  uint32_t list[SMP_LIST];                  // candidates of the race
  Cut cut;
  Last last;
  uint64_t sort[SMP_SORT];                  // tokens to be put in order: key, and the index from above
  // of the tokens in a bin: their number, and the sums of the lower 13 and of the other bits of their mass_bits; once find() has
  // been over a bin, its mass in units of 2^-40
  alignas(16) uint32_t count[SMP_BINS];
  uint32_t mass_lo[SMP_BINS], mass_hi[SMP_BINS];
};
constexpr size_t SMP_SHARED = (sizeof(SampleShared) + 15) & ~size_t(15);

// order-preserving map of a float to an unsigned integer (both zeros are equal)
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }
// A weight 2^-o of the octave `oct` (o = oct + a fraction) as an integer of 26 bits, and such integers in units of 2^-40:
// sums of them do not depend on the order.
__device__ __forceinline__ uint32_t mass_bits(float o, uint32_t oct) {
  return __float2uint_rn(__uint_as_float(__float_as_uint(ex2(-o)) + (oct << 23)) * 67108864.f);
}
__device__ __forceinline__ uint64_t mass_units(uint64_t bits, uint32_t oct) { return oct <= 14 ? bits << (14 - oct) : bits >> (oct - 14); }
__device__ __forceinline__ void add_shared_if(bool yes, uint32_t* to, uint32_t x) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p red.shared.add.u32 [%0], %1;\n\t}"
               ::"r"(umma::smem_u32(to)), "r"(x), "r"((uint32_t)yes) : "memory");
}
// adds to the same place of another block's shared memory
__device__ __forceinline__ void add_remote(uint32_t* at, uint32_t block, uint32_t x) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(umma::map_to_cta(umma::smem_u32(at), block)), "r"(x) : "memory");
}
__device__ __forceinline__ uint64_t join64(uint32_t lo, uint32_t hi) { return ((uint64_t)hi << 32) | lo; }

// the 32 random bits of a token: the same 16 of two counters
__device__ __forceinline__ uint32_t random_bits(uint32_t token, uint32_t k0, uint32_t k1) {
  const uint32_t half = token & 7u, s = 16 * (half & 1u);
  uint32_t bits = 0;
  #pragma unroll 1
  for (uint32_t part = 0; part < 2; ++part) {
    const uint4 r = philox4x32_10(token >> 3, part, 0, 0, k0, k1);
    const uint32_t w = half < 2 ? r.x : half < 4 ? r.y : half < 6 ? r.z : r.w;
    bits = (bits << 16) | ((w >> s) & 0xFFFFu);
  }
  return bits;
}
// the time at which a token finishes, off by less than 1e-4 of itself
__device__ __forceinline__ float finish32(uint32_t bits, float octaves) {
  const float e = bits < 0x40000000u ? -log1pf(-((float)bits + 0.5f) * 2.3283064e-10f) : -logf(((float)~bits + 0.5f) * 2.3283064e-10f);
  return e * ex2(octaves);
}

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
  constexpr int THREADS = SMP_THREADS, WARPS = THREADS / 32;
  constexpr uint32_t ALL = 0xFFFFFFFFu;
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t C = cluster.num_blocks(), rank = cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  SampleShared& sh = *reinterpret_cast<SampleShared*>(smem_raw);
  T* piece = reinterpret_cast<T*>(smem_raw + SMP_SHARED);
  int turn = 0;

  auto barrier = [&]() { if (C > 1) { __syncwarp(); umma::cluster_sync_all(); } else __syncthreads(); };
  // Tell every block of the cluster W words (of the first threads, the same in each) and wait; returns those of all blocks.
  auto exchange = [&](const uint32_t* v, int W) -> const uint32_t (*)[4] {
    const int t = turn;
    turn ^= 1;
    if (tid < (int)C) {
      uint32_t* to = cluster.map_shared_rank(&sh.slots[t][rank][0], tid);
      for (int i = 0; i < W; ++i) to[i] = v[i];
    }
    barrier();
    return sh.slots[t];
  };
  // Combine the words of every thread of the block in its first warp; op(x, y) folds y into x.
  auto reduce_block = [&](auto& v, auto op) {
    constexpr int W = sizeof(v) / 4;
    auto fold = [&](int widest) {
      #pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        if (d > widest) continue;
        uint32_t o[W];
        #pragma unroll
        for (int i = 0; i < W; ++i) o[i] = __shfl_xor_sync(ALL, v[i], d);
        op(v, o);
      }
    };
    fold(16);
    uint32_t (*each)[4] = sh.warp[turn];
    if (lane == 0)
      for (int i = 0; i < W; ++i) each[warp][i] = v[i];
    __syncthreads();
    if (warp == 0) {
      for (int i = 0; i < W; ++i) v[i] = each[lane & (WARPS - 1)][i];
      fold(WARPS / 2);
    }
  };
  // The same over the cluster: all threads get the result.
  auto reduce = [&](auto& v, auto op) {
    constexpr int W = sizeof(v) / 4;
    reduce_block(v, op);
    const uint32_t (*all)[4] = exchange(v, W);
    for (int i = 0; i < W; ++i) v[i] = all[0][i];
    for (uint32_t r = 1; r < C; ++r) op(v, all[r]);
  };
  auto add = [](uint32_t& x, uint32_t y) { x = __float_as_uint(__uint_as_float(x) + __uint_as_float(y)); };
  auto larger = [](uint32_t* x, const uint32_t* y) { x[0] = __float_as_uint(max_nan(__uint_as_float(x[0]), __uint_as_float(y[0]))); };

  wait_for_previous();
  const int row = blockIdx.x / C;
  const uint32_t begin = rank * (uint32_t)a.piece;
  const int n = max(0, min(a.piece, a.V - (int)begin));       // tokens of this block
  const int n_vec = (n + 7) / 8;

  // ---- the row's piece into shared memory: a thread fetches the eights of tokens that it will look at
  {
    const T* from = static_cast<const T*>(a.z) + (int64_t)row * a.ld + begin;
    const bool aligned = (reinterpret_cast<uintptr_t>(from) & 15u) == 0;
    #pragma unroll 2
    for (int v = tid; v < n_vec; v += THREADS) {
      if (aligned && 8 * v + 8 <= n) {
        #pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                       ::"r"(umma::smem_u32(reinterpret_cast<uint8_t*>(piece + 8 * v) + 16 * h)),
                         "l"(reinterpret_cast<const uint8_t*>(from + 8 * v) + 16 * h) : "memory");
      } else {
        #pragma unroll 1
        for (int i = 8 * v; i < 8 * v + 8; ++i) piece[i] = i < n ? from[i] : T(-CUDART_INF_F);   // behind the end: no weight
      }
    }
  }
  const float temperature = a.temperature ? a.temperature[row] : a.temperature_all;
  const float min_p = a.min_p ? a.min_p[row] : a.min_p_all, top_p = a.top_p ? a.top_p[row] : a.top_p_all;
  int32_t top_k = a.top_k ? a.top_k[row] : a.top_k_all;
  if (top_k <= 0 || top_k >= a.V) top_k = 0;
  const uint64_t seed = (uint64_t)a.seeds[row];
  const uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
  const bool greedy = temperature == 0.f || top_k == 1 || top_p <= 0.f;
  const bool by_mass = top_p < 1.f && !greedy, by_count = top_k > 0 && !greedy, cuts = by_mass || by_count;
  if (cuts) {
    uint4* h = reinterpret_cast<uint4*>(sh.count);
    for (int i = tid; i < 3 * SMP_BINS / 4; i += THREADS) h[i] = make_uint4(0, 0, 0, 0);
  }
  if (tid == 0) { sh.n_list = 0; sh.n_sort = 0; }
  barrier();                                    // every block's shared memory is there before the first store to it
  asm volatile("cp.async.wait_all;" ::: "memory");

  // Values of the block's threads in order, largest first: bitonic; partners in other warps meet in shared memory.  Only
  // the first `many` threads have something else than 0.
  auto sorted = [&](auto x, uint32_t many) {
    auto* meet = reinterpret_cast<decltype(x)*>(sh.sort);
    #pragma unroll 1
    for (uint32_t size = 2; (size >> 1) < many && size <= (uint32_t)THREADS; size <<= 1)
      #pragma unroll 1
      for (uint32_t d = size >> 1; d > 0; d >>= 1) {
        auto y = x;
        if (d >= 32) {
          meet[tid] = x;
          __syncthreads();
          y = meet[tid ^ d];
          __syncthreads();
        } else y = __shfl_xor_sync(ALL, x, d);
        const bool want_larger = ((tid & d) == 0) == ((tid & size) == 0);
        x = (x > y) == want_larger ? x : y;
      }
    return x;
  };

  // ---- the largest logit: of the block, and of the row.  Without cuts and min_p the sums below are formed against the
  //      block's and told together with it.  With a small top_k: also a logit that at least top_k tokens reach, from the
  //      threads' largest ones: the larger of any block's k-th, and of the least of the blocks' (k / C)-th.
  const bool settings_ok = temperature >= 0.f && temperature < CUDART_INF_F && min_p >= 0.f && top_p == top_p;
  const bool alone = !cuts && settings_ok && !(min_p > 0.f);
  const bool few = by_count && top_k <= THREADS / 2;
  uint32_t top[1];
  float zmax, reached = -CUDART_INF_F;
  {
    float m = -CUDART_INF_F;
    for (int v = tid; v < n_vec; v += THREADS) m = max_nan(m, Vec<T>::most(piece + 8 * v));
    top[0] = __float_as_uint(m);
    if (alone) {
      reduce_block(top, larger);
      if (tid == 0) sh.scan[0][0] = top[0];
      __syncthreads();
      zmax = __uint_as_float(sh.scan[0][0]);
      top[0] = __float_as_uint(zmax);
    } else if (few) {
      const bool bad = __syncthreads_or(!(m < CUDART_INF_F));
      const uint32_t x = sorted(order_key(m), THREADS);
      if (tid == 0) sh.scan[0][0] = bad ? 0x7FFFFFFFu : __float_as_uint(key_value(x));            // (NaN)
      if (tid == top_k - 1) sh.scan[0][1] = __float_as_uint(key_value(x));
      if (tid == (top_k + (int)C - 1) / (int)C - 1) sh.scan[0][2] = __float_as_uint(key_value(x));
      __syncthreads();
      const uint32_t v[3] = {sh.scan[0][0], sh.scan[0][1], sh.scan[0][2]};
      const uint32_t (*all)[4] = exchange(v, 3);
      zmax = -CUDART_INF_F;
      float least = CUDART_INF_F;
      for (uint32_t r = 0; r < C; ++r) {
        zmax = max_nan(zmax, __uint_as_float(all[r][0]));
        reached = fmaxf(reached, __uint_as_float(all[r][1]));
        least = fminf(least, __uint_as_float(all[r][2]));
      }
      reached = fmaxf(reached, least);
    } else {
      reduce(top, larger);
      zmax = __uint_as_float(top[0]);
    }
  }
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
  // act(index in the piece, logit) for each token of this thread's that `take` picks; the few that are picked are gone through
  // in a loop, so that the code stays short: it is fetched once a call, which is most of what a single row takes
  auto for_each = [&](auto take, auto act) {
    #pragma unroll 1
    for (int v = tid; v < n_vec; v += THREADS) {
      float z[8];
      Vec<T>::get(piece + 8 * v, z);
      uint32_t picked = 0;
      #pragma unroll
      for (int i = 0; i < 8; ++i) picked |= (uint32_t)take(z[i]) << i;
      if (8 * v + 8 > n) picked &= (1u << (n - 8 * v)) - 1u;
      #pragma unroll 1
      for (; picked; picked &= picked - 1) {
        const int i = 8 * v + __ffs(picked) - 1;
        act(i, as_float(piece[i]));
      }
    }
  };
  // the weight of a token in units of 2^-40
  auto mass_of = [&](float z) -> uint64_t {
    const float o = octaves(z);
    const uint32_t oct = min(bin_of(o) >> 6, 31u);
    return o < 100.f ? mass_units(mass_bits(o, oct), oct) : 0;
  };
  // the octaves of the piece's tokens into bins, those of the last bin left out; returns the weight of these
  auto histogram = [&]() -> float {
    float far = 0.f;
    for (int v = tid; v < n_vec; v += THREADS) {
      float z[8];
      Vec<T>::get(piece + 8 * v, z);
      #pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float o = octaves(z[i]);
        const bool near = o < (SMP_BINS - 1) / SMP_BINS_PER_OCTAVE;      // (behind the row's end it is infinite)
        const uint32_t bin = bin_of(o);
        add_shared_if(near, &sh.count[bin], 1u);
        if (by_mass) {
          const uint32_t m = mass_bits(o, bin >> 6);
          add_shared_if(near, &sh.mass_lo[bin], m & 8191u);
          add_shared_if(near, &sh.mass_hi[bin], m >> 13);
          far += near ? 0.f : ex2(-o);
        }
      }
    }
    return far;
  };

  // an empty histogram, in all blocks
  auto clear = [&]() {
    uint4* h = reinterpret_cast<uint4*>(sh.count);
    for (int i = tid; i < 3 * SMP_BINS / 4; i += THREADS) h[i] = make_uint4(0, 0, 0, 0);
    barrier();
  };
  // Adds the block's histogram to the blocks that look after its bins (each to an equal share), but for its own share.  Done
  // once this block's own additions are, and complete at the next barrier of the cluster.
  auto share_histogram = [&]() {
    __syncthreads();
    const int per_block = SMP_BINS / (int)C;
    for (int i = tid; i < SMP_BINS; i += THREADS) {
      const uint32_t owner = (uint32_t)(i / per_block), c = sh.count[i];
      if (owner == rank || c == 0) continue;
      add_remote(&sh.count[i], owner, c);
      if (by_mass) { add_remote(&sh.mass_lo[i], owner, sh.mass_lo[i]); add_remote(&sh.mass_hi[i], owner, sh.mass_hi[i]); }
    }
  };

  // ---- sums of the weights at temperature 1 and at the row's, of the tokens that min_p keeps; the first token with the
  //      largest logit; for top-k and top-p a histogram of the octaves, without the tokens of its last bin
  uint32_t sums[4];
  {
    float2 s1 = both(0.f), sT = both(0.f);
    float far = 0.f;
    uint32_t first = ALL;
    // (a block of -inf, or with a NaN or +inf, has no largest logit to go by: its sums are 0, or the row is bad)
    const float ref = fabsf(zmax) < CUDART_INF_F ? zmax : 0.f;
    const bool other = !greedy && !cuts && (scale != SMP_LOG2E || floor_octaves < CUDART_INF_F);
    for (int v = tid; v < n_vec; v += THREADS) {
      float z[8];
      Vec<T>::get(piece + 8 * v, z);
      #pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 x = mul2(add2(make_float2(z[2 * i], z[2 * i + 1]), both(-ref)), both(SMP_LOG2E));
        s1 = add2(s1, make_float2(ex2(x.x), ex2(x.y)));
      }
    }
    if (cuts) {
      if (!few) { far = histogram(); share_histogram(); }
    } else if (other) {
      for (int v = tid; v < n_vec; v += THREADS) {
        float z[8];
        Vec<T>::get(piece + 8 * v, z);
        #pragma unroll
        for (int i = 0; i < 8; ++i) { const float o = (ref - z[i]) * scale; sT.x += o <= floor_octaves ? ex2(-o) : 0.f; }
      }
    } else if (greedy) {
      for_each([&](float z) { return z == zmax; }, [&](int i, float) { first = min(first, begin + i); });
    }
    sums[0] = __float_as_uint(s1.x + s1.y); sums[1] = other ? __float_as_uint(sT.x) : sums[0]; sums[2] = first; sums[3] = __float_as_uint(far);
    if (alone) {
      // words of a block: its sums against its largest logit, its first token with it, that logit
      reduce_block(sums, [&](uint32_t* x, const uint32_t* y) { add(x[0], y[0]); add(x[1], y[1]); x[2] = min(x[2], y[2]); });
      if (!other) sums[1] = sums[0];
      sums[3] = top[0];
      const uint32_t (*all)[4] = exchange(sums, 4);
      zmax = -CUDART_INF_F;
      for (uint32_t r = 0; r < C; ++r) zmax = max_nan(zmax, __uint_as_float(all[r][3]));
      if (bad_row()) return;
      float u1 = 0.f, uT = 0.f;
      first = ALL;
      for (uint32_t r = 0; r < C; ++r) {
        const float less = zmax - __uint_as_float(all[r][3]);
        u1 += __uint_as_float(all[r][0]) * ex2(-less * SMP_LOG2E);
        uT += __uint_as_float(all[r][1]) * ex2(-less * scale);
        if (less == 0.f) first = min(first, all[r][2]);
      }
      sums[0] = __float_as_uint(u1); sums[1] = __float_as_uint(uT); sums[2] = first;
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
  // The time at which a token finishes: in 64 bits, and in 32.
  auto finish = [&](uint32_t token, float z) -> double {
    const double e = -log1p(-((double)random_bits(token, k0, k1) + 0.5) * 2.3283064365386963e-10);
    return e * exp(((double)zmax - (double)z) * fmin(1.0 / (double)temperature, 1e30));
  };
  auto finish_near = [&](uint32_t token, float z) -> float { return finish32(random_bits(token, k0, k1), octaves(z)); };
  // The first to finish, and how near the second comes: words first time, its token, second time, a flag.
  auto two_first = [](uint32_t* x, const uint32_t* y) {
    const float a1 = __uint_as_float(x[0]), b1 = __uint_as_float(y[0]), a2 = __uint_as_float(x[2]), b2 = __uint_as_float(y[2]);
    x[2] = __float_as_uint(fminf(fmaxf(a1, b1), fminf(a2, b2)));
    if (b1 < a1) { x[0] = y[0]; x[1] = y[1]; }
    x[3] |= y[3];
  };
  // the first in 64 bits, the lower index where two finish together; words: time, index, a flag
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
  uint32_t key_cut = 0, index_cut = ALL;
  if (cuts) {
    // The bin of the histogram in which the search ends: the one with the target-th token, or the one where the mass
    // reaches `target` (of_total: times the mass of all).  octave < 0: a histogram of the octaves, beyond which there are
    // the tokens of its last bin; else one of keys, of tokens of that octave.  Each block looks through its share of the bins.
    struct Found { Cut cut; double target; };
    auto find = [&](bool mass_wanted, double target, bool of_total, uint32_t before, uint64_t before_mass, int octave) -> Found {
      const bool with_far = octave < 0;
      const int per_block = SMP_BINS / (int)C, per = max(1, per_block / THREADS), bin0 = (int)rank * per_block + tid * per;
      uint32_t c_sum = 0; uint64_t m_sum = 0;
      if (tid * per < per_block)
        #pragma unroll 1
        for (int i = bin0; i < bin0 + per; ++i) {
          const uint32_t lo = sh.mass_lo[i], hi = sh.mass_hi[i];
          const uint64_t m = mass_units(((uint64_t)hi << 13) + lo, with_far ? (uint32_t)i >> 6 : (uint32_t)octave);
          sh.mass_lo[i] = (uint32_t)m; sh.mass_hi[i] = (uint32_t)(m >> 32);
          c_sum += sh.count[i]; m_sum += m;
        }
      uint32_t c_in = c_sum; uint64_t m_in = m_sum;               // inclusive sums over the threads
      #pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t x = __shfl_up_sync(ALL, c_in, d);
        const uint64_t y = __shfl_up_sync(ALL, m_in, d);
        if (lane >= d) { c_in += x; m_in += y; }
      }
      if (lane == 31) { sh.scan[warp][0] = c_in; sh.scan[warp][1] = (uint32_t)m_in; sh.scan[warp][2] = (uint32_t)(m_in >> 32); }
      __syncthreads();
      uint32_t total[3] = {0, 0, 0}, c_base = 0;
      uint64_t m_all = 0, m_base = 0;
      #pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        if (w == warp) { c_base = total[0]; m_base = m_all; }
        const uint4 x = *reinterpret_cast<const uint4*>(sh.scan[w]);
        total[0] += x.x; m_all += join64(x.y, x.z);
      }
      total[1] = (uint32_t)m_all; total[2] = (uint32_t)(m_all >> 32);
      const uint32_t (*all)[4] = exchange(total, 3);
      uint32_t c_at = before + c_base + c_in - c_sum, c_end = before;
      uint64_t m_at = before_mass + m_base + m_in - m_sum, m_end = before_mass;
      #pragma unroll
      for (uint32_t r = 0; r < SMP_MAX_CLUSTER; ++r) {
        if (r >= C) break;
        if (r == rank) { c_at += c_end - before; m_at += m_end - before_mass; }
        const uint4 x = *reinterpret_cast<const uint4*>(all[r]);
        c_end += x.x; m_end += join64(x.y, x.z);
      }
      const uint32_t far_count = with_far ? (uint32_t)a.V - c_end : 0;
      const uint64_t far_mass = with_far ? (uint64_t)((double)__uint_as_float(sums[3]) * 1099511627776.0) : 0;
      if (of_total) target *= (double)(m_end + far_mass);
      const Cut beyond{SMP_BINS - 1, c_end, far_count, (uint32_t)far_mass, (uint32_t)(far_mass >> 32), (uint32_t)m_end, (uint32_t)(m_end >> 32)};
      if (mass_wanted ? (double)m_end < target : (double)c_end < target) {       // the same in all blocks
        barrier();
        return Found{beyond, target};
      }
      // the thread whose bins hold it
      if (c_sum > 0 && (mass_wanted ? (double)m_at < target && (double)(m_at + m_sum) >= target : (double)c_at < target && (double)(c_at + c_sum) >= target)) {
        int i = bin0;
        for (;; ++i) {
          const uint32_t c = sh.count[i]; const uint64_t m = join64(sh.mass_lo[i], sh.mass_hi[i]);
          if (i == bin0 + per - 1 || (c > 0 && (mass_wanted ? (double)(m_at + m) >= target : (double)(c_at + c) >= target))) break;
          c_at += c; m_at += m;
        }
        const Cut cut{(uint32_t)i, c_at, sh.count[i], sh.mass_lo[i], sh.mass_hi[i], (uint32_t)m_at, (uint32_t)(m_at >> 32)};
        #pragma unroll 1
        for (uint32_t r = 0; r < C; ++r) *cluster.map_shared_rank(&sh.cut, r) = cut;
      }
      barrier();
      return Found{sh.cut, target};
    };
    // The tokens that `take` picks, if there are at most SMP_SORT in the cluster: in the first block, in order, one a
    // thread (0: none).  Returns how many there are.
    auto gather_sorted = [&](auto take, uint64_t& x) -> uint32_t {
      if (tid == 0) sh.n_sort = 0;
      __syncthreads();
      for_each(take, [&](int i, float z) {
        const uint32_t at = atomicAdd(&sh.n_sort, 1u);
        if (at < SMP_SORT) sh.sort[at] = ((uint64_t)order_key(z) << 32) | (ALL - (begin + i));
      });
      __syncthreads();
      const uint32_t mine = sh.n_sort, which = min(mine, (uint32_t)SMP_SORT);
      const uint64_t own = tid < (int)which ? sh.sort[tid] : 0;
      const uint32_t (*all)[4] = exchange(&mine, 1);
      uint32_t before = 0, many = 0;
      for (uint32_t r = 0; r < C; ++r) { if (r == rank) before = many; many += all[r][0]; }
      x = 0;
      if (many > SMP_SORT) return many;                    // the same in all blocks
      if (tid < (int)which) *cluster.map_shared_rank(&sh.sort[before + tid], 0) = own;
      barrier();
      if (rank != 0) return many;
      if (tid < (int)many) x = sh.sort[tid];
      __syncthreads();
      x = sorted(x, many);
      return many;
    };
    // inclusive sum over the block's threads
    auto scan_mass = [&](uint64_t m) -> uint64_t {
      #pragma unroll
      for (int d = 1; d < 32; d <<= 1) { const uint64_t y = __shfl_up_sync(ALL, m, d); if (lane >= d) m += y; }
      if (lane == 31) { sh.scan[warp][0] = (uint32_t)m; sh.scan[warp][1] = (uint32_t)(m >> 32); }
      __syncthreads();
      #pragma unroll 1
      for (int w = 0; w < warp; ++w) m += join64(sh.scan[w][0], sh.scan[w][1]);
      __syncthreads();
      return m;
    };

    // ---- few tokens can stay: the first block sorts them, cuts by all three rules and runs the race
    auto among_few = [&](uint64_t x, double mass_target) {
      bool in = x != 0 && (!by_count || tid < top_k);
      const float z = key_value((uint32_t)(x >> 32));
      if (by_mass) {
        const uint64_t m = in ? mass_of(z) : 0, incl = scan_mass(m);
        if (tid == THREADS - 1) { sh.scan[0][2] = (uint32_t)incl; sh.scan[0][3] = (uint32_t)(incl >> 32); }
        __syncthreads();
        if (by_count) mass_target = (double)top_p * (double)join64(sh.scan[0][2], sh.scan[0][3]);
        in = in && (tid == 0 || (double)(incl - m) < mass_target);
      }
      in = in && octaves(z) <= floor_octaves;
      const uint32_t token = ALL - (uint32_t)x;
      uint32_t win[4] = {__float_as_uint(CUDART_INF_F), ALL, __float_as_uint(CUDART_INF_F), 0u};
      if (in) { win[0] = __float_as_uint(finish_near(token, z)); win[1] = token; }
      const float mine = __uint_as_float(win[0]);
      reduce_block(win, two_first);
      if (tid == 0) { sh.scan[0][0] = win[0]; sh.scan[0][1] = win[1]; sh.scan[0][2] = win[2]; }
      __syncthreads();
      uint32_t who = sh.scan[0][1];
      const float first = __uint_as_float(sh.scan[0][0]);
      if (__uint_as_float(sh.scan[0][2]) <= first * SMP_TIE || !(first < 1e37f)) {       // the same for all threads
        uint32_t v[4];
        words(v, CUDART_INF, ALL, 0u);
        if (in && (mine <= first * SMP_TIE || !(first < 1e37f))) words(v, finish(token, z), token, 0u);
        reduce_block(v, earlier);
        if (tid == 0) sh.scan[0][0] = v[2];
        __syncthreads();
        who = sh.scan[0][0];
      }
      if (in && token == who) { a.ids[row] = (int32_t)token; a.logp[row] = (z - zmax) - log_sum; }
    };
    if (few) {
      uint64_t x;
      const uint32_t many = gather_sorted([&](float z) { return z >= reached; }, x);
      if (many <= SMP_SORT) {
        if (rank == 0) among_few(x, 0.0);
        return;
      }
      sums[3] = __float_as_uint(histogram());                  // (too many equal ones): as with a large top_k
      share_histogram();
      sums[0] = sums[1] = sums[2] = 0;
      reduce(sums, [&](uint32_t* p, const uint32_t* q) { add(p[3], q[3]); });
    }
    const Found f = find(!by_count, by_count ? (double)top_k : (double)top_p, !by_count, 0, 0, -1);
    if (f.cut.before + f.cut.count <= SMP_SORT) {
      const uint32_t bin = f.cut.bin;
      uint64_t x;
      gather_sorted([&](float z) { return bin_of(octaves(z)) <= bin; }, x);
      if (rank == 0) among_few(x, f.target);
      return;
    }
    // From a bin to the last token that stays.  Returns the mass of what stays.
    auto search = [&](const Found& found, bool mass_wanted) -> uint64_t {
      Cut cut = found.cut;
      const double target = found.target;
      if (cut.count <= SMP_SORT) {
        uint64_t x;
        gather_sorted([&](float z) { return bin_of(octaves(z)) == cut.bin; }, x);
        if (rank == 0) {
          const uint64_t before = join64(cut.before_lo, cut.before_hi), m = by_mass && x != 0 ? mass_of(key_value((uint32_t)(x >> 32))) : 0;
          const uint64_t incl = before + (by_mass ? scan_mass(m) : 0);
          const bool stays = x != 0 && (mass_wanted ? tid == 0 || (double)(incl - m) < target : tid < (int)(top_k - cut.before));
          const int last = __syncthreads_count(stays) - 1;
          if (tid == last) {
            const Last l{(uint32_t)(x >> 32), ALL - (uint32_t)x, (uint32_t)incl, (uint32_t)(incl >> 32)};
            for (uint32_t r = 0; r < C; ++r) *cluster.map_shared_rank(&sh.last, r) = l;
          }
        }
        barrier();
        key_cut = sh.last.key; index_cut = sh.last.index;
        return join64(sh.last.kept_lo, sh.last.kept_hi);
      }
      // Many tokens in one bin: their range of keys is cut into bins again, until a single key is left.
      const uint32_t oct = cut.bin >> 6;
      uint32_t key_low = 0, key_high = 0;
      #pragma unroll 1
      for (int level = 0; level < 5; ++level) {      // 32 bits of key in steps of 11, and the look that finds one key
        auto inside = [&](float z) { return level == 0 ? bin_of(octaves(z)) == cut.bin : order_key(z) >= key_low && order_key(z) <= key_high; };
        uint32_t range[2] = {ALL, 0};
        for_each(inside, [&](int, float z) { range[0] = min(range[0], order_key(z)); range[1] = max(range[1], order_key(z)); });
        reduce(range, [](uint32_t* x, const uint32_t* y) { x[0] = min(x[0], y[0]); x[1] = max(x[1], y[1]); });
        key_low = range[0]; key_high = range[1];
        if (key_low >= key_high) break;
        int shift = 0;
        while (((key_high - key_low) >> shift) >= SMP_BINS) ++shift;
        clear();
        for_each([&](float z) { return order_key(z) >= key_low && order_key(z) <= key_high; },
                 [&](int, float z) {
                   const uint32_t bin = (key_high - order_key(z)) >> shift;
                   atomicAdd(&sh.count[bin], 1u);
                   if (!by_mass) return;
                   const uint32_t m = mass_bits(octaves(z), oct);      // (the tokens of one bin are of one octave)
                   atomicAdd(&sh.mass_lo[bin], m & 8191u);
                   atomicAdd(&sh.mass_hi[bin], m >> 13);
                 });
        share_histogram();
        barrier();
        cut = find(mass_wanted, target, false, cut.before, join64(cut.before_lo, cut.before_hi), (int)oct).cut;
        if (cut.count == 0) {                        // the mass falls short of the target by rounding: all of them stay
          key_cut = key_low; index_cut = ALL;
          return (uint64_t)target;
        }
        key_high -= cut.bin << shift;
        key_low = max(key_low, key_high - ((1u << shift) - 1));
      }
      // how many of the tokens with this key stay, and up to which index
      const uint64_t before = join64(cut.before_lo, cut.before_hi), mass = by_mass ? mass_of(key_value(key_low)) : 0;
      uint32_t stay = cut.count;
      if (!mass_wanted) stay = (uint32_t)target - cut.before;
      else if (mass > 0) stay = (uint32_t)fmin((double)cut.count, fmax(1.0, ceil((target - (double)before) / (double)mass)));
      key_cut = key_low; index_cut = ALL;
      if (stay < cut.count) {
        // warps hold runs of eights in index order: tokens of this key a warp, then a block has
        const int per_warp = (n_vec + WARPS - 1) / WARPS, v0 = warp * per_warp, v1 = min(n_vec, v0 + per_warp);
        auto bits_of = [&](int v) -> uint32_t {
          uint32_t bits = 0;
          if (v < v1) {
            float z[8];
            Vec<T>::get(piece + 8 * v, z);
            #pragma unroll
            for (int i = 0; i < 8; ++i) bits |= (uint32_t)(8 * v + i < n && order_key(z[i]) == key_cut) << i;
          }
          return bits;
        };
        uint32_t mine = 0;
        #pragma unroll 1
        for (int v = v0 + lane; v < v1; v += 32) mine += __popc(bits_of(v));
        mine = __reduce_add_sync(ALL, mine);
        __syncthreads();
        if (lane == 0) sh.scan[warp][3] = mine;
        __syncthreads();
        uint32_t all_of_block = 0, at = 0;
        for (int w = 0; w < WARPS; ++w) { if (w == warp) at = all_of_block; all_of_block += sh.scan[w][3]; }
        const uint32_t (*all)[4] = exchange(&all_of_block, 1);
        for (uint32_t r = 0; r < rank; ++r) at += all[r][0];
        uint32_t who[1] = {ALL};
        if (at < stay && at + mine >= stay) {        // the last that stays is one of this warp's
          #pragma unroll 1
          for (int v = v0; v < v1 && who[0] == ALL; v += 32) {
            const uint32_t bits = bits_of(v + lane);
            uint32_t in = __popc(bits);
            #pragma unroll
            for (int d = 1; d < 32; d <<= 1) { const uint32_t x = __shfl_up_sync(ALL, in, d); if (lane >= d) in += x; }
            uint32_t at_lane = at + in - __popc(bits), mine_at = ALL;
            for (int i = 0; i < 8; ++i)
              if ((bits >> i) & 1u) { if (++at_lane == stay) mine_at = begin + 8 * (v + lane) + i; }
            who[0] = __reduce_min_sync(ALL, mine_at);
            at += __shfl_sync(ALL, in, 31);
          }
        }
        reduce(who, [](uint32_t* x, const uint32_t* y) { x[0] = min(x[0], y[0]); });
        index_cut = who[0];
      }
      return before + mass * stay;
    };
    uint64_t stays = search(f, !by_count);
    if (by_count && by_mass) {
      clear();
      sums[3] = __float_as_uint(histogram());
      share_histogram();
      sums[0] = sums[1] = sums[2] = 0;
      reduce(sums, [&](uint32_t* p, const uint32_t* q) { add(p[3], q[3]); });
      stays = search(find(true, (double)top_p * (double)stays, false, 0, 0, -1), true);
    }
    weight = (float)((double)stays * 9.094947017729282e-13);      // 2^-40
    if (!by_mass || floor_octaves < CUDART_INF_F) {               // not known from the search, or min_p takes some out
      uint32_t w[1];
      float s = 0.f;
      for_each([&](float z) { return order_key(z) >= key_cut && octaves(z) <= floor_octaves; },
               [&](int i, float z) { if (order_key(z) > key_cut || begin + i <= index_cut) s += ex2(-octaves(z)); });
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
  for (int v = tid; v < n_vec; v += THREADS) {
    float z[8];
    Vec<T>::get(piece + 8 * v, z);
    const uint4 r = philox4x32_10((begin >> 3) + v, 0, 0, 0, k0, k1);
    const uint32_t word[4] = {r.x, r.y, r.z, r.w};
    float lead[2] = {-1.f, -1.f};
    #pragma unroll
    for (int i = 0; i < 4; ++i) {                 // 2^23 + 1 + bound w against 2^23 + the upper bits
      const float2 x = mul2(add2(make_float2(z[2 * i], z[2 * i + 1]), both(-zmax)), both(scale));
      const float2 may = fma2(make_float2(ex2(x.x), ex2(x.y)), both(bound), both(8388609.f));
      lead[0] = fmaxf(lead[0], may.x - __uint_as_float(__byte_perm(word[i], 0x4B000000u, 0x7610)));
      lead[1] = fmaxf(lead[1], may.y - __uint_as_float(__byte_perm(word[i], 0x4B000000u, 0x7632)));
    }
    if (fmaxf(lead[0], lead[1]) >= 0.f) {
      #pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        const uint32_t w = i < 2 ? r.x : i < 4 ? r.y : i < 6 ? r.z : r.w, upper = (i & 1) ? w >> 16 : w & 0xFFFFu;
        const float zi = as_float(piece[8 * v + i]);
        if (!((float)upper <= fmaf(ex2(-octaves(zi)), bound * 1.001f, 2.f)) || !kept(zi, 8 * v + i)) continue;
        const uint32_t at = atomicAdd(&sh.n_list, 1u);
        if (at < SMP_LIST) sh.list[at] = 8 * v + i;
      }
    }
  }
  __syncthreads();
  uint32_t win[4] = {__float_as_uint(CUDART_INF_F), ALL, __float_as_uint(CUDART_INF_F), 0u};
  const uint32_t listed = sh.n_list;
  if (warp == 0) {                                 // the list is short: one warp works it out
    #pragma unroll 1
    for (uint32_t j = lane; j < min(listed, (uint32_t)SMP_LIST); j += 32) {
      const uint32_t i = sh.list[j], o[4] = {__float_as_uint(finish_near(begin + i, as_float(piece[i]))), begin + i, __float_as_uint(CUDART_INF_F), 0u};
      two_first(win, o);
    }
    win[3] = listed > SMP_LIST ? 1u : 0u;
    #pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      uint32_t o[4];
      #pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __shfl_xor_sync(ALL, win[i], d);
      two_first(win, o);
    }
  }
  {
    const uint32_t (*all)[4] = exchange(win, 4);
    for (int i = 0; i < 4; ++i) win[i] = all[0][i];
    for (uint32_t r = 1; r < C; ++r) two_first(win, all[r]);
  }
  uint32_t winner = win[1];
  const float first = __uint_as_float(win[0]);
  const bool sure = !win[3] && first < 0.99f * reach;            // nobody outside the lists is earlier
  if (!sure || __uint_as_float(win[2]) <= first * SMP_TIE) {         // the same in all blocks
    double best = CUDART_INF;
    uint32_t who = ALL;
    auto look = [&](int i) {
      const double t = finish(begin + i, as_float(piece[i]));
      if (t < best || (t == best && begin + i < who)) { best = t; who = begin + i; }
    };
    if (sure) { if (tid < (int)listed) look((int)sh.list[tid]); }
    else
      #pragma unroll 1
      for (int v = tid; v < n_vec; v += THREADS)
        #pragma unroll 1
        for (int i = 8 * v; i < 8 * v + 8; ++i) if (kept(as_float(piece[i]), i)) look(i);
    uint32_t v[4];
    words(v, best, best < CUDART_INF ? who : ALL, 0u);
    reduce(v, earlier);
    winner = v[2];
  }
  const int at = (int)(winner - begin);
  if (tid == 0 && winner >= begin && at < n) {             // the winner's block
    a.ids[row] = (int32_t)winner;
    a.logp[row] = (as_float(piece[at]) - zmax) - log_sum;
  }
}

// ---------------------------------------------------------------------------- rows without top-k and top-p
// Every block of a row runs the race of its own tokens against its own largest logit and weight, and ends with its first
// to finish; the first block of the cluster compares the blocks' times.  Until then they do not wait for one another
// (but for the row's largest logit, with min_p), and the others are gone before it does.
// (five blocks of 256 an SM, 512 x 151936 bf16: 109 us; four 118; of 128 or 160 threads 107, but a single row 11.6 us instead of 10.5)
constexpr int RACE_THREADS = 256, RACE_WARPS = RACE_THREADS / 32;
constexpr float RACE_LEAD = 6.f;      // (16: three times as many candidates, 125 us instead of 118; 4: 120)

struct RaceShared {
  uint32_t slots[SMP_MAX_CLUSTER][4];       // of a block: its largest logit, its sum of weights, its first time, its token
  float max_of[SMP_MAX_CLUSTER];
  float warp[2][RACE_WARPS];
  uint32_t first[RACE_WARPS];
  double best; uint32_t who, n_list;
  uint32_t list[SMP_LIST];
};
constexpr size_t RACE_SHARED = (sizeof(RaceShared) + 15) & ~size_t(15);

__device__ __forceinline__ void store_weights(float* p, const float2 (&w)[4]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(w[0].x, w[0].y, w[1].x, w[1].y);
  reinterpret_cast<float4*>(p)[1] = make_float4(w[2].x, w[2].y, w[3].x, w[3].y);
}
__device__ __forceinline__ void store_weights(__nv_bfloat16* p, const float2 (&w)[4]) {
  uint32_t q[4];
  #pragma unroll
  for (int i = 0; i < 4; ++i) { const __nv_bfloat162 b = __floats2bfloat162_rn(w[i].x, w[i].y); q[i] = *reinterpret_cast<const uint32_t*>(&b); }
  *reinterpret_cast<uint4*>(p) = make_uint4(q[0], q[1], q[2], q[3]);
}

template <class T>
__global__ void __launch_bounds__(RACE_THREADS, 5) race_kernel(const SampleArgs a) {
  constexpr uint32_t ALL = 0xFFFFFFFFu;
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t C = cluster.num_blocks(), rank = cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  RaceShared& sh = *reinterpret_cast<RaceShared*>(smem_raw);
  T* piece = reinterpret_cast<T*>(smem_raw + RACE_SHARED);
  auto arrive = []() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); };
  auto wait = []() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); };

  arrive();                            // (waited for before the first store to another block's shared memory)
  wait_for_previous();
  const int row = blockIdx.x / C;
  const uint32_t begin = rank * (uint32_t)a.piece;
  const int n = max(0, min(a.piece, a.V - (int)begin)), n_vec = (n + 7) / 8;      // tokens of this block, and eights of them
  const T* from = static_cast<const T*>(a.z) + (int64_t)row * a.ld + begin;
  {
    const bool aligned = (reinterpret_cast<uintptr_t>(from) & 15u) == 0;
    #pragma unroll 2
    for (int v = tid; v < n_vec; v += RACE_THREADS) {
      if (aligned && 8 * v + 8 <= n) {
        #pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                       ::"r"(umma::smem_u32(reinterpret_cast<uint8_t*>(piece + 8 * v) + 16 * h)),
                         "l"(reinterpret_cast<const uint8_t*>(from + 8 * v) + 16 * h) : "memory");
      } else {
        #pragma unroll 1
        for (int i = 8 * v; i < 8 * v + 8; ++i) piece[i] = i < n ? from[i] : T(-CUDART_INF_F);   // behind the end: no weight
      }
    }
  }
  const float temperature = a.temperature ? a.temperature[row] : a.temperature_all, min_p = a.min_p ? a.min_p[row] : a.min_p_all;
  const uint64_t seed = (uint64_t)a.seeds[row];
  const uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
  const bool greedy = temperature == 0.f || a.top_k_all == 1;
  const bool settings_ok = temperature >= 0.f && temperature < CUDART_INF_F && min_p >= 0.f;
  const float scale = greedy ? SMP_LOG2E : fminf(SMP_LOG2E / temperature, 1e30f);
  if (tid == 0) sh.n_list = 0;
  asm volatile("cp.async.wait_all;" ::: "memory");

  // ---- the largest logit
  float zmax = -CUDART_INF_F;
  for (int v = tid; v < n_vec; v += RACE_THREADS) zmax = max_nan(zmax, Vec<T>::most(piece + 8 * v));
  #pragma unroll
  for (int d = 16; d > 0; d >>= 1) zmax = max_nan(zmax, __shfl_xor_sync(ALL, zmax, d));
  if (lane == 0) sh.warp[0][warp] = zmax;
  __syncthreads();
  #pragma unroll
  for (int w = 0; w < RACE_WARPS; ++w) zmax = max_nan(zmax, sh.warp[0][w]);
  bool waited = false;
  float floor_octaves = CUDART_INF_F;
  if (min_p > 0.f && !greedy) {                    // min_p goes by the row's largest
    __syncwarp();
    wait();
    waited = true;
    if (tid < (int)C) *cluster.map_shared_rank(&sh.max_of[rank], tid) = zmax;
    __syncwarp();
    umma::cluster_sync_all();
    for (uint32_t r = 0; r < C; ++r) zmax = max_nan(zmax, sh.max_of[r]);
    floor_octaves = fmaxf(-log2f(min_p), 0.f);
  }
  const bool usable = fabsf(zmax) < CUDART_INF_F;  // (a block of -inf, or with a NaN or +inf, has nothing in the race)
  const float ref = usable ? zmax : 0.f;
  uint32_t first = ALL;               // greedy: the first token with the largest logit
  if (greedy) {
    #pragma unroll 1
    for (int v = tid; v < n_vec; v += RACE_THREADS)
      #pragma unroll 1
      for (int i = 8 * v; i < 8 * v + 8; ++i) if (as_float(piece[i]) == zmax) first = min(first, begin + i);
  }

  // ---- the weights: at temperature 1 for the log-prob; at the row's for the race, kept in place of the logits (those of
  //      bf16 logits as bf16: the race has room for that)
  float s1 = 0.f, sT = 0.f;
  const bool other = scale != SMP_LOG2E || floor_octaves < CUDART_INF_F;
  {
    float2 sum1 = both(0.f), sum2 = both(0.f);
    if (!other) {
      for (int v = tid; v < n_vec; v += RACE_THREADS) {
        float z[8];
        Vec<T>::get(piece + 8 * v, z);
        float2 w[4];
        #pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 x = mul2(add2(make_float2(z[2 * i], z[2 * i + 1]), both(-ref)), both(SMP_LOG2E));
          w[i] = make_float2(ex2(x.x), ex2(x.y));
          sum1 = add2(sum1, w[i]);
        }
        store_weights(piece + 8 * v, w);
      }
    } else {
      for (int v = tid; v < n_vec; v += RACE_THREADS) {
        float z[8];
        Vec<T>::get(piece + 8 * v, z);
        float2 w[4];
        #pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 d = add2(make_float2(z[2 * i], z[2 * i + 1]), both(-ref)), x = mul2(d, both(SMP_LOG2E)), o = mul2(d, both(scale));
          sum1 = add2(sum1, make_float2(ex2(x.x), ex2(x.y)));
          w[i] = make_float2(-o.x <= floor_octaves ? ex2(o.x) : 0.f, -o.y <= floor_octaves ? ex2(o.y) : 0.f);
          sum2 = add2(sum2, w[i]);
        }
        store_weights(piece + 8 * v, w);
      }
    }
    s1 = sum1.x + sum1.y; sT = sum2.x + sum2.y;
  }
  #pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    s1 += __shfl_xor_sync(ALL, s1, d);
    if (other) sT += __shfl_xor_sync(ALL, sT, d);
  }
  if (greedy) first = __reduce_min_sync(ALL, first);
  __syncthreads();
  if (lane == 0) { sh.warp[0][warp] = s1; sh.warp[1][warp] = sT; sh.first[warp] = first; }
  __syncthreads();
  s1 = 0.f; sT = 0.f;
  #pragma unroll
  for (int w = 0; w < RACE_WARPS; ++w) { s1 += sh.warp[0][w]; sT += sh.warp[1][w]; }
  const float weight = other ? sT : s1;

  // ---- the race
  auto finish = [&](uint32_t token, float z, float top) -> double {          // against the logit `top`, in 64 bits
    const double e = -log1p(-((double)random_bits(token, k0, k1) + 0.5) * 2.3283064365386963e-10);
    return e * exp(((double)top - (double)z) * fmin(1.0 / (double)temperature, 1e30));
  };
  uint32_t out[4] = {__float_as_uint(zmax), __float_as_uint(s1), __float_as_uint(CUDART_INF_F), ALL};      // what the block has to say
  if (greedy) {
    for (int w = 0; w < RACE_WARPS; ++w) out[3] = min(out[3], sh.first[w]);
  } else if (usable && weight > 0.f) {
    // A token is worth working out if it may finish before `lead` / weight; the block's first does with probability
    // 1 - exp(-lead), else the block looks again, further.  The eights with such a token are listed.
    float t1 = CUDART_INF_F;
    #pragma unroll 1
    for (float lead = RACE_LEAD; lead < 1e4f; lead *= 4.f) {
      const float reach = lead / weight, bound = 65536.f * reach * 1.01f;
      for (int v = tid; v < n_vec; v += RACE_THREADS) {
        float w[8];
        Vec<T>::get(piece + 8 * v, w);
        const uint4 r = philox4x32_10((begin >> 3) + v, 0, 0, 0, k0, k1);
        const uint32_t word[4] = {r.x, r.y, r.z, r.w};
        float ahead[2] = {-1.f, -1.f};
        #pragma unroll
        for (int i = 0; i < 4; ++i) {               // 2^23 + 1 + bound w against 2^23 + the upper bits
          const float2 may = fma2(make_float2(w[2 * i], w[2 * i + 1]), both(bound), both(8388609.f));
          ahead[0] = fmaxf(ahead[0], may.x - __uint_as_float(__byte_perm(word[i], 0x4B000000u, 0x7610)));
          ahead[1] = fmaxf(ahead[1], may.y - __uint_as_float(__byte_perm(word[i], 0x4B000000u, 0x7632)));
        }
        if (fmaxf(ahead[0], ahead[1]) >= 0.f) {
          const uint32_t at = atomicAdd(&sh.n_list, 1u);
          if (at < SMP_LIST) sh.list[at] = v;
        }
      }
      __syncthreads();
      const uint32_t listed = min(sh.n_list, (uint32_t)SMP_LIST), looked = 8 * listed;
      const bool all_listed = sh.n_list <= SMP_LIST;
      if (warp == 0) {                             // the list is short: one warp works it out
        t1 = CUDART_INF_F;
        float t2 = CUDART_INF_F;
        uint32_t who = ALL;
        #pragma unroll 1
        for (uint32_t j = lane; j < looked; j += 32) {
          const int i = 8 * (int)sh.list[j >> 3] + (int)(j & 7u);
          const float o = i < n ? (zmax - as_float(from[i])) * scale : CUDART_INF_F;
          const float t = o <= floor_octaves ? finish32(random_bits(begin + i, k0, k1), o) : CUDART_INF_F;
          t2 = fminf(t2, fmaxf(t1, t));
          if (t < t1) { t1 = t; who = begin + i; }
        }
        #pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
          const float u1 = __shfl_xor_sync(ALL, t1, d), u2 = __shfl_xor_sync(ALL, t2, d);
          const uint32_t x = __shfl_xor_sync(ALL, who, d);
          t2 = fminf(fmaxf(t1, u1), fminf(t2, u2));
          if (u1 < t1 || (u1 == t1 && x < who)) { t1 = u1; who = x; }
        }
        if (t2 <= t1 * SMP_TIE && t1 < CUDART_INF_F) {       // two come near: in 64 bits
          double best = CUDART_INF;
          uint32_t winner = ALL;
          #pragma unroll 1
          for (uint32_t j = lane; j < looked; j += 32) {
            const int i = 8 * (int)sh.list[j >> 3] + (int)(j & 7u);
            const float z = i < n ? as_float(from[i]) : -CUDART_INF_F;
            if (!((zmax - z) * scale <= floor_octaves)) continue;
            const double t = finish(begin + i, z, zmax);
            if (t < best || (t == best && begin + i < winner)) { best = t; winner = begin + i; }
          }
          #pragma unroll 1
          for (int d = 16; d > 0; d >>= 1) {
            const double t = __shfl_xor_sync(ALL, best, d);
            const uint32_t x = __shfl_xor_sync(ALL, winner, d);
            if (t < best || (t == best && x < winner)) { best = t; winner = x; }
          }
          if (winner != ALL) { who = winner; t1 = (float)best; }
        }
        if (lane == 0) { sh.warp[0][0] = t1; sh.who = who; sh.n_list = 0; }
      }
      __syncthreads();
      t1 = sh.warp[0][0];
      out[2] = __float_as_uint(t1); out[3] = sh.who;
      if (t1 < 0.99f * reach && all_listed) break;
      t1 = CUDART_INF_F;
      if (!all_listed) break;
    }
    if (t1 == CUDART_INF_F) {                      // too many to list, or none in reach at all: every token
      double best = CUDART_INF;
      uint32_t who = ALL;
      #pragma unroll 1
      for (int i = tid; i < n; i += RACE_THREADS) {
        const float z = as_float(from[i]);
        if (!((zmax - z) * scale <= floor_octaves)) continue;
        const double t = finish(begin + i, z, zmax);
        if (t < best) { best = t; who = begin + i; }
      }
      __syncthreads();
      if (tid == 0) { sh.best = CUDART_INF; sh.who = ALL; }
      #pragma unroll 1
      for (int turn = 0; turn < RACE_THREADS; ++turn) {
        __syncthreads();
        if (tid == turn && (best < sh.best || (best == sh.best && who < sh.who))) { sh.best = best; sh.who = who; }
      }
      __syncthreads();
      out[2] = __float_as_uint((float)sh.best); out[3] = sh.who;
    }
  }

  // ---- the first block compares the blocks
  __syncwarp();
  if (!waited) wait();
  if (tid == 0) {
    uint32_t* to = cluster.map_shared_rank(&sh.slots[rank][0], 0);
    for (int i = 0; i < 4; ++i) to[i] = out[i];
  }
  __syncwarp();
  arrive();
  if (rank != 0) return;
  wait();
  if (tid != 0) return;
  float top = -CUDART_INF_F, total = 0.f, t1 = CUDART_INF_F, t2 = CUDART_INF_F;
  uint32_t who = ALL;
  for (uint32_t r = 0; r < C; ++r) top = max_nan(top, __uint_as_float(sh.slots[r][0]));
  if (!(top < CUDART_INF_F) || top == -CUDART_INF_F || !settings_ok) {
    a.ids[row] = -1; a.logp[row] = 0.f;
    if (!settings_ok || top != -CUDART_INF_F) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
    return;
  }
  auto time_of = [&](uint32_t r) { return __uint_as_float(sh.slots[r][2]) * ex2((top - __uint_as_float(sh.slots[r][0])) * scale); };
  for (uint32_t r = 0; r < C; ++r) {
    const float less = top - __uint_as_float(sh.slots[r][0]);
    total += __uint_as_float(sh.slots[r][1]) * ex2(-less * SMP_LOG2E);
    if (sh.slots[r][3] == ALL) continue;
    if (greedy) { if (less == 0.f) who = min(who, sh.slots[r][3]); continue; }
    const float t = time_of(r);
    t2 = fminf(t2, fmaxf(t1, t));
    if (t < t1) { t1 = t; who = sh.slots[r][3]; }
  }
  const T* z_row = static_cast<const T*>(a.z) + (int64_t)row * a.ld;
  if (!greedy && (t2 <= t1 * SMP_TIE || !(t1 < 1e37f))) {                // two blocks' come near: in 64 bits
    double best = CUDART_INF;
    for (uint32_t r = 0; r < C; ++r) {
      const uint32_t token = sh.slots[r][3];
      if (token == ALL || (t1 < 1e37f && time_of(r) > t1 * SMP_TIE)) continue;
      const double t = finish(token, as_float(z_row[token]), top);
      if (t < best || (t == best && token < who)) { best = t; who = token; }
    }
  }
  a.ids[row] = (int32_t)who;
  a.logp[row] = (as_float(z_row[who]) - top) - logf(total);
}

// How many blocks share a row: so many that an SM has room for its share of them (`most` bytes of logits each); a batch
// that would not fill the device is cut finer, down to 2048 tokens a block.
static int blocks_of_row(const SampleArgs& a, size_t size, int64_t most, int sms, int32_t& piece) {
  const auto piece_of = [&](int c) { return round_up<int64_t>(ceil_div<int64_t>(a.V, c), 8); };
  int C = 1;
  while (C < SMP_MAX_CLUSTER && piece_of(C) * (int64_t)size > most) C *= 2;
  while (C < SMP_MAX_CLUSTER && (int64_t)a.B * C * 2 <= 2 * sms && piece_of(C) > 2048) C *= 2;
  piece = (int32_t)piece_of(C);
  return C;
}

template <class Kernel>
static int launch_sample(Kernel kernel, bool (&allowed)[MAX_DEVICES], int threads, size_t shared, size_t size, int64_t most, SampleArgs a, int sms,
                         cudaStream_t st) {
  const int C = blocks_of_row(a, size, most, sms, a.piece), dev = current_device();
  if (a.piece * size > SMP_MAX_PIECE) return SAPO_ERR_UNSUPPORTED_SHAPE;
  if (dev < 0) return SAPO_ERR_CUDA;
  if (!allowed[dev]) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(shared + SMP_MAX_PIECE)) != cudaSuccess) return SAPO_ERR_CUDA;
    allowed[dev] = true;
  }
  KernelScope scope(SAPO_K_SAMPLE, st);
  return launch_overlapped(kernel, dim3((unsigned)(a.B * C)), threads, shared + a.piece * size, C, st, a);
}
template <class T>
static int launch_sample(const SampleArgs& a, int sms, cudaStream_t st) {
  static bool allowed[2][MAX_DEVICES] = {{false}, {false}};
  if (a.top_k || a.top_p || a.top_k_all > 1 || a.top_p_all < 1.f)      // (top_k 1 is the largest logit)
    return launch_sample(sample_kernel<T>, allowed[0], SMP_THREADS, SMP_SHARED, sizeof(T), 76 * 1024, a, sms, st);
  return launch_sample(race_kernel<T>, allowed[1], RACE_THREADS, RACE_SHARED, sizeof(T), 40 * 1024, a, sms, st);
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
  if (V > SMP_MAX_TOKENS || (int64_t)V * (int64_t)size > (int64_t)SMP_MAX_CLUSTER * (int64_t)SMP_MAX_PIECE - 64 * SMP_MAX_CLUSTER || B > (1 << 24)) return SAPO_ERR_UNSUPPORTED_SHAPE;
  if (reinterpret_cast<uintptr_t>(logits) % size) return SAPO_ERR_INVALID_ARG;
  const int sms = sm_count();
  if (sms <= 0) return SAPO_ERR_CUDA;
  const SampleArgs a{logits, ld, B, V, 0, seeds, h_cfg->temperature_rows, h_cfg->top_k_rows, h_cfg->top_p_rows, h_cfg->min_p_rows,
                     h_cfg->temperature, h_cfg->top_k, h_cfg->top_p, h_cfg->min_p, ids, logp, status};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return dtype == SAPO_DTYPE_BF16 ? launch_sample<__nv_bfloat16>(a, sms, st) : launch_sample<float>(a, sms, st);
}
