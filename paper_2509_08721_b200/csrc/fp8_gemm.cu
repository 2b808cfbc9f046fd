// sapo_fp8_matmul: y = x W^T of two matrices in 8-bit floating point,
//   y[t, n] = sum_kb sx[t, kb] sw[n / 128, kb] sum_{k in block kb} x[t, k] W[n, k].
// The tensor cores form the inner sum of one block of 128 (four tcgen05.mma of depth 32) into tensor memory; the scales
// differ from block to block, so each such partial product is taken out, scaled and added up in fp32 registers, while
// the tensor cores are on the next block in another part of tensor memory.
//
// Two kernels.  fp8_wide_kernel: a pair of CTAs (cta_group::2) on a tile of 256 tokens x 256 columns; a thread holds 128
// columns of one token, whose scale is one number per block of 128.  fp8_narrow_kernel: 128 rows of W by 16 to 128
// tokens, W on the side of the 128 lanes, for few tokens (the head is read once, at the rate of memory) and for
// matrices too small to fill the device with wide tiles; where even its tiles are few, a cluster of CTAs shares one
// along K and adds up in shared memory, in a fixed order.
//
// What bounds them.  Wide, 8192 x 14336 x 3584: 421 us in a burst (2.0 PFLOP/s), 484 sustained under the power cap; without
// the scaling warps' work 427 sustained, with a hand-over every fourth block of K 371.  So taking 128 x 256 partial sums out of
// tensor memory per block costs a quarter; loads of 8 or 32 columns instead of 16, 16 warps instead of 8 and more registers
// for them were each slower (442 to 587 in a burst).  4096 x 151936 x 896 (7 blocks of K a tile): 655 / 770 us, the output of a
// tile adds to its 7 blocks.  Narrow, 1 x 151936 x 896: 29 us (4.7 TB/s; the last of nine rounds, the launch and the pipeline's
// filling take a quarter); 64 x 152064 x 3584: 132 us (4.4 TB/s; the token tile is fetched again with every 128 rows of W, half
// as many bytes as these; without the scaling work 117).
#include <cuda_bf16.h>

#include "common.cuh"
#include "paired.cuh"
#include "umma.cuh"

namespace sapo {
using namespace umma;

constexpr int F8_K = 128;                                  // depth of a stage and of a scale: one 128-byte row segment
constexpr uint32_t F8_BOX = 128 * F8_K;                    // 128 rows of a stage

struct Fp8GemmArgs {
  const float* sx; int64_t ld_sx;
  const float* sw; int64_t ld_sw;
  void* y; int64_t ld_y;
  int64_t T; int32_t N, num_kb, out_bf16;
  int32_t group_m;          // wide: token blocks that are walked before the next column block
  int32_t tma_store;        // wide: y can be written by TMA
  int32_t split;            // narrow: CTAs that share a tile along K
  int32_t rows, nt;         // narrow: rows of W (at most 128) and tokens (a multiple of 16, at most NT) of a tile
  int32_t unit0, units;     // the tiles of this launch
  int32_t of_wide;          // narrow: four tiles each of the wide tiles from unit0 on, which have this order's num_m, num_n
  int32_t num_m, num_n;     // wide tiles along tokens and columns
  int32_t tail_follows;     // another launch of this call takes the last tiles: it may start as soon as this one runs
  int32_t tail;             // this is that launch
  long long wait_limit;
  int32_t* status;
};

// Instruction descriptor of tcgen05.mma kind::f8f6f4, both operands e4m3 (type 0) and K-major, fp32 accumulation.
__host__ __device__ constexpr uint32_t make_idesc_f8(int M, int N) {
  return (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
__device__ __forceinline__ void mma_f8(uint32_t tmem_d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(tmem_d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_f8_pair(uint32_t tmem_d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(tmem_d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// wait until all but the last of this thread's groups of stores have finished reading shared memory
__device__ __forceinline__ void bulk_wait_read_but_one() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }
// named_barrier_sync that also says whether `yes` holds in all its threads
__device__ __forceinline__ bool named_barrier_and(int id, int n_threads, bool yes) {
  uint32_t all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %3, 0;\n\tbarrier.cta.red.and.pred q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(all) : "r"(id), "r"(n_threads), "r"((uint32_t)yes) : "memory");
  return all != 0;
}
// 16 accumulator columns of this thread's lane
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&v)[16]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                 "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr) : "memory");
}

// wait for this thread's loads; the values are tied to the wait, so that no use of them moves in front of it
__device__ __forceinline__ void tmem_ld_wait16(float (&v)[16]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
}

// A grid of one CTA pair per SM pair leaves most of the device idle while the last, partial round of wide tiles runs; a
// second launch takes these tiles in narrow ones, and shares each of those among several CTAs along K.  It does not wait for the first one's results, so
// the first lets it start (behind its own wait for what comes before the call) and its CTAs fill SMs as they fall idle;
// what follows the call must wait for both, so the second waits for the first before it ends.
__device__ __forceinline__ void begin_launch(const Fp8GemmArgs& a) {
  if (!a.tail) wait_for_previous();
  if (a.tail_follows) let_next_start();
}
__device__ __forceinline__ void end_launch(const Fp8GemmArgs& a) { if (a.tail) wait_for_previous(); }

// ---------------------------------------------------------------------------- wide tiles
constexpr int F8W_STAGES = 5;
constexpr int F8W_THREADS = 320;                           // warp 0: TMA, warp 1: MMA, warps 2-9: scaling and output
constexpr uint32_t F8W_STAGE = 2 * F8_BOX;                 // this CTA's 128 tokens, and its half of the 256 columns
constexpr uint32_t F8W_STAGING = 128 * 128;                // output on its way: 128 rows of 128 bytes, two per half of the columns
constexpr size_t F8W_SMEM = 1024 + F8W_STAGES * F8W_STAGE + 4 * F8W_STAGING + 256;
static_assert(F8W_SMEM <= 232448, "more shared memory than a CTA can have");

// Tile `unit`: groups of group_m token blocks; inside a group the token block runs fastest, so that a group's tokens stay
// in L2 while W streams past them once.
__device__ __forceinline__ void wide_tile(const Fp8GemmArgs& a, int unit, int& mb, int& nb) {
  const int per_group = a.group_m * a.num_n, g = unit / per_group, r = unit - g * per_group;
  const int rows = min(a.group_m, a.num_m - g * a.group_m);
  nb = r / rows;
  mb = g * a.group_m + (r - nb * rows);
}

__global__ void __launch_bounds__(F8W_THREADS, 1)
fp8_wide_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                const __grid_constant__ CUtensorMap map_y, const Fp8GemmArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* staging = smem + F8W_STAGES * F8W_STAGE;
  uint64_t* bars = reinterpret_cast<uint64_t*>(staging + 4 * F8W_STAGING);
  uint64_t* full = bars;                          // TMA -> MMA             (even CTA's are used)
  uint64_t* empty = bars + F8W_STAGES;            // MMA -> TMA             (each CTA waits on its own)
  uint64_t* acc_full = bars + 2 * F8W_STAGES;     // [2] MMA -> scaling     (each CTA waits on its own)
  uint64_t* acc_empty = acc_full + 2;             // [2] scaling -> MMA     (even CTA's are used)
  uint64_t* drain = acc_empty + 2;                // MMA thread only, after a wait ran out
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_cta_rank();
  const int pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
  const int units = a.units;
  if (threadIdx.x == 0) {
    for (int i = 0; i < F8W_STAGES; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], 16); }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tensormap(&map_x); prefetch_tensormap(&map_w); prefetch_tensormap(&map_y);
  }
  if (warp == 1) { tmem_alloc_pair(tmem_slot, 512); tmem_relinquish_pair(); }
  fence_before_sync();
  __syncthreads();
  cluster_sync_all();
  begin_launch(a);
  fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  const uint32_t full0 = map_to_cta(smem_u32(full), 0), acc_empty0 = map_to_cta(smem_u32(acc_empty), 0);
  const uint32_t empty_of[2] = {map_to_cta(smem_u32(empty), 0), map_to_cta(smem_u32(empty), 1)};
  const uint32_t acc_full_of[2] = {map_to_cta(smem_u32(acc_full), 0), map_to_cta(smem_u32(acc_full), 1)};

  if (warp == 0 && lane == 0) {
    // ------------------------------------------------------------ TMA (both CTAs)
    int stage = 0; uint32_t phase = 0, in_flight = 0;
    bool ok = true;
    for (int unit = pair; ok && unit < units; unit += num_pairs) {
      int mb, nb;
      wide_tile(a, unit, mb, nb);
      for (int kb = 0; kb < a.num_kb; ++kb) {
        if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag, a.wait_limit)) { ok = false; break; }
        if (rank == 0) mbar_arrive_expect_tx(&full[stage], 2 * F8W_STAGE);
        uint8_t* to = smem + stage * F8W_STAGE;
        tma_load_2d_pair(to, &map_x, full0 + stage * 8, kb * F8_K, mb * 256 + (int)rank * 128);
        tma_load_2d_pair(to + F8_BOX, &map_w, full0 + stage * 8, kb * F8_K, nb * 256 + (int)rank * 128);
        in_flight |= 1u << stage;
        if (++stage == F8W_STAGES) { stage = 0; phase ^= 1; }
      }
    }
    if (!ok && rank == 0)                           // copies already issued get a bounded chance to land
      for (int i = 0; i < F8W_STAGES; ++i) {
        if (!(in_flight & (1u << i))) continue;
        const uint32_t ph = i < stage ? phase : phase ^ 1;
        for (int spin = 0; spin < (1 << 20) && !mbar_try_wait(&full[i], ph); ++spin) {}
      }
  } else if (warp == 1 && lane == 0 && rank == 0) {
    // ------------------------------------------------------------ MMA (even CTA)
    constexpr uint32_t idesc = make_idesc_f8(256, 256);
    int stage = 0, acc = 0; uint32_t phase = 0, acc_phase = 0;
    bool ok = true;
    for (int unit = pair; ok && unit < units; unit += num_pairs)
      for (int kb = 0; kb < a.num_kb; ++kb) {
        if (!mbar_wait(&acc_empty[acc], acc_phase ^ 1, abort_flag, a.wait_limit) ||
            !mbar_wait(&full[stage], phase, abort_flag, a.wait_limit)) { ok = false; break; }
        fence_after_sync();
        const uint32_t at = smem_u32(smem + stage * F8W_STAGE);
        #pragma unroll
        for (int k = 0; k < 4; ++k)                 // 32 values of K: 32 bytes along the row
          mma_f8_pair(tmem_base + acc * 256, make_smem_desc(at + 32 * k, 16, 1024), make_smem_desc(at + F8_BOX + 32 * k, 16, 1024), idesc, k != 0);
        mma_commit_pair(empty_of[0] + stage * 8);
        mma_commit_pair(empty_of[1] + stage * 8);
        mma_commit_pair(acc_full_of[0] + acc * 8);
        mma_commit_pair(acc_full_of[1] + acc * 8);
        if (++stage == F8W_STAGES) { stage = 0; phase ^= 1; }
        if (++acc == 2) { acc = 0; acc_phase ^= 1; }
      }
    if (!ok) {                                      // no MMA may still run when tensor memory is freed
      mma_commit_pair(map_to_cta(smem_u32(drain), 0));
      for (int spin = 0; spin < (1 << 22) && !mbar_try_wait(drain, 0); ++spin) {}
    }
  } else if (warp >= 2) {
    // ------------------------------------------------------------ scaling and output (8 warps, both CTAs)
    // warps 2-5 take the tile's first 128 columns, warps 6-9 the others: one block of W's scales each
    const int quad = warp & 3, half = (warp - 2) >> 2, r = quad * 32 + lane;
    const uint32_t bufs = smem_u32(staging) + half * 2 * F8W_STAGING;
    const bool elected = quad == 0 && lane == 0;
    int acc = 0; uint32_t acc_phase = 0, turn = 0;
    bool ok = true;
    for (int unit = pair; ok && unit < units; unit += num_pairs) {
      int mb, nb;
      wide_tile(a, unit, mb, nb);
      const int64_t row0 = (int64_t)mb * 256 + rank * 128;
      const int col0 = nb * 256 + half * 128;
      const float* sx = a.sx + min(row0 + r, a.T - 1) * a.ld_sx;                      // rows and columns past the end are
      const float* sw = a.sw + (int64_t)(min(col0, a.N - 1) >> 7) * a.ld_sw;          // not stored
      float2 sum[64];
      #pragma unroll
      for (int j = 0; j < 64; ++j) sum[j] = both(0.f);
      float next = __ldg(sx) * __ldg(sw);
      for (int kb = 0; kb < a.num_kb; ++kb) {
        const float2 s = both(next);
        if (kb + 1 < a.num_kb) next = __ldg(sx + kb + 1) * __ldg(sw + kb + 1);
        if (!__all_sync(0xFFFFFFFFu, mbar_wait(&acc_full[acc], acc_phase, abort_flag, a.wait_limit))) { ok = false; break; }
        fence_after_sync();
        const uint32_t t_addr = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + acc * 256 + half * 128;
        float v[2][16];
        tmem_ld16(t_addr, v[0]);
        #pragma unroll
        for (int c = 0; c < 8; ++c) {
          tmem_ld_wait16(v[c & 1]);
          if (c < 7) tmem_ld16(t_addr + 16 * (c + 1), v[(c + 1) & 1]);
          else {
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(acc_empty0 + acc * 8);
          }
          #pragma unroll
          for (int j = 0; j < 8; ++j) sum[8 * c + j] = fma2(s, make_float2(v[c & 1][2 * j], v[c & 1][2 * j + 1]), sum[8 * c + j]);
        }
        if (++acc == 2) { acc = 0; acc_phase ^= 1; }
      }
      ok = named_barrier_and(1 + half, 128, ok);     // the four warps store together, or none of them
      if (!ok) break;
      // output by pieces of 128 bytes a row: 64 columns of bf16 or 32 of fp32, in the 128-byte swizzle
      const int pieces = a.out_bf16 ? 2 : 4, width = a.out_bf16 ? 64 : 32;
      #pragma unroll
      for (int p = 0; p < 4; ++p) {
        if (p >= pieces || col0 + p * width >= a.N || row0 >= a.T) break;             // the same for all 128 threads
        const uint32_t buf = bufs + (turn & 1u) * F8W_STAGING;
        ++turn;
        if (a.tma_store && elected) bulk_wait_read_but_one();      // the store before the last has left this buffer
        named_barrier_sync(1 + half, 128);
        #pragma unroll
        for (int q = 0; q < 8; ++q) {
          uint32_t w[4];
          if (a.out_bf16) {
            #pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 f = sum[(p & 1) * 32 + 4 * q + i];
              const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
              w[i] = *reinterpret_cast<const uint32_t*>(&b);
            }
          } else {
            #pragma unroll
            for (int i = 0; i < 4; ++i) { const float2 f = sum[p * 16 + 2 * q + (i >> 1)]; w[i] = __float_as_uint((i & 1) ? f.y : f.x); }
          }
          st_shared_v4(buf + r * 128 + ((q ^ (r & 7)) << 4), w[0], w[1], w[2], w[3]);
        }
        if (a.tma_store) {
          fence_proxy_async_smem();
          named_barrier_sync(1 + half, 128);
          if (elected) { tma_store_2d(&map_y, buf, col0 + p * width, (int32_t)row0); bulk_commit_group(); }
        } else {                                    // rows of y on no 16-byte boundary: a warp writes a row's columns
          named_barrier_sync(1 + half, 128);
          const uint8_t* from = staging + (buf - smem_u32(staging));
          for (int i = 0; i < 32; ++i) {
            const int rr = quad * 32 + i;
            if (row0 + rr >= a.T) break;
            if (a.out_bf16) {
              #pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int c = lane + 32 * h;
                if (col0 + p * 64 + c < a.N)
                  static_cast<__nv_bfloat16*>(a.y)[(row0 + rr) * a.ld_y + col0 + p * 64 + c] =
                      *reinterpret_cast<const __nv_bfloat16*>(from + rr * 128 + (((c >> 3) ^ (rr & 7)) << 4) + 2 * (c & 7));
              }
            } else if (col0 + p * 32 + lane < a.N)
              static_cast<float*>(a.y)[(row0 + rr) * a.ld_y + col0 + p * 32 + lane] =
                  *reinterpret_cast<const float*>(from + rr * 128 + (((lane >> 2) ^ (rr & 7)) << 4) + 4 * (lane & 3));
          }
        }
      }
    }
    if (elected) bulk_wait_all();       // stores done before shared memory goes away
  }
  fence_before_sync();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) { fence_after_sync(); tmem_dealloc_pair(tmem_base, 512); }
  if (threadIdx.x == 0 && *abort_flag) raise_status(a.status, SAPO_ST_WAIT_TIMEOUT);
}

// ---------------------------------------------------------------------------- narrow tiles
constexpr int F8N_BUFFERS = 4;                    // partial products in tensor memory
constexpr int F8N_SCALES = 32;                    // blocks of K whose token scales are in shared memory
template <int NT> struct Narrow {
  static constexpr int GROUPS = NT >= 64 ? 2 : 1, WARPS = 4 * GROUPS, COLS = NT / GROUPS;      // warps that scale; tokens of a thread
  static constexpr int THREADS = 64 + 32 * WARPS;                                              // warp 0: TMA, warp 1: MMA
  static constexpr uint32_t STAGE = F8_BOX + NT * F8_K, OUT = NT * 128 * 4;
  static constexpr int STAGES = (220 * 1024 - (int)OUT) / (int)STAGE < 10 ? (220 * 1024 - (int)OUT) / (int)STAGE : 10;
  static constexpr uint32_t TMEM = NT * F8N_BUFFERS < 64 ? 64 : NT * F8N_BUFFERS;
  static constexpr size_t SMEM = 1024 + STAGES * STAGE + OUT + F8N_SCALES * NT * 4 + 256;
  static_assert((TMEM & (TMEM - 1)) == 0 && TMEM <= 512 && SMEM <= 232448 && STAGES >= 4, "tensor or shared memory");
};

template <int NT>
__global__ void __launch_bounds__(Narrow<NT>::THREADS, 1)
fp8_narrow_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const Fp8GemmArgs a) {
  using Z = Narrow<NT>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* out = reinterpret_cast<float*>(smem + Z::STAGES * Z::STAGE);         // [NT][128]: a tile's sums
  float* scales = out + NT * 128;                                             // [F8N_SCALES][NT]
  uint64_t* bars = reinterpret_cast<uint64_t*>(scales + F8N_SCALES * NT);
  uint64_t* full = bars;
  uint64_t* empty = bars + Z::STAGES;
  uint64_t* acc_full = bars + 2 * Z::STAGES;
  uint64_t* acc_empty = acc_full + F8N_BUFFERS;
  uint64_t* drain = acc_empty + F8N_BUFFERS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert((2 * Z::STAGES + 2 * F8N_BUFFERS + 2) * 8 <= 256, "barriers overflow their region");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < Z::STAGES; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < F8N_BUFFERS; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], Z::WARPS); }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tensormap(&map_x); prefetch_tensormap(&map_w);
  }
  if (warp == 1) { tmem_alloc(tmem_slot, Z::TMEM); tmem_relinquish(); }
  fence_before_sync();
  __syncthreads();
  if (a.split > 1) cluster_sync_all();
  begin_launch(a);
  fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  const int rank = blockIdx.x % a.split, first = blockIdx.x / a.split, stride = gridDim.x / a.split;
  const int kb0 = (int)((int64_t)a.num_kb * rank / a.split), kb1 = (int)((int64_t)a.num_kb * (rank + 1) / a.split);
  const int num_t = (int)((a.T + a.nt - 1) / a.nt);
  // tile u: rows of W [rows nb, + rows), tokens [nt tb, + nt); the token tiles of a block of W follow one another
  auto tile = [&](int u, int& nb, int& tb) {
    if (a.of_wide) {
      int wm, wn;
      wide_tile(a, a.unit0 + (u >> 2), wm, wn);
      nb = 2 * wn + ((u >> 1) & 1); tb = 2 * wm + (u & 1);
    } else { nb = (a.unit0 + u) / num_t; tb = a.unit0 + u - nb * num_t; }
  };
  const uint32_t stage_bytes = (uint32_t)(a.rows + a.nt) * F8_K;

  if (warp == 0 && lane == 0) {
    // ------------------------------------------------------------ TMA
    int stage = 0; uint32_t phase = 0, in_flight = 0;
    bool ok = true;
    for (int unit = first; ok && unit < a.units; unit += stride) {
      int nb, tb;
      tile(unit, nb, tb);
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag, a.wait_limit)) { ok = false; break; }
        mbar_arrive_expect_tx(&full[stage], stage_bytes);
        uint8_t* to = smem + stage * Z::STAGE;             // (what a smaller box leaves of the stage makes sums that are not stored)
        tma_load_2d(to, &map_w, &full[stage], kb * F8_K, nb * a.rows);
        tma_load_2d(to + F8_BOX, &map_x, &full[stage], kb * F8_K, tb * a.nt);
        in_flight |= 1u << stage;
        if (++stage == Z::STAGES) { stage = 0; phase ^= 1; }
      }
    }
    if (!ok)
      for (int i = 0; i < Z::STAGES; ++i) {
        if (!(in_flight & (1u << i))) continue;
        const uint32_t ph = i < stage ? phase : phase ^ 1;
        for (int spin = 0; spin < (1 << 20) && !mbar_try_wait(&full[i], ph); ++spin) {}
      }
  } else if (warp == 1 && lane == 0) {
    // ------------------------------------------------------------ MMA
    const uint32_t idesc = make_idesc_f8(128, a.nt);
    int stage = 0, acc = 0; uint32_t phase = 0, acc_phase = 0;
    bool ok = true;
    for (int unit = first; ok && unit < a.units; unit += stride)
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(&acc_empty[acc], acc_phase ^ 1, abort_flag, a.wait_limit) ||
            !mbar_wait(&full[stage], phase, abort_flag, a.wait_limit)) { ok = false; break; }
        fence_after_sync();
        const uint32_t at = smem_u32(smem + stage * Z::STAGE);
        #pragma unroll
        for (int k = 0; k < 4; ++k)
          mma_f8(tmem_base + acc * NT, make_smem_desc(at + 32 * k, 16, 1024), make_smem_desc(at + F8_BOX + 32 * k, 16, 1024), idesc, k != 0);
        mma_commit(&empty[stage]);
        mma_commit(&acc_full[acc]);
        if (++stage == Z::STAGES) { stage = 0; phase ^= 1; }
        if (++acc == F8N_BUFFERS) { acc = 0; acc_phase ^= 1; }
      }
    if (!ok) {
      mma_commit(drain);
      for (int spin = 0; spin < (1 << 22) && !mbar_try_wait(drain, 0); ++spin) {}
    }
  } else if (warp >= 2) {
    // ------------------------------------------------------------ scaling and output: a thread has one row of W, COLS tokens
    constexpr int EPI = 32 * Z::WARPS;
    const int quad = warp & 3, group = (warp - 2) >> 2, r = quad * 32 + lane, e = threadIdx.x - 64;
    int acc = 0; uint32_t acc_phase = 0;
    bool ok = true;
    int held_tb = -1, held_kb = -1;                // token scales in shared memory: of token tile held_tb, from block held_kb on
    for (int unit = first; unit < a.units; unit += stride) {
      int nb, tb;
      tile(unit, nb, tb);
      const int64_t t0 = (int64_t)tb * a.nt;
      const float* sw = a.sw + (int64_t)(min(nb * a.rows + r, a.N - 1) >> 7) * a.ld_sw;      // (rows past the end are not stored)
      float2 sum[Z::COLS / 2];
      #pragma unroll
      for (int j = 0; j < Z::COLS / 2; ++j) sum[j] = both(0.f);
      float next_w = kb0 < kb1 ? __ldg(sw + kb0) : 0.f;
      #pragma unroll 1
      for (int kb = kb0; kb < kb1; ++kb) {
        const int kb_base = kb0 + ((kb - kb0) / F8N_SCALES) * F8N_SCALES;
        if (tb != held_tb || kb_base != held_kb) {      // the same for all these warps
          named_barrier_sync(1, EPI);
          const int t = e % NT, blocks = min(F8N_SCALES, kb1 - kb_base);
          const float* from = a.sx + min(t0 + t, a.T - 1) * a.ld_sx + kb_base;
          #pragma unroll 8
          for (int k = e / NT; k < blocks; k += EPI / NT) scales[k * NT + t] = __ldg(from + k);
          held_tb = tb; held_kb = kb_base;
          named_barrier_sync(1, EPI);
        }
        const float* s = scales + (kb - kb_base) * NT;
        const float2 scale_w = both(next_w);
        if (kb + 1 < kb1) next_w = __ldg(sw + kb + 1);
        // (after a wait that ran out the warps go on without waiting: the barriers among them stay in step)
        if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&acc_full[acc], acc_phase, abort_flag, a.wait_limit));
        if (ok) {
          fence_after_sync();
          const uint32_t t_addr = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + acc * NT + group * Z::COLS;
          float v[2][16];
          tmem_ld16(t_addr, v[0]);
          #pragma unroll
          for (int c = 0; c < Z::COLS / 16; ++c) {
            tmem_ld_wait16(v[c & 1]);
            if (c + 1 < Z::COLS / 16) tmem_ld16(t_addr + 16 * (c + 1), v[(c + 1) & 1]);
            else {
              fence_before_sync();
              __syncwarp();
              if (lane == 0) mbar_arrive(&acc_empty[acc]);
            }
            #pragma unroll
            for (int j = 0; j < 8; j += 2) {
              const float4 f = *reinterpret_cast<const float4*>(s + group * Z::COLS + 16 * c + 2 * j);
              sum[8 * c + j] = fma2(mul2(make_float2(f.x, f.y), scale_w), make_float2(v[c & 1][2 * j], v[c & 1][2 * j + 1]), sum[8 * c + j]);
              sum[8 * c + j + 1] = fma2(mul2(make_float2(f.z, f.w), scale_w), make_float2(v[c & 1][2 * j + 2], v[c & 1][2 * j + 3]), sum[8 * c + j + 1]);
            }
          }
        }
        if (++acc == F8N_BUFFERS) { acc = 0; acc_phase ^= 1; }
      }
      // through shared memory: the loop over the tokens is short code there, whatever their number
      named_barrier_sync(1, EPI);
      #pragma unroll
      for (int j = 0; j < Z::COLS / 2; ++j) {
        out[(group * Z::COLS + 2 * j) * 128 + r] = sum[j].x;
        out[(group * Z::COLS + 2 * j + 1) * 128 + r] = sum[j].y;
      }
      if (a.split == 1) {
        named_barrier_sync(1, EPI);
        const int n = nb * a.rows + (e & 127);
        if ((e & 127) < a.rows && n < a.N) {
          #pragma unroll 4
          for (int j = e >> 7; j < a.nt; j += Z::GROUPS) {
            if (t0 + j >= a.T) break;
            if (a.out_bf16) static_cast<__nv_bfloat16*>(a.y)[(t0 + j) * a.ld_y + n] = __float2bfloat16_rn(out[j * 128 + (e & 127)]);
            else            static_cast<float*>(a.y)[(t0 + j) * a.ld_y + n] = out[j * 128 + (e & 127)];
          }
        }
      }
    }
  }
  if (a.split > 1) {                  // a cluster has one tile: its CTAs add up a share of the tokens each
    __syncthreads();
    cluster_sync_all();
    int nb, tb;
    tile(first, nb, tb);
    const int r = threadIdx.x & 127, n = nb * a.rows + r;
    const int j0 = a.nt * rank / a.split, j1 = a.nt * (rank + 1) / a.split;
    if (threadIdx.x < 128 * Z::GROUPS && r < a.rows && n < a.N)
      #pragma unroll 1
      for (int j = j0 + ((int)threadIdx.x >> 7); j < j1 && (int64_t)tb * a.nt + j < a.T; j += Z::GROUPS) {
        float s = 0.f;
        #pragma unroll 4
        for (int c = 0; c < a.split; ++c) {
          float p;
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(p) : "r"(map_to_cta(smem_u32(out) + (uint32_t)(j * 128 + r) * 4, c)));
          s += p;
        }
        const int64_t at = ((int64_t)tb * a.nt + j) * a.ld_y + n;
        if (a.out_bf16) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(s);
        else            static_cast<float*>(a.y)[at] = s;
      }
    cluster_sync_all();               // nobody leaves while its sums are read
  }
  fence_before_sync();
  __syncthreads();
  if (warp == 1) { fence_after_sync(); tmem_dealloc(tmem_base, Z::TMEM); }
  if (threadIdx.x == 0 && *abort_flag) raise_status(a.status, SAPO_ST_WAIT_TIMEOUT);
  end_launch(a);
}

// ---------------------------------------------------------------------------- host
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiledFn encoder() {
  static EncodeTiledFn fn = nullptr;
  if (fn == nullptr) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(p);
  }
  return fn;
}
// [rows, cols] with `pitch` bytes between rows, boxes of 128 bytes x box_rows in the 128-byte swizzle; zeros outside
static bool map_rows(CUtensorMap* map, CUtensorMapDataType type, int size, const void* base, int64_t cols, int64_t rows, int64_t pitch, int box_rows) {
  EncodeTiledFn fn = encoder();
  if (fn == nullptr) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
  const cuuint32_t box[2] = {(cuuint32_t)(128 / size), (cuuint32_t)box_rows}, step[2] = {1u, 1u};
  return fn(map, type, 2, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class Kernel>
static bool allow_smem(Kernel kernel, size_t bytes, bool (&done)[MAX_DEVICES]) {
  const int dev = current_device();
  if (dev < 0) return false;
  if (!done[dev]) done[dev] = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
  return done[dev];
}

// CTAs that share a tile along K, for `tiles` tiles: as many as the SMs allow, each with at least two blocks of K
static int split_of(int64_t tiles, int num_kb, int sms) {
  int split = 1;
  while (split < 8 && tiles * split * 2 <= sms && num_kb >= 4 * split) split *= 2;
  return split;
}

template <int NT>
static int launch_narrow(const CUtensorMap& map_x, const CUtensorMap& map_w, const Fp8GemmArgs& a, int sms, cudaStream_t st) {
  static bool done[MAX_DEVICES] = {false};
  if (!allow_smem(fp8_narrow_kernel<NT>, Narrow<NT>::SMEM, done)) return SAPO_ERR_CUDA;
  const int grid = a.split > 1 ? a.units * a.split : (a.units < sms ? a.units : sms);
  KernelScope scope(SAPO_K_FP8_MATMUL, st);
  return launch_overlapped(fp8_narrow_kernel<NT>, dim3((unsigned)grid), Narrow<NT>::THREADS, Narrow<NT>::SMEM, a.split > 1 ? a.split : 0, st, map_x, map_w, a);
}

template <int NT>
static int run_narrow(const sapo_fp8& x, const sapo_fp8& w, int32_t K, Fp8GemmArgs a, int sms, cudaStream_t st) {
  a.nt = (int32_t)(a.T < NT ? round_up<int64_t>(a.T, 16) : NT);
  const int64_t num_t = ceil_div<int64_t>(a.T, a.nt), full = ceil_div<int64_t>(a.N, 128) * num_t, rounds = ceil_div<int64_t>(full, sms);
  if (full > 0x7FFFFFFF / 32) return SAPO_ERR_UNSUPPORTED_SHAPE;
  // Thin tiles: as few rows of W as make the last round of CTAs full (151936 rows are 9 rounds of 148 tiles of 115, not 8
  // rounds of 128 and a ninth of 3 tiles).
  const int64_t along_n = rounds * sms / num_t, least = a.nt > 32 ? a.nt : 32;
  const int64_t even = along_n < 1 ? 128 : ceil_div<int64_t>(a.N, along_n), thin = even > 128 ? 128 : (even < least ? least : even);
  // Against them: one round, its tiles shared along K; or, of several rounds, the last one shared so by a second launch.  An
  // SM takes in about 40 KB a us, and not more than a block of K in 0.3; sharing a tile costs 3 us (a cluster's barriers and
  // sums), a second launch 3.5.
  const auto round_us = [&](int64_t rows) { const double us = (double)(rows + a.nt) * 128. / 40e3; return a.num_kb * (us > 0.3 ? us : 0.3); };
  const double thin_us = rounds * round_us(thin);
  const int64_t last = full % sms;
  const int split = split_of(rounds == 1 ? full : last, a.num_kb, sms);
  double shared_us = 1e30;
  if (split > 1) shared_us = rounds == 1 ? round_us(128) / split + 3. : (rounds - 1 + 1. / split) * round_us(128) + 3.5;
  const bool shared = shared_us < thin_us;
  a.rows = (int32_t)(shared ? 128 : thin);
  CUtensorMap map_x, map_w;
  if (!map_rows(&map_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, x.data, K, a.T, a.T == 1 ? round_up<int64_t>(K, 16) : x.ld, a.nt) ||
      !map_rows(&map_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, w.data, K, a.N, a.N == 1 ? round_up<int64_t>(K, 16) : w.ld, a.rows)) return SAPO_ERR_CUDA;
  a.units = (int32_t)(ceil_div<int64_t>(a.N, a.rows) * num_t);
  a.split = shared && rounds == 1 ? split : 1;
  if (!shared || rounds == 1) return launch_narrow<NT>(map_x, map_w, a, sms, st);
  a.units -= (int32_t)last;
  a.tail_follows = 1;
  const int rc = launch_narrow<NT>(map_x, map_w, a, sms, st);
  if (rc != SAPO_OK) return rc;
  a.unit0 = a.units; a.units = (int32_t)last; a.split = split; a.tail_follows = 0; a.tail = 1;
  return launch_narrow<NT>(map_x, map_w, a, sms, st);
}

static int run_wide(const sapo_fp8& x, const sapo_fp8& w, int32_t K, Fp8GemmArgs a, int sms, cudaStream_t st) {
  static bool done[MAX_DEVICES] = {false};
  if (!allow_smem(fp8_wide_kernel, F8W_SMEM, done)) return SAPO_ERR_CUDA;
  const int size = a.out_bf16 ? 2 : 4;
  a.tma_store = aligned16(a.y) && (a.ld_y * size) % 16 == 0;
  CUtensorMap map_x, map_w, map_y;
  if (!map_rows(&map_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, x.data, K, a.T, x.ld, 128) ||
      !map_rows(&map_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, w.data, K, a.N, a.N == 1 ? round_up<int64_t>(K, 16) : w.ld, 128)) return SAPO_ERR_CUDA;
  map_y = map_x;
  if (a.tma_store && !map_rows(&map_y, a.out_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, size, a.y, a.N, a.T,
                               a.ld_y * size, 128)) return SAPO_ERR_CUDA;
  const int64_t num_m = ceil_div<int64_t>(a.T, 256), num_n = ceil_div<int64_t>(a.N, 256), units = num_m * num_n;
  if (units > 0x7FFFFFFF / 8) return SAPO_ERR_UNSUPPORTED_SHAPE;
  a.num_m = (int32_t)num_m; a.num_n = (int32_t)num_n;
  const int64_t fit = (32ll << 20) / ((int64_t)256 * K);                    // token blocks that stay in a part of L2
  a.group_m = (int32_t)(fit < 1 ? 1 : (fit < num_m ? fit : num_m));
  // a last round of at most half the SM pairs is left to narrow tiles, four of a wide one, unless it is short (a second
  // launch takes 3 to 4 us; 14 blocks of K take a wide tile 8)
  const int pairs = sms / 2, rest = (int)(units % pairs);
  const bool tail = units > pairs && rest > 0 && 4 * rest <= sms && a.num_kb >= 14;
  a.units = (int32_t)units - (tail ? rest : 0);
  a.tail_follows = tail;
  {
    KernelScope scope(SAPO_K_FP8_MATMUL, st);
    const int rc = launch_overlapped(fp8_wide_kernel, dim3((unsigned)(2 * (a.units < pairs ? a.units : pairs))), F8W_THREADS, F8W_SMEM, 2, st,
                                     map_x, map_w, map_y, a);
    if (rc != SAPO_OK || !tail) return rc;
  }
  a.unit0 = a.units; a.units = 4 * rest; a.of_wide = 1; a.rows = 128; a.nt = 128; a.tail_follows = 0; a.tail = 1;
  a.split = split_of(a.units, a.num_kb, sms);
  return launch_narrow<128>(map_x, map_w, a, sms, st);
}

static bool usable(const sapo_fp8& m, int64_t rows, int32_t K) {
  return m.data && m.scale && aligned16(m.data) && (reinterpret_cast<uintptr_t>(m.scale) & 3u) == 0 && m.ld >= K &&
         (rows == 1 || m.ld % 16 == 0) && m.ld_scale >= ceil_div<int64_t>(K, 128);
}

}  // namespace sapo

extern "C" int sapo_fp8_matmul(const sapo_fp8* h_x, int64_t T, const sapo_fp8* h_w, int32_t N, int32_t K, void* y, int32_t y_dtype,
                               int64_t ld_y, int32_t* status, void* stream) {
  using namespace sapo;
  if (!h_x || !h_w || !status || T < 0 || N < 1 || K < 1 || ld_y < N || (y_dtype != SAPO_DTYPE_BF16 && y_dtype != SAPO_DTYPE_F32)) return SAPO_ERR_INVALID_ARG;
  if (h_x->blocks != 0 || h_w->blocks != 1) return SAPO_ERR_INVALID_ARG;
  if (T == 0) return SAPO_OK;
  if (T > 0x7FFFFF00 || N > 0x7FFFFF00 || K > (1 << 24)) return SAPO_ERR_UNSUPPORTED_SHAPE;
  if (!y || reinterpret_cast<uintptr_t>(y) % (y_dtype == SAPO_DTYPE_BF16 ? 2 : 4) || !usable(*h_x, T, K) || !usable(*h_w, N, K)) return SAPO_ERR_INVALID_ARG;
  const int sms = sm_count();
  if (sms <= 0) return SAPO_ERR_CUDA;
  Fp8GemmArgs a{};
  a.sx = h_x->scale; a.ld_sx = h_x->ld_scale; a.sw = h_w->scale; a.ld_sw = h_w->ld_scale;
  a.y = y; a.ld_y = ld_y; a.T = T; a.N = N; a.num_kb = ceil_div(K, 128); a.out_bf16 = y_dtype == SAPO_DTYPE_BF16;
  a.wait_limit = WAIT_LIMIT_CLOCKS; a.status = status; a.split = 1; a.group_m = 1;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (T > 128 && ceil_div<int64_t>(T, 256) * ceil_div<int64_t>(N, 256) >= sms / 4) return run_wide(*h_x, *h_w, K, a, sms, st);
  if (T <= 16) return run_narrow<16>(*h_x, *h_w, K, a, sms, st);
  if (T <= 32) return run_narrow<32>(*h_x, *h_w, K, a, sms, st);
  if (T <= 64) return run_narrow<64>(*h_x, *h_w, K, a, sms, st);
  return run_narrow<128>(*h_x, *h_w, K, a, sms, st);
}
