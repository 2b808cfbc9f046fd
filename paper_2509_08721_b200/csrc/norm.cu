// The norm in front of the LM head (layer norm or RMS norm), forward and backward, and activation
// checkpoints in 8 bits: sapo_norm_fwd, sapo_norm_replay, sapo_norm_bwd, sapo_ckpt8_store,
// sapo_ckpt8_restore.  All of them pass over [T, H] once.  Host side and C ABI; the kernels are in norm_rows.cuh
// (rows that can be copied 16 bytes at a time) and norm_any.cuh (all others, and short rows).
#include "norm_any.cuh"
#include "norm_rows.cuh"

namespace sapo {

// ---------------------------------------------------------------------------- host side
// Rows through shared memory: whole vectors of 8 columns, more of them than one 16-thread group has, rows
// (and weights) on 16-byte boundaries.
static bool ring_ok(int32_t H, bool vec, bool w_vec, int least) { return vec && w_vec && H > least && H % 8 == 0; }
// Columns up to which norm_any.cuh's kernels were faster (120 million columns of bf16; 200 a row: forward 134 us there and
// 170 us here, backward 131 us here)
constexpr int FWD_RING_ABOVE = 256, BWD_RING_ABOVE = 128;
struct RingPlan { int wpr, vpl, threads, rows_per_block; };
// At most 4 vectors a thread up to 8192 columns: a row is then in fewer places of memory at a time (with a whole row of
// 1536 columns per warp, 16 rows an SM, the forward takes 167 us for 146382 of them, with two warps a row 152), while
// the row's sums cross few enough warps (2 vectors a thread: 235).
static RingPlan fwd_ring_plan(int32_t H) {
  const int nvec = ceil_div(H, 8);
  RingPlan p;
  p.wpr = 1;
  while (p.wpr < 8 && p.wpr * 32 * 4 < nvec) p.wpr <<= 1;
  p.vpl = ceil_div(nvec, p.wpr * 32);
  if (p.vpl > 4) p.vpl = 8;
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

constexpr int RING_TOO_WIDE = 1;         // rows and weights do not fit: norm_fwd_any_kernel takes them
template <class TX, int VPL, bool FULL>
static int launch_fwd_ring_full(const NormFwdArgs& a, const RingPlan& p, int sms, cudaStream_t st) {
  // (by the width of the row in 256 columns, which the weights' share of shared memory follows)
  static int cache[NORM_MAX_H / 256 + 1][MAX_DEVICES] = {{0}};
  auto kernel = norm_fwd_ring_kernel<TX, VPL, FULL>;
  const int steps = ceil_div(a.H, 256);
  const size_t smem = FwdRing<TX, VPL>::smem(steps * 256);
  if (smem > SMEM_MAX) return RING_TOO_WIDE;
  const int per_sm = resident_blocks(kernel, p.threads, smem, cache[steps]);
  if (per_sm == 0) return SAPO_ERR_CUDA;
  int64_t blocks = ceil_div<int64_t>(a.T, p.rows_per_block);
  if (blocks > (int64_t)sms * per_sm) blocks = (int64_t)sms * per_sm;
  KernelScope scope(SAPO_K_NORM_FWD, st);
  return launch_overlapped(kernel, dim3((unsigned)blocks), p.threads, smem, 0, st, a, p.wpr);
}
// FULL: the row's last warp has all its columns too, so that nothing is predicated.  (With 8 vectors a thread that is
// the widest row only, which does not fit in fp32.)
template <class TX, int VPL>
static int launch_fwd_ring_vpl(const NormFwdArgs& a, const RingPlan& p, int sms, cudaStream_t st) {
  if constexpr (VPL < 8 || FwdRing<TX, VPL>::smem(NORM_MAX_H) <= SMEM_MAX) {
    if (a.H == p.wpr * VPL * 256) return launch_fwd_ring_full<TX, VPL, true>(a, p, sms, st);
  }
  return launch_fwd_ring_full<TX, VPL, false>(a, p, sms, st);
}
template <class TX>
static int launch_fwd_ring(const NormFwdArgs& a, int sms, cudaStream_t st) {
  const RingPlan p = fwd_ring_plan(a.H);
  switch (p.vpl) {                         // (rows of more than FWD_RING_ABOVE columns: two vectors at least)
    case 2: return launch_fwd_ring_vpl<TX, 2>(a, p, sms, st);
    case 3: return launch_fwd_ring_vpl<TX, 3>(a, p, sms, st);
    case 4: return launch_fwd_ring_vpl<TX, 4>(a, p, sms, st);
    default: return launch_fwd_ring_vpl<TX, 8>(a, p, sms, st);
  }
}

// launch == false: only how many blocks of the plan an SM holds (0: this form does not exist)
template <class TX, class TDY, int VPL, int MAX_THREADS, int SLOTS, bool FULL>
static int bwd_ring_full(const NormBwdArgs& a, const RingPlan& p, int blocks, bool launch, cudaStream_t st) {
  using Ring = BwdRing<TX, TDY, VPL, MAX_THREADS>;
  if constexpr (!Ring::FITS) {
    return launch ? SAPO_ERR_CUDA : 0;
  } else {
    static int cache[33][MAX_DEVICES] = {{0}};                       // by warps of the block
    auto kernel = norm_bwd_ring_kernel<TX, TDY, VPL, MAX_THREADS, SLOTS, FULL>;
    const size_t smem = (size_t)Ring::STAGES * (p.threads / 32) * Ring::WARP_BYTES;
    if (!launch) return resident_blocks(kernel, p.threads, smem, cache[p.threads / 32]);
    KernelScope scope(SAPO_K_NORM_BWD, st);
    return launch_overlapped(kernel, dim3((unsigned)blocks), p.threads, smem, 0, st, a, p.wpr);
  }
}
template <class TX, class TDY, int VPL, int MAX_THREADS, int SLOTS>
static int bwd_ring_vpl(const NormBwdArgs& a, const RingPlan& p, int blocks, bool launch, cudaStream_t st) {
  return a.H == p.wpr * VPL * 256 ? bwd_ring_full<TX, TDY, VPL, MAX_THREADS, SLOTS, true>(a, p, blocks, launch, st)
                                  : bwd_ring_full<TX, TDY, VPL, MAX_THREADS, SLOTS, false>(a, p, blocks, launch, st);
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

// How norm_any.cuh's kernels take a row.  `lanes`: of a row in Vector form (rows of up to 256 columns in whole vectors on
// 16-byte boundaries), or 0: `e` columns a lane, `wpr` warps a row.
struct AnyPlan { int lanes, e, wpr, threads, rows_per_block; };
static AnyPlan any_plan(int32_t H, bool vec, bool backward) {
  AnyPlan p;
  p.lanes = !vec || H % 8 != 0 || H > 256 ? 0 : (H <= 32 ? 4 : (H <= 64 ? 8 : (H <= 128 ? 16 : 32)));
  p.e = H <= 128 ? 4 : (H <= 8192 ? 16 : 32);
  p.wpr = ceil_div(H, 32 * p.e);
  const int groups = p.wpr >= 8 ? 1 : 8 / p.wpr;
  p.threads = p.wpr * groups * 32;
  // rows a lane takes at a time, and rows of a warp
  const int u = p.lanes != 0 ? (backward && p.lanes == 4 ? 2 : 4) : (p.e == 4 ? (backward ? 4 : 8) : (p.e == 16 && p.wpr <= 4 && !backward ? 2 : 1));
  p.rows_per_block = groups * u * (p.lanes != 0 ? 32 / p.lanes : 1);
  return p;
}
// whether rows start on boundaries of two elements
static bool pairs_ok(const Mat& m) { return (reinterpret_cast<uintptr_t>(m.p) & (2 * esize(m.dtype) - 1)) == 0 && m.ld % 2 == 0; }
static bool pairs_ok(const Q8Mat& q) { return (reinterpret_cast<uintptr_t>(q.p) & 1u) == 0 && q.ld % 2 == 0; }

template <class TX, class A, int U>
static int launch_fwd_any_shape(const NormFwdArgs& a, const AnyPlan& p, int sms, cudaStream_t st) {
  static int cache[NORM_MAX_THREADS / 32 + 1][MAX_DEVICES] = {{0}};
  auto kernel = norm_fwd_any_kernel<TX, A, U>;
  const int per_sm = resident_blocks(kernel, p.threads, 0, cache[p.threads / 32]);
  if (per_sm == 0) return SAPO_ERR_CUDA;
  int64_t blocks = ceil_div<int64_t>(a.T, p.rows_per_block);
  if (blocks > (int64_t)sms * per_sm) blocks = (int64_t)sms * per_sm;
  KernelScope scope(SAPO_K_NORM_FWD, st);
  return launch_overlapped(kernel, dim3((unsigned)blocks), p.threads, 0, 0, st, a, p.wpr);
}
template <class TX, int W>
static int launch_fwd_any_w(const NormFwdArgs& a, const AnyPlan& p, int sms, cudaStream_t st) {
  if (p.e == 4) return launch_fwd_any_shape<TX, Cols<W, 4>, 8>(a, p, sms, st);
  if (p.e == 16 && p.wpr <= 4) return launch_fwd_any_shape<TX, Cols<W, 16>, 2>(a, p, sms, st);
  if (p.e == 16) return launch_fwd_any_shape<TX, Cols<W, 16>, 1>(a, p, sms, st);
  return launch_fwd_any_shape<TX, Cols<W, 32>, 1>(a, p, sms, st);
}
template <class TX>
static int launch_fwd_any(const NormFwdArgs& a, const AnyPlan& p, bool pairs, int sms, cudaStream_t st) {
  if (p.lanes == 4) return launch_fwd_any_shape<TX, Vector<4>, 4>(a, p, sms, st);
  if (p.lanes == 8) return launch_fwd_any_shape<TX, Vector<8>, 4>(a, p, sms, st);
  if (p.lanes == 16) return launch_fwd_any_shape<TX, Vector<16>, 4>(a, p, sms, st);
  if (p.lanes == 32) return launch_fwd_any_shape<TX, Vector<32>, 4>(a, p, sms, st);
  return pairs ? launch_fwd_any_w<TX, 2>(a, p, sms, st) : launch_fwd_any_w<TX, 1>(a, p, sms, st);
}
// replay: x comes from the checkpoint
static int launch_fwd(const NormFwdArgs& a, bool replay, cudaStream_t st) {
  if (a.T == 0) return SAPO_OK;
  const int sms = sm_count();
  if (sms <= 0) return SAPO_ERR_CUDA;
  const bool held = a.q.p != nullptr;
  const bool vec = (replay || vec_ok(a.x)) && vec_ok(a.y) && (!held || vec_ok(a.q));
  if (ring_ok(a.H, vec, aligned16(a.gamma) && aligned16(a.beta), FWD_RING_ABOVE)) {
    const int rc = replay ? launch_fwd_ring<int8_t>(a, sms, st)
                          : (a.x.dtype == SAPO_DTYPE_F32 ? launch_fwd_ring<float>(a, sms, st) : launch_fwd_ring<__nv_bfloat16>(a, sms, st));
    if (rc != RING_TOO_WIDE) return rc;
  }
  const bool pairs = a.H % 2 == 0 && (replay || pairs_ok(a.x)) && pairs_ok(a.y) && (!held || pairs_ok(a.q));
  const AnyPlan p = any_plan(a.H, vec, false);
  if (replay) return launch_fwd_any<int8_t>(a, p, pairs, sms, st);
  return a.x.dtype == SAPO_DTYPE_F32 ? launch_fwd_any<float>(a, p, pairs, sms, st) : launch_fwd_any<__nv_bfloat16>(a, p, pairs, sms, st);
}

template <class TX, class A, int U>
static int launch_bwd_any_shape(const NormBwdArgs& a, const AnyPlan& p, int blocks, cudaStream_t st) {
  const int groups = p.threads / 32 / p.wpr;
  const size_t smem = groups > 1 ? (size_t)groups * 2 * a.H * sizeof(float) : 0;      // 8 warps with up to 512 columns each: 32 KB
  KernelScope scope(SAPO_K_NORM_BWD, st);
  return launch_overlapped(norm_bwd_any_kernel<TX, A, U>, dim3((unsigned)blocks), p.threads, smem, 0, st, a, p.wpr);
}
template <class TX, int W>
static int launch_bwd_any_w(const NormBwdArgs& a, const AnyPlan& p, int blocks, cudaStream_t st) {
  if (p.e == 4) return launch_bwd_any_shape<TX, Cols<W, 4>, 4>(a, p, blocks, st);
  if (p.e == 16) return launch_bwd_any_shape<TX, Cols<W, 16>, 1>(a, p, blocks, st);
  return launch_bwd_any_shape<TX, Cols<W, 32>, 1>(a, p, blocks, st);
}
template <class TX>
static int launch_bwd_any(const NormBwdArgs& a, const AnyPlan& p, bool pairs, int blocks, cudaStream_t st) {
  if (p.lanes == 4) return launch_bwd_any_shape<TX, Vector<4>, 2>(a, p, blocks, st);
  if (p.lanes == 8) return launch_bwd_any_shape<TX, Vector<8>, 4>(a, p, blocks, st);
  if (p.lanes == 16) return launch_bwd_any_shape<TX, Vector<16>, 4>(a, p, blocks, st);
  if (p.lanes == 32) return launch_bwd_any_shape<TX, Vector<32>, 4>(a, p, blocks, st);
  return pairs ? launch_bwd_any_w<TX, 2>(a, p, blocks, st) : launch_bwd_any_w<TX, 1>(a, p, blocks, st);
}

// One launch of a checkpoint kernel: `units` pieces of work of a warp, `per_row` of them a row (or a set of rows), `n` at a time.
template <class Launch, class Kernel>
static int launch_ckpt8_warps(Kernel kernel, int64_t units, int32_t per_row, int n, int* cache, int sms, Launch launch) {
  const int per_sm = resident_blocks(kernel, 256, 0, cache);
  if (per_sm == 0) return SAPO_ERR_CUDA;
  int64_t blocks = ceil_div<int64_t>(units, (int64_t)8 * n);
  if (blocks > (int64_t)sms * per_sm) blocks = (int64_t)sms * per_sm;
  return launch(dim3((unsigned)blocks), blocks * 8 / per_row, (int32_t)(blocks * 8 % per_row));
}
template <class TX, int L, int N, bool RESTORE>
static int launch_ckpt8_rows(const Ckpt8Args& a, int sms, cudaStream_t st) {
  static int cache[MAX_DEVICES] = {0};
  auto kernel = ckpt8_rows_kernel<TX, L, N, RESTORE>;
  const int32_t segments = L == 32 ? ceil_div(a.H, N * 256) : 1;
  const int64_t units = ceil_div<int64_t>(a.T, L == 32 ? 1 : N * (32 / L)) * segments;
  KernelScope scope(SAPO_K_CKPT8, st);
  return launch_ckpt8_warps(kernel, units, segments, 1, cache, sms, [&](dim3 blocks, int64_t rows, int32_t segs) {
    return launch_overlapped(kernel, blocks, 256, 0, 0, st, a, segments, rows, segs);
  });
}
template <class TX, int W, bool RESTORE>
static int launch_ckpt8_any(const Ckpt8Args& a, int sms, cudaStream_t st) {
  static int cache[MAX_DEVICES] = {0};
  auto kernel = ckpt8_any_kernel<TX, W, RESTORE>;
  const int32_t groups = ceil_div(a.H, Q8_GROUP);
  KernelScope scope(SAPO_K_CKPT8, st);
  return launch_ckpt8_warps(kernel, a.T * groups, groups, CkptAny<RESTORE>::GROUPS, cache, sms, [&](dim3 blocks, int64_t rows, int32_t g) {
    return launch_overlapped(kernel, blocks, 256, 0, 0, st, a, rows, g);
  });
}
template <class TX, bool RESTORE>
static int launch_ckpt8(const Ckpt8Args& a, int sms, cudaStream_t st) {
  if (a.H % 8 == 0 && vec_ok(a.x) && vec_ok(a.q)) {
    if (a.H <= 32) return launch_ckpt8_rows<TX, 4, RESTORE ? 2 : 4, RESTORE>(a, sms, st);
    if (a.H <= 64) return launch_ckpt8_rows<TX, 8, RESTORE ? 2 : 4, RESTORE>(a, sms, st);
    if (a.H <= 128) return launch_ckpt8_rows<TX, 16, RESTORE ? 2 : 4, RESTORE>(a, sms, st);
    // vectors a lane takes of a row: up to 4 (2 on the way back), as many as leave the fewest of the row's last segment unused
    const int steps = ceil_div(a.H, 256), segments = ceil_div(steps, RESTORE ? 2 : 4), n = ceil_div(steps, segments);
    if constexpr (!RESTORE) {
      if (n == 3) return launch_ckpt8_rows<TX, 32, 3, RESTORE>(a, sms, st);
      if (n == 4) return launch_ckpt8_rows<TX, 32, 4, RESTORE>(a, sms, st);
    }
    return n == 1 ? launch_ckpt8_rows<TX, 32, 1, RESTORE>(a, sms, st) : launch_ckpt8_rows<TX, 32, 2, RESTORE>(a, sms, st);
  }
  if (a.H % 2 == 0 && pairs_ok(a.x) && pairs_ok(a.q)) return launch_ckpt8_any<TX, 2, RESTORE>(a, sms, st);
  return launch_ckpt8_any<TX, 1, RESTORE>(a, sms, st);
}
template <bool RESTORE>
static int launch_ckpt8_x(const Ckpt8Args& a, cudaStream_t st) {
  if (a.T == 0) return SAPO_OK;
  const int sms = sm_count();
  if (sms <= 0) return SAPO_ERR_CUDA;
  return a.x.dtype == SAPO_DTYPE_F32 ? launch_ckpt8<float, RESTORE>(a, sms, st) : launch_ckpt8<__nv_bfloat16, RESTORE>(a, sms, st);
}

long long bounds_violations_norm() { return read_bounds_violations(); }
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
  return launch_fwd(NormFwdArgs{mx, my, q8_of(h_ckpt), gamma, beta, h_cfg->w_dtype, h_cfg->kind, h_cfg->eps, mean, rstd, T, H,
                                status}, false, static_cast<cudaStream_t>(stream));
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
  return launch_fwd(NormFwdArgs{Mat{nullptr, 0, SAPO_DTYPE_BF16}, my, q8_of(h_x), gamma, beta, h_cfg->w_dtype, h_cfg->kind, 0.f,
                                const_cast<float*>(mean), const_cast<float*>(rstd), T, H, nullptr}, true,
                    static_cast<cudaStream_t>(stream));
}

extern "C" size_t sapo_norm_workspace_bytes(int64_t T, int32_t H) {
  using namespace sapo;
  if (dims_check(T, H) != SAPO_OK) return 0;
  int sms = sm_count();
  if (sms <= 0) sms = 148;
  // the larger of what the forms of the kernel take, whatever the alignment of the rows will be
  const int few = any_plan(H, true, true).rows_per_block, fewer = any_plan(H, false, true).rows_per_block;
  int64_t blocks = bwd_blocks(T > 0 ? T : 1, few < fewer ? few : fewer, 2, sms);
  const int64_t ring = bwd_blocks(T > 0 ? T : 1, bwd_ring_plan(H).rows_per_block, 2, sms);
  if (ring > blocks) blocks = ring;
  return round_up<size_t>((size_t)blocks * 2 * part_pitch(H) * sizeof(float), 256);
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
  const NormBwdArgs a{mdy, mx, mdx, q8_of(h_ckpt), gamma, h_cfg->w_dtype, h_cfg->kind, mean, rstd, T, H,
                      static_cast<float*>(workspace), dgamma, dbeta, accumulate};
  const AnyPlan p = any_plan(H, vec, true);
  const RingPlan rp = bwd_ring_plan(H);
  const int resident = ring_ok(H, vec, aligned16(gamma), BWD_RING_ABOVE) ? bwd_ring(a, rp, 0, false, st) : 0;
  const bool ring = resident > 0;
  const int blocks = (int)bwd_blocks(T, ring ? rp.rows_per_block : p.rows_per_block, ring && resident < 2 ? resident : 2, sms);
  if (reduce && blocks > 1) {
    if (!workspace || !aligned16(workspace)) return SAPO_ERR_INVALID_ARG;
    if (workspace_bytes < (size_t)blocks * 2 * part_pitch(H) * sizeof(float)) return SAPO_ERR_WORKSPACE_TOO_SMALL;
  }
  const bool pairs = H % 2 == 0 && pairs_ok(mdy) && pairs_ok(mdx) && (h_ckpt ? pairs_ok(a.q) : pairs_ok(mx));
  if (ring) rc = bwd_ring(a, rp, blocks, true, st);
  else if (h_ckpt) rc = launch_bwd_any<int8_t>(a, p, pairs, blocks, st);
  else rc = x_dtype == SAPO_DTYPE_F32 ? launch_bwd_any<float>(a, p, pairs, blocks, st) : launch_bwd_any<__nv_bfloat16>(a, p, pairs, blocks, st);
  if (rc != SAPO_OK || !reduce || blocks == 1) return rc;
  KernelScope scope(SAPO_K_NORM_REDUCE, st);
  return launch_overlapped(norm_reduce_kernel, dim3((unsigned)ceil_div(H, 32), dgamma && dbeta ? 2 : 1), REDUCE_WARPS * 32, 0, 0, st, a.part, blocks, H, dgamma, dbeta, accumulate);
}

extern "C" int sapo_ckpt8_store(const void* x, int32_t x_dtype, int64_t T, int32_t H, int64_t ld_x,
                                const sapo_ckpt8* h_out, int32_t* status, void* stream) {
  using namespace sapo;
  int rc = dims_check(T, H);
  if (rc != SAPO_OK) return rc;
  const Mat mx{const_cast<void*>(x), ld_x, x_dtype};
  if ((rc = mat_check(mx, T, H)) != SAPO_OK || (rc = ckpt_check(h_out, T, H)) != SAPO_OK) return rc;
  if (!status) return SAPO_ERR_INVALID_ARG;
  return launch_ckpt8_x<false>(Ckpt8Args{mx, q8_of(h_out), T, H, status}, static_cast<cudaStream_t>(stream));
}

extern "C" int sapo_ckpt8_restore(const sapo_ckpt8* h_in, int64_t T, int32_t H, void* x, int32_t x_dtype,
                                  int64_t ld_x, void* stream) {
  using namespace sapo;
  int rc = dims_check(T, H);
  if (rc != SAPO_OK) return rc;
  const Mat mx{x, ld_x, x_dtype};
  if ((rc = mat_check(mx, T, H)) != SAPO_OK || (rc = ckpt_check(h_in, T, H)) != SAPO_OK) return rc;
  return launch_ckpt8_x<true>(Ckpt8Args{mx, q8_of(h_in), T, H, nullptr}, static_cast<cudaStream_t>(stream));
}
