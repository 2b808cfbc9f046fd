// sapo_preference_loss: a preference loss over the completions of a question, from per-token
// log-probs to the gradient factor of every token.
//   R_s = sum over the tokens of s of (logp - ref_logp)   (divided by T_s with length_norm)
//   pairs (i, j) of one question, i preferred to j (reward_i > reward_j);  h = beta (R_i - R_j)
//   loss = 1/Q sum_q 1/n_q sum_pairs l(h)
// A question's completions are neighbours in the packed batch, so a question is one cluster's work:
// the sums of its sequences, its pairs, and one factor per sequence written to all its tokens.
// Reads 8 bytes and writes 4 per token.
#include <math.h>

#include <atomic>

#include "preference.cuh"

namespace sapo {

constexpr int PREF_THREADS = 512;
constexpr int PREF_WARPS = PREF_THREADS / 32;
constexpr int PREF_MAX_CLUSTER = 16;
constexpr int PREF_SEQS = 1024;          // completions of a question whose sums are kept in shared memory

__device__ __forceinline__ int32_t clamp_to(int32_t x, int32_t hi, bool& bad) {
  const int32_t c = x < 0 ? 0 : (x > hi ? hi : x);
  bad |= c != x;
  return c;
}

// [a, b) = offsets[i], offsets[i+1], clamped to [0, hi] and to a <= b; `bad` says whether they had to be
__device__ __forceinline__ void offset_range(const int32_t* offsets, int32_t i, int32_t hi, int32_t& a, int32_t& b, bool& bad) {
  a = clamp_to(offsets[i], hi, bad);
  b = clamp_to(offsets[i + 1], hi, bad);
  if (b < a) { b = a; bad = true; }
}

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
// all threads of the cluster; orders their shared and global memory accesses
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_barrier() { cluster_arrive(); cluster_wait(); }
// *p = x in the shared memory of the cluster's first block
__device__ __forceinline__ void store_to_first(float* p, float x) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(x) : "memory");
}

template <class T>
__device__ __forceinline__ T warp_sum(T x) {
  #pragma unroll
  for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  return x;
}

// value and derivative (by h) of one pair's loss
__device__ __forceinline__ void pair_loss(const PrefArgs& a, float h, float& l, float& dl) {
  if (a.kind == SAPO_PREF_SIGMOID) {
    // softplus(-h) and softplus(h) = softplus(-h) + h;  sigma(h) without overflow on either side
    const float e = expf(-fabsf(h));
    const float sp = log1pf(e);
    const float sig = (h >= 0.f ? 1.f : e) / (1.f + e);
    const float neg = (h >= 0.f ? e : 1.f) / (1.f + e);       // 1 - sigma(h)
    l = (1.f - a.smoothing) * (fmaxf(-h, 0.f) + sp) + a.smoothing * (fmaxf(h, 0.f) + sp);
    dl = a.smoothing * sig - (1.f - a.smoothing) * neg;
  } else if (a.kind == SAPO_PREF_SQUARED) {
    const float u = (h - 0.5f) / a.beta;                      // R_i - R_j - 1 / (2 beta)
    l = u * u;
    dl = 2.f * u / a.beta;
  } else {
    l = fmaxf(1.f - h, 0.f);
    dl = h < 1.f ? -1.f : 0.f;
  }
}

// log ratio of token t, NaN or infinite where the token is masked
__device__ __forceinline__ float token_ratio(const PrefArgs& a, int32_t t) {
  if (!SAPO_IN_BOUNDS(t >= 0 && t < a.T)) return NAN;
  return a.ref_logp != nullptr ? a.logp[t] - a.ref_logp[t] : a.logp[t];
}

__device__ __forceinline__ float load_from_first(const float* p) {
  uint32_t at;
  float x;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
  return x;
}

// Mean of the questions' losses, added up in their order by one warp.
__device__ __forceinline__ void mean_loss(const float* q_loss, int32_t Q, float* loss, int lane) {
  double x = 0.0;
  for (int32_t q = lane; q < Q; q += 32) x += (double)__ldcg(q_loss + q);
  x = warp_sum(x);
  if (lane == 0) *loss = (float)(x / (double)Q);
}

// A cluster of blocks per question.  The question's tokens are one range, cut into equal pieces for the
// cluster's warps whatever its sequences' lengths are, so that few long sequences keep as many SMs
// busy as many short ones:
//   1. every warp sums the pieces of sequences in its range.  The piece with which the range begins goes
//      to `head` of the first block; any other piece holds its sequence's first token, and goes to
//      seq_logratio[s]
//   2. the first block adds up each sequence's pieces (in order), then the pairs: a warp per completion,
//      lanes over the others
//   3. every warp writes the factors of its tokens
// A small batch is a chain of waits for memory (each about half a microsecond), so a question's offsets and
// rewards are read into shared memory at once, and what passes between the steps stays there, for questions of
// up to PREF_SEQS completions.
// Bound by those waits, not by its 12 bytes a token: 4 questions x 8 completions 6.0 us (the call's host side takes 8.5),
// 64 x 8 completions of 640 tokens 10.2 us, 2 questions of 105000 tokens 10.3 us (389 with a block per question), 512 x 8
// of 600 tokens 22 us.
template <bool SOLO>
__global__ void __launch_bounds__(PREF_THREADS) preference_kernel(PrefArgs a) {
  // Another block's shared memory may only be accessed once that block has started, which being scheduled together
  // does not say: every block of a cluster arrives here, and waits for the others before its first store to the first
  // block.  The wait for the kernel before this one lies in between, so it costs nothing that was measured.
  if (!SOLO) cluster_arrive();
  wait_for_previous();
  let_next_start();
  if (!SOLO) cluster_wait();
  __shared__ float head[PREF_MAX_CLUSTER * PREF_WARPS];
  __shared__ int32_t cu_s[PREF_SEQS + 1];
  __shared__ float R_s[PREF_SEQS], r_s[PREF_SEQS], g_s[PREF_SEQS];     // sums, rewards, factors
  __shared__ float sums[2][PREF_WARPS];
  __shared__ int32_t counts[PREF_WARPS];
  __shared__ float scale_s;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t Tc = (int32_t)a.T;
  // SOLO: the grid is one cluster whose blocks take questions each by itself, and the first adds up the losses
  const int rank = SOLO ? 0 : (int)cluster_rank(), size = SOLO ? 1 : (int)cluster_size();
  const int gw = rank * PREF_WARPS + warp, n_warps = size * PREF_WARPS;
  const int32_t cluster = (int32_t)(blockIdx.x / size);
  auto team_barrier = [] { if (SOLO) __syncthreads(); else cluster_barrier(); };
  auto to_first = [](float* p, float x) { if (SOLO) *p = x; else store_to_first(p, x); };
  bool bad_offset = false, bad_value = false, bad_reward = false;
  if (cluster >= a.q_clusters) {
    // the clusters behind those of the questions: what no question covers, sequences before the first and after the
    // last one and their tokens, gets zeros
    bool ignore = false;
    const int32_t s_lo = clamp_to(a.group_offsets[0], a.S, ignore);
    int32_t s_hi = clamp_to(a.group_offsets[a.Q], a.S, ignore);
    if (s_hi < s_lo) s_hi = s_lo;
    const int32_t t_lo = clamp_to(a.cu[s_lo], Tc, ignore);
    int32_t t_hi = clamp_to(a.cu[s_hi], Tc, ignore);
    if (t_hi < t_lo) t_hi = t_lo;
    const int64_t skip = (int64_t)a.q_clusters * size;
    const int64_t first = (blockIdx.x - skip) * PREF_THREADS + threadIdx.x, step = (gridDim.x - skip) * PREF_THREADS;
    for (int64_t i = first; i < (int64_t)t_lo + (Tc - t_hi); i += step) {
      const int64_t t = i < t_lo ? i : t_hi + (i - t_lo);
      if (SAPO_IN_BOUNDS(t >= 0 && t < a.T)) a.gscale[t] = 0.f;
    }
    for (int64_t i = first; i < (int64_t)s_lo + (a.S - s_hi); i += step) {
      const int64_t s = i < s_lo ? i : s_hi + (i - s_lo);
      if (!SAPO_IN_BOUNDS(s >= 0 && s < a.S)) continue;
      a.seq_logratio[s] = 0.f;
      a.seq_grad[s] = 0.f;
    }
    if (!SOLO) return;
  }
  for (int32_t q = cluster; q < a.Q; q += a.q_clusters) {
    int32_t s0, s1;
    offset_range(a.group_offsets, q, a.S, s0, s1, bad_offset);
    const bool kept = s1 - s0 <= PREF_SEQS;
    if (kept) {
      // (the previous question's readers are behind the barrier that ended its step 2, or read their own block's)
      __syncthreads();
      for (int32_t i = threadIdx.x; i <= s1 - s0; i += PREF_THREADS) {
        if (!SAPO_IN_BOUNDS(s0 >= 0 && s0 + i <= a.S && i <= PREF_SEQS)) continue;
        cu_s[i] = a.cu[s0 + i];
        if (i < s1 - s0) r_s[i] = a.rewards[s0 + i];
      }
      __syncthreads();
    }
    const int32_t* cu = kept ? cu_s - s0 : a.cu;             // indexed by sequence
    const int32_t ta = clamp_to(cu[s0], Tc, bad_offset);
    int32_t tb = clamp_to(cu[s1], Tc, bad_offset);
    if (tb < ta) tb = ta;
    // tokens per warp: whole steps of 32
    const int32_t piece = (int32_t)round_up<int64_t>(ceil_div<int64_t>((int64_t)tb - ta, n_warps), 32) + (tb == ta ? 32 : 0);
    const int64_t begin64 = (int64_t)ta + (int64_t)gw * piece;
    const int32_t begin = begin64 < tb ? (int32_t)begin64 : tb;
    const int32_t end = begin64 + piece < tb ? (int32_t)(begin64 + piece) : tb;
    // the sequence of the range's first token: the first one that ends behind it
    int32_t s_first = s0;
    if (begin < end) {
      int32_t lo = s0, hi = s1;
      while (lo < hi) { const int32_t mid = lo + ((hi - lo) >> 1); if (cu[mid + 1] > begin) hi = mid; else lo = mid + 1; }
      s_first = lo;
    }
    bool masked = false;                       // a token of this lane's in the range is masked
    // 1.
    if (begin < end) {
      for (int32_t s = s_first; s < s1; ++s) {
        int32_t t0, t1;
        offset_range(cu, s, Tc, t0, t1, bad_offset);
        if (t0 >= end) break;
        const int32_t from = t0 > begin ? t0 : begin, to = t1 < end ? t1 : end;
        if (from >= to) continue;
        float part[4] = {0.f, 0.f, 0.f, 0.f};
        int32_t t = from + lane;
        for (; t + 96 < to; t += 128) {
          float d[4];
          #pragma unroll
          for (int k = 0; k < 4; ++k) d[k] = token_ratio(a, t + 32 * k);
          #pragma unroll
          for (int k = 0; k < 4; ++k) { if (isfinite(d[k])) part[k] += d[k]; else masked = true; }
        }
        for (; t < to; t += 32) {
          const float d = token_ratio(a, t);
          if (isfinite(d)) part[0] += d; else masked = true;
        }
        const float sum = warp_sum((part[0] + part[1]) + (part[2] + part[3]));
        if (lane == 0 && SAPO_IN_BOUNDS(gw < PREF_MAX_CLUSTER * PREF_WARPS && s >= 0 && s < a.S)) {
          if (t0 <= begin) to_first(&head[gw], sum);
          else if (kept) to_first(&R_s[s - s0], sum);
          else a.seq_logratio[s] = sum;
        }
      }
    }
    bad_value |= masked;
    team_barrier();
    // 2.
    if (rank == 0) {
      for (int32_t s = s0 + warp; s < s1; s += PREF_WARPS) {
        int32_t t0, t1;
        offset_range(cu, s, Tc, t0, t1, bad_offset);
        const int32_t n = t1 - t0;
        float R = 0.f;
        if (n > 0) {
          // its pieces: the first where it begins (in R_s unless it begins a range), then the heads of the
          // ranges that it runs into.  (Malformed offsets, reported above, could point outside the ranges.)
          const int32_t w0 = t0 < ta ? 0 : (t0 - ta) / piece;
          int32_t w1 = t1 <= ta ? 0 : (t1 - 1 - ta) / piece;
          if (w1 >= n_warps) w1 = n_warps - 1;
          const bool inside = t0 - ta > w0 * piece;
          float x = 0.f;
          for (int32_t w = w0 + (inside ? 1 : 0) + lane; w <= w1; w += 32)
            if (SAPO_IN_BOUNDS(w >= 0 && w < n_warps)) x += head[w];
          R = warp_sum(x) + (inside ? (kept ? R_s[s - s0] : __ldcg(a.seq_logratio + s)) : 0.f);
          if (a.length_norm) R /= (float)n;
        }
        __syncwarp();
        if (lane == 0 && SAPO_IN_BOUNDS(s >= 0 && s < a.S)) {
          const float r = kept ? r_s[s - s0] : a.rewards[s];
          if (!isfinite(r)) bad_reward = true;
          a.seq_logratio[s] = R;
          // a completion takes part if it has a token and a finite reward
          if (kept) { R_s[s - s0] = R; r_s[s - s0] = n > 0 && isfinite(r) ? r : NAN; }
        }
      }
      __syncthreads();
      auto reward_of = [&](int32_t s) {          // NaN: takes no part, and compares as neither more nor less
        if (kept) return r_s[s - s0];
        bool ignore = false;
        int32_t t0, t1;
        offset_range(cu, s, Tc, t0, t1, ignore);
        const float r = a.rewards[s];
        return t1 > t0 && isfinite(r) ? r : NAN;
      };
      auto ratio_of = [&](int32_t s) { return kept ? R_s[s - s0] : __ldcg(a.seq_logratio + s); };
      int32_t best = -1, worst = -1;
      if (a.pairs == SAPO_PREF_BEST_WORST) {
        float hi = -INFINITY, lo = INFINITY;
        for (int32_t s = s0 + lane; s < s1; s += 32) {       // every warp for itself
          const float r = reward_of(s);
          if (r > hi) { hi = r; best = s; }
          if (r < lo) { lo = r; worst = s; }
        }
        #pragma unroll
        for (int d = 16; d > 0; d >>= 1) {                   // the lower index where rewards tie
          const float h2 = __shfl_xor_sync(0xffffffffu, hi, d), l2 = __shfl_xor_sync(0xffffffffu, lo, d);
          const int32_t b2 = __shfl_xor_sync(0xffffffffu, best, d), w2 = __shfl_xor_sync(0xffffffffu, worst, d);
          if (b2 >= 0 && (best < 0 || h2 > hi || (h2 == hi && b2 < best))) { hi = h2; best = b2; }
          if (w2 >= 0 && (worst < 0 || l2 < lo || (l2 == lo && w2 < worst))) { lo = l2; worst = w2; }
        }
      }
      // (a lane adds up its pairs in 64 bits; the few lanes' and warps' sums are joined in 32)
      double loss = 0.0, margin = 0.0;
      int32_t count = 0;
      for (int32_t i = s0 + warp; i < s1; i += PREF_WARPS) {
        const float r = reward_of(i), R = ratio_of(i);
        double f = 0.0;
        for (int32_t j = s0 + lane; j < s1; j += 32) {
          const float rj = reward_of(j);
          const bool wins = r > rj, loses = r < rj;
          if (!(wins || loses)) continue;
          if (a.pairs == SAPO_PREF_BEST_WORST && !(wins ? (i == best && j == worst) : (j == best && i == worst))) continue;
          const float Rj = ratio_of(j);
          const float h = a.beta * (wins ? R - Rj : Rj - R);
          if (!isfinite(h)) continue;                        // a sum that left the fp32 range
          float l, dl;
          pair_loss(a, h, l, dl);
          f += wins ? (double)dl : -(double)dl;
          if (wins) { loss += (double)l; margin += (double)h; ++count; }          // each pair once
        }
        const float factor = warp_sum((float)f);
        if (lane == 0) { if (kept) g_s[i - s0] = factor; else a.seq_grad[i] = factor; }   // scaled below, once the pairs are counted
      }
      const float loss_w = warp_sum((float)loss), margin_w = warp_sum((float)margin);
      count = __reduce_add_sync(0xffffffffu, count);
      if (lane == 0) { sums[0][warp] = loss_w; sums[1][warp] = margin_w; counts[warp] = count; }
      __syncthreads();
      if (warp == 0) {
        const float loss_q = warp_sum(lane < PREF_WARPS ? sums[0][lane] : 0.f), margin_q = warp_sum(lane < PREF_WARPS ? sums[1][lane] : 0.f);
        count = __reduce_add_sync(0xffffffffu, lane < PREF_WARPS ? counts[lane] : 0);
        const float per = count > 0 ? 1.f / (float)count : 0.f;
        if (lane == 0) {
          a.q_loss[q] = loss_q * per;
          if (a.q_margin != nullptr) a.q_margin[q] = margin_q * per;
          if (a.q_pairs != nullptr) a.q_pairs[q] = count;
          scale_s = a.grad_scale * a.beta * per / (float)a.Q;
        }
      }
      __syncthreads();
      for (int32_t i = s0 + threadIdx.x; i < s1; i += PREF_THREADS) {
        const float g = (kept ? g_s[i - s0] : a.seq_grad[i]) * scale_s;
        if (kept) g_s[i - s0] = g;
        a.seq_grad[i] = g;
      }
    }
    team_barrier();
    // 3.
    if (begin < end) {
      for (int32_t s = s_first; s < s1; ++s) {
        bool ignore = false;
        int32_t t0, t1;
        offset_range(cu, s, Tc, t0, t1, ignore);
        if (t0 >= end) break;
        const int32_t from = t0 > begin ? t0 : begin, to = t1 < end ? t1 : end;
        if (from >= to) continue;
        float g = !kept ? __ldcg(a.seq_grad + s) : (SOLO ? g_s[s - s0] : load_from_first(&g_s[s - s0]));
        if (a.length_norm) g /= (float)(t1 - t0);
        // the lane that summed a token writes its factor, and knows whether any of its tokens was masked
        for (int32_t t = from + lane; t < to; t += 32)
          if (SAPO_IN_BOUNDS(t >= 0 && t < a.T)) a.gscale[t] = masked && !isfinite(token_ratio(a, t)) ? 0.f : g;
      }
    }
  }
  if (bad_offset) raise_status(a.status, SAPO_ST_BAD_INDEX);
  if (bad_value && a.ref_logp != nullptr) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
  if (bad_reward) raise_status(a.status, SAPO_ST_NONFINITE_REWARD);
  // the first block's shared memory stays until the others have read the factors from it
  cluster_barrier();
  // The loss is the mean of the questions' losses, added up in their order by the block that comes last (SOLO: by the
  // first, behind the barrier).
  if (rank != 0 || warp != 0 || (SOLO && blockIdx.x != 0)) return;
  if (!SOLO) {
    if (a.ticket == nullptr) return;                       // preference_mean_kernel follows
    uint32_t before = 0;
    if (lane == 0) {
      __threadfence();                                     // this block's q_loss before its ticket
      before = atomicAdd(a.ticket, 1u);
    }
    if (__shfl_sync(0xffffffffu, before, 0) != (uint32_t)a.q_clusters - 1u) return;
    __threadfence();
    if (lane == 0) *a.ticket = 0u;
  }
  mean_loss(a.q_loss, a.Q, a.loss, lane);
}

// The last step of preference_kernel<false> in a launch of its own (one warp).
__global__ void __launch_bounds__(32) preference_mean_kernel(const float* q_loss, int32_t Q, float* loss) {
  let_next_start();
  wait_for_previous();
  mean_loss(q_loss, Q, loss, threadIdx.x);
}

// How many clusters of a launch have finished: one counter per launch, left at zero by it.  Launches take them in turn,
// so two that run at the same time (other streams, other threads) would share one only with 16384 launches in
// flight between them.  A graph would replay its launch with the same counter for good, beside later launches that
// get it in turn: a launch that is captured takes none, and preference_mean_kernel adds the losses up behind it.
constexpr int PREF_TICKETS = 16384;
static __device__ uint32_t g_pref_tickets[PREF_TICKETS];
static uint32_t* next_ticket(int dev) {
  static uint32_t* base[MAX_DEVICES] = {nullptr};
  static std::atomic<uint32_t> next{0};
  if (base[dev] == nullptr) {
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_pref_tickets) != cudaSuccess) return nullptr;
    base[dev] = static_cast<uint32_t*>(p);
  }
  return base[dev] + next.fetch_add(1u) % PREF_TICKETS;
}

int pref_check_cfg(const sapo_pref_cfg* c) {
  if (!c || !(c->beta > 0.f) || !isfinite(c->beta) || !isfinite(c->grad_scale)) return SAPO_ERR_INVALID_ARG;
  if (c->kind != SAPO_PREF_SIGMOID && c->kind != SAPO_PREF_SQUARED && c->kind != SAPO_PREF_HINGE) return SAPO_ERR_INVALID_ARG;
  if (c->pairs != SAPO_PREF_ALL && c->pairs != SAPO_PREF_BEST_WORST) return SAPO_ERR_INVALID_ARG;
  if (!(c->label_smoothing >= 0.f && c->label_smoothing < 0.5f)) return SAPO_ERR_INVALID_ARG;
  if (c->label_smoothing != 0.f && c->kind != SAPO_PREF_SIGMOID) return SAPO_ERR_INVALID_ARG;
  if (c->length_norm != 0 && c->length_norm != 1) return SAPO_ERR_INVALID_ARG;
  return SAPO_OK;
}

// Blocks per question: a power of two, enough for one to have about 4096 tokens of an average question
// (8 a thread), while all questions' blocks together still fit on the device at once.  The lengths are on the device,
// so the average is what the host has: a question that is far longer than the others is one cluster's work all the same
// (500 questions of 1000 tokens 19 us, with one of 500000 more 119 us).
static int pref_cluster(int64_t T, int32_t Q, int sms) {
  int c = 1;
  while (c < PREF_MAX_CLUSTER && (int64_t)Q * c * 4096 < T && (int64_t)Q * c * 2 <= 2 * (int64_t)sms) c <<= 1;
  return c;
}

int launch_preference(PrefArgs a, cudaStream_t st) {
  const int sms = sm_count();
  const int dev = current_device();
  if (sms <= 0 || dev < 0) return SAPO_ERR_CUDA;
  static bool wide[MAX_DEVICES] = {false};                   // clusters of 16 blocks allowed
  if (!wide[dev]) {
    if (cudaFuncSetAttribute(preference_kernel<false>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
        cudaFuncSetAttribute(preference_kernel<true>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
      return SAPO_ERR_CUDA;
    wide[dev] = true;
  }
  int cluster = pref_cluster(a.T, a.Q, sms);
  // Few questions of few tokens: one cluster has a block for each and one for what they do not cover, and its barrier
  // takes the place of the count of finished clusters.
  if (cluster == 1 && a.Q < PREF_MAX_CLUSTER && a.T <= 65536) {
    while (cluster <= a.Q) cluster <<= 1;
    a.q_clusters = a.Q;
    KernelScope scope(SAPO_K_PREFERENCE, st);
    return launch_overlapped(preference_kernel<true>, dim3((unsigned)cluster), PREF_THREADS, 0, cluster, st, a);
  }
  const int64_t most = (int64_t)sms * 4 / cluster;
  a.q_clusters = (int32_t)(a.Q < most ? a.Q : most);
  // clusters for what no question covers: a capacity behind the last token can be large
  int64_t outside = ceil_div<int64_t>(a.T, (int64_t)65536 * cluster);
  outside = outside < 1 ? 1 : (outside > 32 ? 32 : outside);
  cudaStreamCaptureStatus capture;
  if (cudaStreamIsCapturing(st, &capture) != cudaSuccess) return SAPO_ERR_CUDA;
  a.ticket = nullptr;
  if (capture == cudaStreamCaptureStatusNone && (a.ticket = next_ticket(dev)) == nullptr) return SAPO_ERR_CUDA;
  KernelScope scope(SAPO_K_PREFERENCE, st);
  const int rc = launch_overlapped(preference_kernel<false>, dim3((unsigned)((a.q_clusters + outside) * cluster)), PREF_THREADS, 0, cluster, st, a);
  if (rc != SAPO_OK || a.ticket != nullptr) return rc;
  ++kernel_timer().launches;
  return launch_overlapped(preference_mean_kernel, dim3(1), 32, 0, 0, st, (const float*)a.q_loss, a.Q, a.loss);
}

long long bounds_violations_preference() { return read_bounds_violations(); }
}  // namespace sapo

extern "C" int sapo_preference_loss(const float* logp, const float* ref_logp, int64_t T, const int32_t* cu_seqlens,
                                    int32_t S, const float* rewards, const int32_t* group_offsets, int32_t Q,
                                    const sapo_pref_cfg* h_cfg, float* gscale, float* seq_logratio, float* seq_grad,
                                    float* q_loss, float* q_margin, int32_t* q_pairs, float* loss,
                                    int32_t* status, void* stream) {
  using namespace sapo;
  int rc = pref_check_cfg(h_cfg);
  if (rc != SAPO_OK) return rc;
  if (T < 0 || S < 1 || Q < 1) return SAPO_ERR_INVALID_ARG;
  if (T > 0x7fffff00LL) return SAPO_ERR_UNSUPPORTED_SHAPE;
  if ((T > 0 && (!logp || !ref_logp || !gscale)) || !cu_seqlens || !rewards || !group_offsets || !seq_logratio ||
      !seq_grad || !q_loss || !loss || !status)
    return SAPO_ERR_INVALID_ARG;
  // an empty batch has no pointers to read through, but the kernel asks which kind of input it has
  PrefArgs a{logp, ref_logp, T, cu_seqlens, S, rewards, group_offsets, Q, h_cfg->beta, h_cfg->label_smoothing,
             h_cfg->grad_scale, h_cfg->kind, h_cfg->pairs, h_cfg->length_norm, gscale, seq_logratio, seq_grad,
             q_loss, q_margin, q_pairs, loss, status, 0, nullptr};
  return launch_preference(a, static_cast<cudaStream_t>(stream));
}
