// sapo_preference_loss: a preference loss over the completions of a question, from per-token
// log-probs to the gradient factor of every token.
//   R_s = sum over the tokens of s of (logp - ref_logp)   (divided by T_s with length_norm)
//   pairs (i, j) of one question, i preferred to j (reward_i > reward_j);  h = beta (R_i - R_j)
//   loss = 1/Q sum_q 1/n_q sum_pairs l(h)
// A question's completions are neighbours in the packed batch, so a question is one block's work:
// the sums of its sequences, its pairs, and one factor per sequence written to all its tokens.
// Reads 8 bytes and writes 4 per token.
#include <math.h>

#include "preference.cuh"

namespace sapo {

constexpr int PREF_THREADS = 256;

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

__device__ __forceinline__ double block_sum(double x, double* sh) {
  #pragma unroll
  for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < PREF_THREADS / 32; ++i) t += sh[i];
  return t;
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

__global__ void __launch_bounds__(PREF_THREADS) preference_kernel(PrefArgs a) {
  __shared__ double sh[PREF_THREADS / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t Tc = (int32_t)a.T;
  for (int32_t q = blockIdx.x; q < a.Q; q += gridDim.x) {
    bool bad_offset = false, bad_value = false, bad_reward = false;
    int32_t s0, s1;
    offset_range(a.group_offsets, q, a.S, s0, s1, bad_offset);
    // sums of the sequences
    for (int32_t s = s0 + warp; s < s1; s += PREF_THREADS / 32) {
      int32_t t0, t1;
      offset_range(a.cu, s, Tc, t0, t1, bad_offset);
      float sum = 0.f;
      for (int32_t t = t0 + lane; t < t1; t += 32) {
        const float d = a.ref_logp != nullptr ? a.logp[t] - a.ref_logp[t] : a.logp[t];
        if (isfinite(d)) sum += d; else bad_value = true;
      }
      #pragma unroll
      for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      if (lane == 0) a.seq_logratio[s] = a.length_norm && t1 > t0 ? sum / (float)(t1 - t0) : sum;
    }
    __syncthreads();
    // which completions take part: at least one token, a finite reward and a finite sum
    auto takes_part = [&](int32_t s) {
      bool ignore = false;
      int32_t t0, t1;
      offset_range(a.cu, s, Tc, t0, t1, ignore);
      return t1 > t0 && isfinite(a.rewards[s]) && isfinite(a.seq_logratio[s]);
    };
    int32_t best = -1, worst = -1;
    if (a.pairs == SAPO_PREF_BEST_WORST) {
      for (int32_t s = s0; s < s1; ++s) {
        if (!takes_part(s)) continue;
        if (best < 0 || a.rewards[s] > a.rewards[best]) best = s;
        if (worst < 0 || a.rewards[s] < a.rewards[worst]) worst = s;
      }
    }
    // thread per completion: its pairs as the preferred one count towards the loss, both sides
    // towards its factor
    double loss = 0.0, margin = 0.0, count = 0.0;
    for (int32_t i = s0 + threadIdx.x; i < s1; i += PREF_THREADS) {
      const float r = a.rewards[i], R = a.seq_logratio[i];
      if (!isfinite(r)) bad_reward = true;
      double f = 0.0;
      if (takes_part(i)) {
        for (int32_t j = s0; j < s1; ++j) {
          const float rj = a.rewards[j];
          if (rj == r || !takes_part(j)) continue;
          const bool wins = r > rj;
          if (a.pairs == SAPO_PREF_BEST_WORST && !(wins ? (i == best && j == worst) : (j == best && i == worst))) continue;
          const float h = a.beta * (wins ? R - a.seq_logratio[j] : a.seq_logratio[j] - R);
          float l, dl;
          pair_loss(a, h, l, dl);
          f += wins ? (double)dl : -(double)dl;
          if (wins) { loss += (double)l; margin += (double)h; count += 1.0; }
        }
      }
      a.seq_grad[i] = (float)f;                      // scaled below, once the pairs are counted
    }
    loss = block_sum(loss, sh);
    margin = block_sum(margin, sh);
    count = block_sum(count, sh);
    const double per = count > 0.0 ? 1.0 / count : 0.0;
    if (threadIdx.x == 0) {
      a.q_loss[q] = (float)(loss * per);
      if (a.q_margin != nullptr) a.q_margin[q] = (float)(margin * per);
      if (a.q_pairs != nullptr) a.q_pairs[q] = (int32_t)count;
    }
    const float scale = (float)((double)a.grad_scale * (double)a.beta * per / (double)a.Q);
    for (int32_t i = s0 + threadIdx.x; i < s1; i += PREF_THREADS) a.seq_grad[i] *= scale;
    __syncthreads();
    for (int32_t s = s0 + warp; s < s1; s += PREF_THREADS / 32) {
      bool ignore = false;
      int32_t t0, t1;
      offset_range(a.cu, s, Tc, t0, t1, ignore);
      const float g = a.length_norm && t1 > t0 ? a.seq_grad[s] / (float)(t1 - t0) : a.seq_grad[s];
      for (int32_t t = t0 + lane; t < t1; t += 32) {
        const float d = a.ref_logp != nullptr ? a.logp[t] - a.ref_logp[t] : a.logp[t];
        a.gscale[t] = isfinite(d) ? g : 0.f;
      }
    }
    if (bad_offset) raise_status(a.status, SAPO_ST_BAD_INDEX);
    if (bad_value && a.ref_logp != nullptr) raise_status(a.status, SAPO_ST_NONFINITE_INPUT);
    if (bad_reward) raise_status(a.status, SAPO_ST_NONFINITE_REWARD);
    __syncthreads();
  }
}

// What no question covers: sequences before the first and after the last one, and their tokens, get
// zeros.  One block also adds up the questions' losses.
__global__ void __launch_bounds__(PREF_THREADS) preference_final_kernel(PrefArgs a) {
  __shared__ double sh[PREF_THREADS / 32];
  bool ignore = false;
  const int32_t Tc = (int32_t)a.T;
  const int32_t s_lo = clamp_to(a.group_offsets[0], a.S, ignore);
  int32_t s_hi = clamp_to(a.group_offsets[a.Q], a.S, ignore);
  if (s_hi < s_lo) s_hi = s_lo;
  const int32_t t_lo = clamp_to(a.cu[s_lo], Tc, ignore);
  int32_t t_hi = clamp_to(a.cu[s_hi], Tc, ignore);
  if (t_hi < t_lo) t_hi = t_lo;
  const int64_t first = (int64_t)blockIdx.x * PREF_THREADS + threadIdx.x, step = (int64_t)gridDim.x * PREF_THREADS;
  for (int64_t i = first; i < (int64_t)t_lo + (Tc - t_hi); i += step) a.gscale[i < t_lo ? i : t_hi + (i - t_lo)] = 0.f;
  for (int64_t i = first; i < (int64_t)s_lo + (a.S - s_hi); i += step) {
    const int64_t s = i < s_lo ? i : s_hi + (i - s_lo);
    a.seq_logratio[s] = 0.f;
    a.seq_grad[s] = 0.f;
  }
  if (blockIdx.x != 0) return;
  double x = 0.0;
  for (int32_t q = threadIdx.x; q < a.Q; q += PREF_THREADS) x += (double)a.q_loss[q];
  x = block_sum(x, sh);
  if (threadIdx.x == 0) *a.loss = (float)(x / (double)a.Q);
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

int launch_preference(const PrefArgs& a, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return SAPO_ERR_CUDA;
  {
    const int64_t most = (int64_t)sms * 8;
    KernelScope scope(SAPO_K_PREFERENCE, st);
    preference_kernel<<<(int)(a.Q < most ? a.Q : most), PREF_THREADS, 0, st>>>(a);
  }
  int64_t blocks = ceil_div<int64_t>(a.T, 4096);
  if (blocks < 1) blocks = 1;
  if (blocks > sms) blocks = sms;
  KernelScope scope(SAPO_K_PREF_FINAL, st);
  preference_final_kernel<<<(int)blocks, PREF_THREADS, 0, st>>>(a);
  return check_launch();
}

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
             q_loss, q_margin, q_pairs, loss, status};
  return launch_preference(a, static_cast<cudaStream_t>(stream));
}
