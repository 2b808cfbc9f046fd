// What the preference loss on per-token log-probs shares with the call that goes through the LM head.
#pragma once

#include "common.cuh"

namespace sapo {

struct PrefArgs {
  // per-token log-probs of the policy and of the reference, or (ref_logp NULL) their difference, a
  // NaN where a token is masked
  const float* logp; const float* ref_logp; int64_t T;
  const int32_t* cu; int32_t S; const float* rewards; const int32_t* group_offsets; int32_t Q;
  float beta, smoothing, grad_scale; int32_t kind, pairs, length_norm;
  float* gscale; float* seq_logratio; float* seq_grad; float* q_loss; float* q_margin; int32_t* q_pairs; float* loss;
  int32_t* status;
  // set by launch_preference: clusters of blocks that take questions, and the counter of those that have finished
  // (NULL: none, the loss is added up by a launch behind)
  int32_t q_clusters; uint32_t* ticket;
};

int pref_check_cfg(const sapo_pref_cfg* h_cfg);
int launch_preference(PrefArgs a, cudaStream_t st);

}  // namespace sapo
