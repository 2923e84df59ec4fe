// Token log probabilities, row entropy and the rows' top alternatives
// (host-side launch interface).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace spec {

constexpr int kLogprobMaxTop = 64;

struct LogprobPlan {
  int rows = 0, V = 0, n_top = 0;
  int chunk = 0, n_chunks = 0;  // n_chunks <= 64
};
LogprobPlan logprob_plan(int rows, int V, int n_top);
size_t logprob_ws_bytes(const LogprobPlan& p);

// logits [rows] rows of V fp32, ld floats apart; temps (null: 1) and tokens
// (null: none asked) one per row; outputs logp, entropy [rows] (null: not
// wanted), top_ids, top_logp [rows, n_top].  All device pointers.
hipError_t launch_logprobs(const LogprobPlan& p, const float* logits, int64_t ld, const float* temps,
                           const int32_t* tokens, float* logp, float* entropy, int32_t* top_ids, float* top_logp,
                           void* ws, hipStream_t st);

}  // namespace spec
