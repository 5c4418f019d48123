// ops.hpp -- operators for policies computed by the caller's own network: the launchers of the
// gated recurrence (scan_kernels.hip), of linear attention (linattn_kernels.hip), of the losses over logits
// (logit_kernels.hip), of log-probabilities (logprob_kernels.hip) and of orthogonalised updates
// (ortho_kernels.hip), and what the entry points (ops.cpp) see of a context.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "batchsim.h"

namespace bsim {

// latched beside the simulator's flags (params.hpp)
enum : uint32_t { ERR_LENGTH = 8u, ERR_DECAY = 16u };

// What an operator needs of a context (runtime.cpp).
struct OpCtx {
  hipStream_t stream;
  int device;
  uint32_t* err;
};
OpCtx op_ctx(sim_ctx* x);
// sets the calling thread's message and returns code
int op_fail(int code, const char* fmt, ...);
// runs launch(arg), bracketed by events of class cls if the context is tracing
hipError_t op_timed(sim_ctx* x, int cls, hipError_t (*launch)(void*), void* arg);

struct ScanArgs {
  sim_scan c;
  sim_seq g, x, y, dy, dg, dx;   // unused ones have a null pointer
  const int32_t* len;
  const void* h0;      // state before the first step (null: 0)
  const void* ds;      // grad: gradient of the last state (null: 0)
  void* state;         // forward: last state; grad: gradient of h0 (may be null)
  uint32_t* err;
  void* work;
};
size_t scan_work_bytes(const sim_scan& c, bool grad);
hipError_t launch_scan(const ScanArgs& a, bool grad, hipStream_t st);

struct PolicyLossArgs {
  sim_policy_loss c;
  sim_mat l, mask, grad;
  const void *act, *adv;
  const float *w, *logp_old, *logp_ref;
  float *logp, *loss;
  uint32_t* err;
  void* work;
};
size_t policy_loss_bytes(const sim_policy_loss& c);
hipError_t launch_policy_loss(const PolicyLossArgs& a, hipStream_t st);

struct BalanceArgs {
  sim_balance c;
  sim_mat l, grad;
  const void* idx;
  const uint8_t* live;
  int64_t* counts;
  float* loss;
  uint32_t* err;
  void* work;
};
size_t balance_bytes(const sim_balance& c);
hipError_t launch_balance(const BalanceArgs& a, hipStream_t st);

struct AttnArgs {
  sim_linear_attn c;
  sim_heads q, k, v, dy, y, dq, dk, dv;   // unused ones have a null pointer
  const float *decay, *s0, *ds;           // grad: ds the gradient of the last state (null: 0)
  const int32_t* len;
  float* state;                           // forward: last state; grad: gradient of s0 (may be null)
  uint32_t* err;
  void* work;
};
size_t attn_work_bytes(const sim_linear_attn& c, bool grad);
hipError_t launch_attn(const AttnArgs& a, bool grad, hipStream_t st);

struct LogprobArgs {
  sim_logprobs c;
  sim_mat l, mask, grad;
  const void* tokens;
  const uint8_t* live;
  const float *dlogp, *dentropy;
  float *logp, *entropy, *top_logp;
  int64_t* top_index;
  uint32_t* err;
  void* work;
};
size_t logprob_bytes(const sim_logprobs& c, bool grad);
hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t st);

struct OrthoArgs {
  sim_ortho c;
  sim_mats u, out;
  void* work;
};
size_t ortho_bytes(const sim_ortho& c);
hipError_t launch_ortho(const OrthoArgs& a, hipStream_t st);

}  // namespace bsim
