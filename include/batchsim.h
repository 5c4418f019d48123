/* batchsim.h -- C ABI of the MI355X (gfx950) batched serving-simulator rollout library.
 *
 * Paper: "Adaptive Inference Batching using Policy Gradients". The library steps many
 * independent environments in lockstep. Each environment is the paper's discrete-event
 * inference-serving simulator (Sec. 3.1): requests arrive (Sec. 3.2 workloads), wait in
 * per-class FIFO queues capped at N with load shedding, and are dispatched in batches to
 * K simulated servers whose batch latency is alpha + beta*b. The agent's MDP (Sec. 4.1)
 * observes a state vector, chooses a (server, batch size) action and receives a reward of
 * throughput minus weighted latency. The policy is an MLP (Sec. 4.2) and the rollout feeds
 * discounted returns / GAE (Sec. 4.3).
 *
 * Conventions
 *   - Every call returns an int status: SIM_OK (0) or a negative SIM_E* code. The message
 *     of the last failure on the calling thread is returned by sim_last_error(); the
 *     string is owned by the library. No call aborts or throws across the ABI.
 *   - "d_" pointers are device pointers (HBM of the context's device), allocated and
 *     owned by the caller; "h_" pointers are host pointers. The library owns the context
 *     and the per-environment state it allocates in sim_create and frees in sim_destroy.
 *   - All device work is enqueued on the stream given to sim_create and is asynchronous;
 *     errors detected on the device (an action out of range, an event loop exceeding its
 *     bound) are latched in a device flag and reported by sim_sync().
 *   - Layouts are time-major, environment-minor: element (t, e) of a [T][E] array is at
 *     t*E + e; feature f of environment e in an [F][E] observation is at f*E + e.
 *   - Times are fp64 seconds; rates are requests per second.
 *   - Randomness is a counter-based Philox4x32-10 stream keyed by the seed, with counter
 *     (env, step, purpose<<24 | j, system); the same seed gives the same rollout.
 */
#ifndef BATCHSIM_H
#define BATCHSIM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define BATCHSIM_ABI_VERSION 2u

enum sim_status {
  SIM_OK = 0,
  SIM_EINVAL = -1,       /* invalid argument or configuration */
  SIM_ENOMEM = -2,       /* device allocation failed */
  SIM_EDEVICE = -3,      /* a HIP runtime call failed */
  SIM_ESTATE = -4,       /* call out of order, or a latched device-side error */
  SIM_EUNSUPPORTED = -5  /* configuration outside the compiled shapes */
};

enum { SIM_ARR_MODULATED = 0, SIM_ARR_TRACE = 1 };
enum { SIM_DWELL_INF = 0, SIM_DWELL_EXP = 1, SIM_DWELL_PARETO = 2, SIM_DWELL_DET = 3 };
enum { SIM_ROUTE_LOWEST = 0, SIM_ROUTE_RANDOM = 1, SIM_ROUTE_ROUND_ROBIN = 2,
       SIM_ROUTE_SHORTEST = 3 };
/* policy network (Sec. 4.2) */
enum { SIM_POLICY_MLP = 0, SIM_POLICY_ATTN = 1 };
enum { SIM_SVC_DET = 0, SIM_SVC_LOGN = 1, SIM_SVC_EXP = 2 };

#define SIM_MAX_SERVERS 16
#define SIM_MAX_CLASSES 4
#define SIM_MAX_STATES 4
#define SIM_MAX_QUEUE 255

/* Simulator and policy configuration (plain data, copied by sim_create).
 *  n_envs          environments stepped in lockstep (E >= 1)
 *  n_servers       K simulated servers per environment (1..16); actions are 6K (Sec. 4.1)
 *  n_classes       request classes / model types (1..4) (Sec. 3.1 request model)
 *  queue_cap       N, waiting requests per environment over all classes (Sec. 3.1, N=100)
 *  obs_dim         F, observation width, at least the state layout's width
 *  tick_s          decision interval (the agent acts once per tick)
 *  arrival_kind    SIM_ARR_MODULATED (Poisson / MMPP / ON-OFF) or SIM_ARR_TRACE
 *  n_states        states of the modulating process (1 = plain Poisson)
 *  rate[i]         arrival rate in state i (0 = no arrivals)
 *  dwell_kind[i]   law of the time spent in state i: INF, EXP(mean dwell_mean[i]),
 *                  PARETO(pareto_alpha[i], pareto_xm[i]) or DET (exactly dwell_mean[i]; a
 *                  process whose state 0 is DET starts in state 0 at t = 0, the square
 *                  wave of the Extreme Burst workload, Sec. 3.2)
 *  class_mix[c]    probability that an arrival is of class c
 *  service_kind[c] DET: alpha + beta*n; LOGN: median*exp(sigma*Z) + beta*n;
 *                  EXP: Exp with mean alpha + beta*n (Sec. 3.1 execution model)
 *  w_thr, w_class  reward weights: w_thr * throughput - latency weighted by class
 *                  (Sec. 4.1); reward_sum = 1 sums the weighted latencies, 0 averages them
 *  obs_tw          time normaliser of ages in the observation (T_window of Sec. 4.1)
 *  lambda_ref      rate normaliser of the arrival-rate features
 *  shadow          1 runs a second system per environment on the same arrivals under the
 *                  static rule "dispatch when static_bmax requests wait or the oldest has
 *                  waited static_timeout" (Sec. 1), with its own reward and counters
 *  mlp_h1, mlp_h2  hidden widths of the policy MLP; mlp_bf16 = 1 for bf16 weights and
 *                  activations with fp32 accumulation, 0 for fp32 throughout
 *  value_head      1 adds a value output column (Sec. 4.2 value head)
 *  trace_max_len   per-environment capacity of the arrays given to sim_set_trace
 *  static_route    server that takes a batch of the static rule: SIM_ROUTE_LOWEST idle
 *                  index, SIM_ROUTE_RANDOM (uniform over the idle servers) or
 *                  SIM_ROUTE_ROUND_ROBIN (first idle server from a per-environment
 *                  pointer); the Random and Round-Robin baselines of Sec. 5.1. Or
 *                  SIM_ROUTE_SHORTEST, the Shortest-Queue baseline of Sec. 5.1: every
 *                  server holds the batch it runs and at most one queued behind it; the
 *                  rule forms a batch whenever its condition holds, whether or not a
 *                  server is idle, and sends it to the server with the fewest requests
 *                  assigned and not completed among those with room (lower index on
 *                  ties), where it starts when that server is free; with no room it waits.
 *                  At most 8 servers (SIM_EUNSUPPORTED otherwise)
 *  policy_kind     SIM_POLICY_MLP (the MLP above) or SIM_POLICY_ATTN, the attention
 *                  policy of Sec. 4.2: the obs_dim features split into attn_tokens
 *                  contiguous groups, each group's terms of the input projection summed
 *                  into one token of width attn_embed; multi-head self-attention with
 *                  attn_heads heads; the mean of the tokens feeds a policy head with
 *                  mlp_h1 GELU units and, with value_head = 1, a separate value head with
 *                  mlp_h2 GELU units. fp32 only (mlp_bf16 = 0). Built shapes:
 *                  attn_embed = 4, attn_heads in {1, 2, 4}, attn_tokens in {1, 2, 4, 8}
 *                  dividing obs_dim <= 64, n_servers in {1, 2, 4}, mlp_h1, mlp_h2 <= 256 */
typedef struct sim_cfg {
  uint32_t abi_version; /* BATCHSIM_ABI_VERSION */
  uint32_t struct_size; /* sizeof(sim_cfg) */
  int32_t n_envs, n_servers, n_classes, queue_cap, obs_dim;
  double tick_s;
  int32_t arrival_kind, n_states;
  double rate[SIM_MAX_STATES];
  int32_t dwell_kind[SIM_MAX_STATES];
  double dwell_mean[SIM_MAX_STATES], pareto_alpha[SIM_MAX_STATES], pareto_xm[SIM_MAX_STATES];
  double class_mix[SIM_MAX_CLASSES];
  int32_t service_kind[SIM_MAX_CLASSES];
  double svc_alpha[SIM_MAX_CLASSES], svc_beta[SIM_MAX_CLASSES], svc_median[SIM_MAX_CLASSES];
  double svc_sigma;
  double w_thr, w_class[SIM_MAX_CLASSES];
  int32_t reward_sum;
  double obs_tw, lambda_ref;
  int32_t shadow;
  double static_timeout;
  int32_t static_bmax;
  int32_t mlp_h1, mlp_h2, mlp_bf16, value_head;
  int32_t trace_max_len;
  int32_t static_route;
  int32_t policy_kind, attn_tokens, attn_embed, attn_heads;
} sim_cfg;

/* Byte offsets of the policy weights inside one caller-owned device buffer. Weights are
 * [in][out] row-major; W1 is [F][H1], W2 [H1][H2], W3 [H2][A'] with A' = 6K + value_head.
 * Matrices are fp32, or bf16 (raw 16-bit patterns) when mlp_bf16 = 1; biases are fp32.  */
typedef struct sim_wlayout {
  size_t w1, b1, w2, b2, w3, b3; /* offsets in bytes, 256-byte aligned (MLP policy only;
                                    zero for the attention policy) */
  size_t bytes;                  /* total size of the buffer (either policy) */
  int32_t n_out;                 /* A' */
  int32_t elem_bytes;            /* 4 (fp32) or 2 (bf16) */
} sim_wlayout;

/* Byte offsets of the attention policy's weights (policy_kind = SIM_POLICY_ATTN) in one
 * caller-owned device buffer of sim_wlayout.bytes bytes, all fp32, [in][out] row-major
 * (D = attn_embed, A = 6K): w_in [F][D] and b_in [D] (input projection), w_qkv [D][3D]
 * (columns: query, key, value) and b_qkv [3D], w_o [D][D] and b_o [D] (attention output),
 * wp1 [D][mlp_h1], bp1, wp2 [mlp_h1][A], bp2 (policy head), wv1 [D][mlp_h2], bv1,
 * wv2 [mlp_h2][1], bv2 [1] (value head). Offsets are 256-byte aligned.                  */
typedef struct sim_attn_layout {
  size_t w_in, b_in, w_qkv, b_qkv, w_o, b_o;
  size_t wp1, bp1, wp2, bp2, wv1, bv1, wv2, bv2;
  size_t bytes;
} sim_attn_layout;

/* Caller-owned device buffers filled by sim_rollout. Only `actions` is required; any
 * other pointer may be NULL to skip that output.                                       */
typedef struct sim_traj {
  uint8_t* actions;       /* [T][E] sampled actions */
  float* logp;            /* [T][E] log-probability of the sampled action */
  double* reward;         /* [T][E] learned system's reward r_k */
  double* reward_shadow;  /* [T][E] static shadow system's reward (cfg.shadow = 1) */
  float* value;           /* [T+1][E] value head (cfg.value_head = 1); row T is V(obs_T) */
  float* obs;             /* [T+1][F][E] observations obs_k, k = 0..T */
  uint64_t* rchk;         /* [T][E] learned system's running checksum after each tick */
} sim_traj;

/* Per-environment integer counters and sums, system s in {0 learned, 1 shadow}. */
#define SIM_NCNT 7 /* arrivals, accepted, dropped, dispatched, batches, completed, inflight */
#define SIM_NSUM 2 /* latency sum, weighted latency sum (seconds) */

typedef struct sim_totals {
  int64_t cnt[2][SIM_NCNT]; /* summed over environments */
  double sum[2][SIM_NSUM];
} sim_totals;

typedef struct sim_ctx sim_ctx;

/* Message of the last failed call on this thread (library-owned, never NULL). */
const char* sim_last_error(void);

/* Library ABI version (BATCHSIM_ABI_VERSION). */
uint32_t sim_abi_version(void);

/* Creates a context on the current HIP device: n_envs copies of the simulator of Sec. 3.1
 * (and of the MDP of Sec. 4.1 around it). Validates cfg (SIM_EINVAL with a message naming the
 * field), allocates the structure-of-arrays environment state and queues in HBM (SIM_ENOMEM). `hip_stream` is a hipStream_t (NULL = default stream). The context is
 * not usable until sim_reset. On failure *out is NULL and nothing stays allocated.     */
int sim_create(const sim_cfg* cfg, void* hip_stream, sim_ctx** out);

/* Waits for the context's stream and frees everything it owns. NULL is allowed.        */
int sim_destroy(sim_ctx* ctx);

/* Explicit arrivals for SIM_ARR_TRACE (Sec. 3.2 trace replay): device arrays times
 * [E][trace_max_len] (nondecreasing seconds), classes [E][trace_max_len], counts [E].
 * The arrays must stay valid until the context is destroyed or given new ones.        */
int sim_set_trace(sim_ctx* ctx, const double* d_times, const uint8_t* d_classes,
                  const int32_t* d_counts);

/* Resets every environment at t = 0 (empty queues, idle servers, zero counters, the
 * modulating state of the Sec. 3.2 arrival process drawn from its stationary law) and sets the
 * tick counter to 0: the start of an episode (Sec. 4.3).                                */
int sim_reset(sim_ctx* ctx, uint64_t seed);

/* Copies the current observation [F][E] fp32 (the state of Sec. 4.1) to d_obs.         */
int sim_obs(sim_ctx* ctx, float* d_obs);

/* One step of the MDP (Sec. 4.1): advances every environment by one tick of the simulator
 * (Sec. 3.1) under the given actions (d_actions [E], values in [0, 6K): server a/6, batch size
 * 2^(a%6)). Optional outputs: the next observation
 * [F][E], the learned and shadow rewards [E]. An action out of range latches SIM_ESTATE.*/
int sim_step(sim_ctx* ctx, const uint8_t* d_actions, float* d_obs_next, double* d_reward,
             double* d_reward_shadow);

/* Current tick index (number of ticks since the last reset). */
int sim_tick(sim_ctx* ctx, int32_t* h_tick);

/* Layout of the weights buffer for this configuration (no device work).                */
int sim_weights_layout(const sim_cfg* cfg, sim_wlayout* out);

/* Offsets of the attention policy's weights (Sec. 4.2); SIM_EINVAL unless
 * cfg->policy_kind = SIM_POLICY_ATTN with a valid attention shape.                      */
int sim_attn_weights_layout(const sim_cfg* cfg, sim_attn_layout* out);

/* Initialises the policy network of Sec. 4.2: writes Xavier-uniform weights drawn from
 * `seed` and zero biases into d_weights
 * (layout of sim_weights_layout, or of sim_attn_weights_layout for the attention policy,
 * whose seven matrices take weight-stream layers 0..6 in layout order).                 */
int sim_init_weights(sim_ctx* ctx, uint64_t seed, void* d_weights);

/* Policy on one batch of observations d_obs [F][E]: MLP (or attention) forward, then an
 * action sampled from the softmax of the logits with the ACTION uniform of (env, step).
 * Outputs (any may be NULL): d_act [E], d_logp [E], d_value [E] (value head),
 * d_logits [A'][E] fp32.                                                                */
int sim_policy(sim_ctx* ctx, const void* d_weights, const float* d_obs, uint32_t step,
               uint8_t* d_act, float* d_logp, float* d_value, float* d_logits);

/* Diagnostics for the parity tests of the policy MLP (Sec. 4.2): sim_policy, run by the same
 * kernel source instantiated with extra stores, which also writes every hidden activation as
 * the kernel hands it to the next layer: d_hidden [H1 + H2][E] fp32 (rows 0..H1-1 the first
 * hidden layer, then the second; in bf16 configurations the bf16 values, widened). Its other
 * outputs equal sim_policy's bit for bit. SIM_EUNSUPPORTED for the attention policy.       */
int sim_policy_hidden(sim_ctx* ctx, const void* d_weights, const float* d_obs, uint32_t step,
                      uint8_t* d_act, float* d_logp, float* d_value, float* d_logits,
                      float* d_hidden);

/* A rollout of the MDP (Sec. 4.1) under the policy of Sec. 4.2, the trajectory that the
 * updates of Sec. 4.3 consume: T ticks of policy + simulator from the current state
 * (obs_k -> a_k -> obs_{k+1}), writing the trajectory; with a value head, row T of
 * traj->value holds V(obs_T). Ordered on the context's stream like every other call: the
 * static shadow system's launches run on a second stream of the context, forked from the
 * context's stream when the rollout starts and joined back before it ends (one stream when
 * sim_set_timing is on). Small batches run all T ticks in one fused launch
 * (sim_set_fused_rollout), with the same outputs. Afterwards sim_obs returns obs_T.      */
int sim_rollout(sim_ctx* ctx, const void* d_weights, int32_t T, const sim_traj* traj);

/* Rollout graphs, on by default: when sim_rollout is called again with the same weights
 * buffer, T, trajectory pointers and starting tick as the call before (a training loop that
 * resets and rolls out into the same buffers), its launch sequence is captured into a HIP
 * graph on a private stream of the context, and that graph is replayed by every further
 * repeat (ordered after earlier work on the context's stream, and before later work, by
 * events). Kernels read the seed from device memory written by sim_reset, so a new seed needs
 * no new graph. Tracing (sim_set_timing) launches eagerly. Per-tick rollouts of large
 * batches (from 8192 environments, 2048 with four servers or more, unless fused) run as two chains
 * of launches side by side, one per half of the batch, from 16 ticks (fewer with many environments
 * and servers), which one replayed graph's branches would not: with up to three servers and 40960
 * environments a repeat of 128 ticks or more replays a graph per half and 256 ticks, other rollouts
 * of such batches are launched (the host then takes about 14 us per tick in two chains). sim_set_trace discards the
 * graphs.
 * on = 0 launches every rollout eagerly.                                                    */
int sim_set_graphs(sim_ctx* ctx, int32_t on);

/* Fused rollouts of small batches (Sec. 4.1-4.2: the same ticks and policy as above): with a
 * few thousand environments a tick's two launches are bound by their start-up and memory
 * latency rather than their work, so sim_rollout may instead run all T ticks in one launch,
 * each workgroup alternating the policy and the tick of its own environments (outputs
 * bit-identical to the per-tick launches). mode SIM_FUSE_AUTO (the default) fuses when the
 * policy is an MLP of a shape that has a fused kernel (the 8-64-64-6 fp32, 12-128-128-6,
 * 32-256-256-24 and 64-256-256-48 bf16 networks, any action count up to the padded width)
 * and all of the batch's workgroups of that kernel are resident on the GPU at once, or, with
 * one or two request classes, at most twice as many (one and a half times from four servers
 * on or beside a shadow system) for rollouts of four ticks or more;
 * SIM_FUSE_ON fuses whenever the shape has a fused kernel; SIM_FUSE_OFF always launches per
 * tick. SIM_EINVAL for another mode. A change discards the rollout graph.                  */
enum { SIM_FUSE_OFF = 0, SIM_FUSE_AUTO = 1, SIM_FUSE_ON = 2 };
int sim_set_fused_rollout(sim_ctx* ctx, int32_t mode);

/* Diagnostics of the rollout graphs: graphs of a whole rollout captured, and rollouts replayed
 * from one, so far (either pointer may be NULL).                                         */
int sim_graph_stats(sim_ctx* ctx, int64_t* h_captures, int64_t* h_replays);

/* Discounted returns and GAE (Sec. 4.3), per environment backwards in t:
 *   delta_t = (r_t + gamma V_{t+1}) - V_t,  A_t = delta_t + (gamma*lambda) A_{t+1},
 *   A_T = 0,  R_t = A_t + V_t.
 * d_r [T][E] fp64; d_v [T+1][E] fp32 or NULL for V = 0 (with lambda = 1 this is the
 * REINFORCE return). Writes d_adv and d_ret [T][E] fp64.                                */
int returns_gae(sim_ctx* ctx, int32_t T, const double* d_r, const float* d_v, double gamma,
                double lambda, double* d_adv, double* d_ret);

/* One PPO minibatch (Sec. 4.3, clipped surrogate): M samples (t, env) drawn with
 * replacement, sample m taking u from the MINIBATCH block at counter
 * (m, 0xFFFFFFFD, MINIBATCH<<24, 0) under `seed` and index i = floor(u T E), t = i / E,
 * env = i % E. Forward through the policy (layer inputs rounded as in sim_policy, exact
 * GELU) and the loss
 *   L = -mean(min(rho A, clip(rho, 1-clip, 1+clip) A)) + c_value mean((V - R)^2)
 *       - c_entropy mean(H),   rho = exp(logp(a) - logp_old),
 * then dL/dW for every weight, the roundings passed through as the identity.
 * Inputs (device, read only): d_weights (layout of sim_weights_layout), d_obs [T][F][E]
 * fp32 (rows 0..T-1 of a rollout's observations), d_actions [T][E] u8, d_logp_old [T][E]
 * fp32, d_adv and d_ret [T][E] fp64. Outputs (device, caller-owned): d_grads fp32,
 * W1 [F][H1], b1 [H1], W2 [H1][H2], b2 [H2], W3 [H2][A'], b3 [A'] packed back to back
 * (A' = 6K + 1; sim_ppo_grad_count gives the total); d_loss [4] fp64 = total, policy,
 * value and entropy terms; d_index [M] int64 (t E + env) or NULL. Requires value_head = 1,
 * M > 0 and a multiple of 16, hidden widths that are multiples of 64, obs_dim <= 128 and
 * A' <= 128 (SIM_EUNSUPPORTED otherwise). The dense products run on the matrix cores: bf16 x bf16 -> fp32
 * for a bf16 policy (the fp32 gradient operand carried as two bf16 terms, 2^-17 relative),
 * fp32 x fp32 otherwise; the reductions over the samples are summed in a fixed order, so
 * repeated calls return identical results. Scratch of at most Mp (e (2 F + 4 H1 + 6 H2 + 4 A')
 * + 4 (H1 + H2 + A')) bytes (Mp = M rounded up to 64, e = 2 bytes for bf16 or 4 for fp32,
 * F and A' rounded up to 64; about half of that for the rollout policies' networks) plus about
 * 8 MiB of split-k partial sums is held by the context after the first call (grown if a later
 * call needs more). A stored action out of range latches SIM_ESTATE (reported by sim_sync);
 * that sample then contributes nothing.
 * For the attention policy (policy_kind = SIM_POLICY_ATTN) the forward is fp32 (GELU no further
 * from its exact value than with erff; sums in another order than sim_policy's, so that the
 * log-probabilities of the two differ by their rounding) and d_grads holds the fourteen arrays of sim_attn_layout in its order (w_in, b_in,
 * w_qkv, b_qkv, w_o, b_o, wp1, bp1, wp2, bp2, wv1, bv1, wv2, bv2), each [in][out] as in the
 * weights; the gradient terms of 32 samples at a time are summed over the minibatch in a fixed
 * order, in a scratch of 4 P + 24 bytes per 32 samples (P = sim_ppo_grad_count; the limit of
 * ppo_minibatch_grad_noalloc is stated by 4 M P + 24 M bytes).                            */
int ppo_minibatch_grad(sim_ctx* ctx, const void* d_weights, int32_t T, const float* d_obs,
                       const uint8_t* d_actions, const float* d_logp_old, const double* d_adv,
                       const double* d_ret, int32_t M, uint64_t seed, float clip, float c_value,
                       float c_entropy, float* d_grads, double* d_loss, int64_t* d_index);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight
 * training loops, harnesses that forbid hipMalloc): ppo_minibatch_grad with the same arguments,
 * inputs, outputs, error behaviour and results, bit for bit, but run on a fixed scratch the
 * library holds in device memory (96 MiB per GPU, allocated when the library's code is loaded
 * on that GPU and kept until the process ends) instead of the context's on-demand buffer. It
 * calls no hipMalloc, hipFree or other allocating routine and records no tracing events.
 * SIM_EINVAL, with the sizes in the message, when the bytes stated for ppo_minibatch_grad (the
 * formula in full, also for networks that need half of it) exceed that (C4's shape at M = 8192:
 * about 76 MiB), whatever the kernels use of them. Every call on a GPU uses the same scratch: calls
 * whose work overlaps on one GPU (several streams or threads) race and must be serialised by
 * the caller; calls in order on one stream are safe. The scratch keeps the previous call's
 * contents; every byte a call reads is written by that call first.                        */
int ppo_minibatch_grad_noalloc(sim_ctx* ctx, const void* d_weights, int32_t T,
                               const float* d_obs, const uint8_t* d_actions,
                               const float* d_logp_old, const double* d_adv, const double* d_ret,
                               int32_t M, uint64_t seed, float clip, float c_value,
                               float c_entropy, float* d_grads, double* d_loss, int64_t* d_index);

/* Number of fp32 gradient values written by ppo_minibatch_grad (no device work), for either
 * policy network.                                                                       */
int sim_ppo_grad_count(const sim_cfg* cfg, int64_t* h_count);

/* REINFORCE with a learned baseline (Sec. 4.3) on one minibatch: as ppo_minibatch_grad, with
 * the policy term -mean(A log pi(a|s)) (A held constant) and no old log-probabilities; the
 * caller passes A = G - V and R = G (returns_gae with lambda = 1 gives both).            */
int reinforce_minibatch_grad(sim_ctx* ctx, const void* d_weights, int32_t T, const float* d_obs,
                             const uint8_t* d_actions, const double* d_adv, const double* d_ret,
                             int32_t M, uint64_t seed, float c_value, float c_entropy,
                             float* d_grads, double* d_loss, int64_t* d_index);

/* Master parameters from a weights buffer: d_params (device, sim_ppo_grad_count fp32 values
 * in the gradient layout) receives the values d_weights holds.                          */
int sim_params_from_weights(sim_ctx* ctx, const void* d_weights, float* d_params);

/* One Adam step (Kingma & Ba 2015, Algorithm 1) on the fp32 master parameters, in place:
 *   m = b1 m + (1-b1) g,  v = b2 v + (1-b2) g^2,  p -= lr (m/(1-b1^t)) / (sqrt(v/(1-b2^t)) + eps)
 * with t = step >= 1 (the step being taken); d_m, d_v are the caller's moment buffers (zero
 * before the first step). With d_weights non-NULL the policy's weights are then rewritten from
 * the parameters (matrices rounded to bf16, nearest even, in bf16 configurations; copied as
 * they are for the fp32 attention policy).                                              */
int adam_update(sim_ctx* ctx, float* d_params, const float* d_grads, float* d_m, float* d_v,
                int32_t step, float lr, float beta1, float beta2, float eps, void* d_weights);

enum sim_algo { SIM_ALGO_PPO = 0, SIM_ALGO_REINFORCE = 1 };

typedef struct sim_update_cfg {
  int32_t algo;         /* SIM_ALGO_PPO or SIM_ALGO_REINFORCE */
  int32_t epochs;       /* passes over the trajectory */
  int32_t minibatches;  /* minibatches per epoch */
  int32_t M;            /* samples per minibatch (multiple of 16) */
  uint64_t seed;        /* minibatch b of epoch e: key seed + (e*minibatches + b)*0x9E3779B97F4A7C15 */
  float clip;           /* PPO clip range epsilon */
  float c_value, c_entropy;
  float lr, beta1, beta2, eps;
} sim_update_cfg;

/* The policy update of Sec. 4.3 over one stored trajectory (d_obs [T][F][E], d_actions,
 * d_logp_old (PPO only) [T][E], d_adv, d_ret [T][E] fp64): for each epoch and minibatch,
 * the minibatch gradient and one Adam step, after which d_weights holds the new policy.
 * *h_step is Adam's step count, advanced once per minibatch. d_losses (optional, device)
 * receives [epochs*minibatches][4] fp64 loss terms, each from the weights before its step. */
int sim_update(sim_ctx* ctx, const sim_update_cfg* cfg, void* d_weights, float* d_params,
               float* d_m, float* d_v, int32_t* h_step, int32_t T, const float* d_obs,
               const uint8_t* d_actions, const float* d_logp_old, const double* d_adv,
               const double* d_ret, double* d_losses);

/* Operators for policies that the caller's own network computes (a sequence model, a router, an
 * action set of any size): the recurrence, linear attention, the policy loss, a router's balance
 * loss and log-probabilities, each with its gradient, and the step of matrices. They use a context for its stream, its device and its error flags only,
 * whatever its configuration; the sizes are their own. Common to them:
 *   - Work memory is the caller's: the *_work calls (no device work) give the bytes, 16-byte
 *     aligned memory; nothing need be in it, and calls that may overlap (two streams, two
 *     graphs) take one each. They allocate nothing and may be captured into a graph (with
 *     sim_set_timing off); the current device may be another than the context's.
 *   - Values are fp64, fp32, bf16 or fp16 (SIM_DT_*), computed in fp32 (fp64 for fp64) and
 *     rounded once, to nearest, on output.
 *   - Strides are in elements. An input may be broadcast by a stride of 0; the elements of an
 *     output must not share memory (SIM_EINVAL). Outputs may not overlap inputs but where
 *     stated. Every array must be aligned to its element. Sizes of 0 are allowed.
 *   - Sums run in a fixed order: repeated calls return the same bits.
 *   - While tracing (sim_set_timing) the recurrence and linear attention count as SIM_KC_GAE, the
 *     others as SIM_KC_PPO.                                                                */
enum { SIM_DT_F64 = 0, SIM_DT_F32 = 1, SIM_DT_BF16 = 2, SIM_DT_F16 = 3 };
enum { SIM_IT_U8 = 0, SIM_IT_I32 = 1, SIM_IT_I64 = 2 };
enum { SIM_GATE_LINEAR = 0, SIM_GATE_SIGMOID = 1 };

/* An array over sequences, steps and channels: element (b, t, d) at b*stride_b + t*stride_t + d. */
typedef struct sim_seq {
  void* data;
  int64_t stride_b, stride_t;
} sim_seq;

/* A matrix over samples and actions: element (n, a) at n*stride_n + a*stride_a. Of logits and
 * their gradient one of the two strides is 1 (rows of actions, or sim_policy's [A][E] logits),
 * unless a dimension is 1. Adjacent samples suit many samples of up to some hundred actions: with
 * more than 384 actions 64 samples share a workgroup, so few samples of many actions are far slower
 * than as rows (bf16 2048 x 50257 2.5 ms, as rows 110 us).                                 */
typedef struct sim_mat {
  void* data;
  int64_t stride_n, stride_a;
} sim_mat;

/* Gated linear recurrence: the recurrence of returns_gae with a gate per step and channel
 * (episodes that end inside a rollout, per-token discounts; Sec. 4.3) and the state of a
 * recurrent policy.
 *  dtype      type of the arrays over steps; states are fp64 for SIM_DT_F64 and fp32 otherwise
 *  kind       SIM_GATE_LINEAR:  h = gate_t h + x_t
 *             SIM_GATE_SIGMOID: f = 1 / (1 + exp(-gate_t)), h = f h + (1 - f) x_t
 *  reverse    0: t = 0, 1, ..; 1: from the last step back to t = 0
 *  B, T, D    sequences, steps (below 2^30), channels (B D below 2^31)                    */
typedef struct sim_scan {
  int32_t dtype, kind, reverse;
  int64_t B, T, D;
} sim_scan;

/* y_t = the state after step t, from the state d_h0 [B][D] (NULL: 0); d_state [B][D] (NULL: not
 * wanted) receives the state after the last step and may be d_h0 itself (serving: T = 1, the
 * state updated in place). y may be NULL (only the state is wanted). d_len [B] int32 (NULL: all
 * T): steps t >= d_len[b] are padding, whatever they hold: they leave the state as it is and
 * their y is 0; a length outside [0, T] latches SIM_ESTATE and is taken as the nearer bound.
 * Up to T = 4 steps are taken one after another. With more, and in the gradient whatever T, a
 * sequence is cut into runs of steps whose gates are multiplied up and joined, runs of any length up
 * to the whole sequence: results differ from a step-by-step sum by rounding, and the product of the
 * gates over any run of steps must be finite in the state's type (an infinite one makes NaN of a state
 * of 0, also where every state is finite). What reaches a state through a run whose product is below
 * the type's smallest number (fp32 2^-149) is lost, also where later gates above 1 would make it large
 * again. With |gate| <= 1, as the factors of sigmoid gates are, products are finite and what is lost
 * is below 2^-149 of the state that it comes from.                                        */
int gated_scan_work(const sim_scan* s, size_t* bytes);
int gated_scan(sim_ctx* ctx, const sim_scan* s, const sim_seq* gate, const sim_seq* x,
               const int32_t* d_len, const void* d_h0, const sim_seq* y, void* d_state,
               void* d_work, size_t work_bytes);

/* Its gradient: from dy and d_dstate [B][D] (gradient of the last state, NULL: 0) the gradients
 * of gate, x and h0 (dgate, dx, d_dh0; each may be NULL). In the opposite order of steps, with
 * C = dstate at first and h' the state before a step (y of the step before it as stored, or h0):
 *   G_t = dy_t + C;  linear:  dx_t = G_t,          dgate_t = G_t h',                 C = gate_t G_t
 *                    sigmoid: dx_t = (1 - f) G_t,  dgate_t = G_t (h' - x_t) f (1 - f),  C = f G_t
 * and dh0 = C at the end. Padding gets 0. The gates' products must be finite as above, with any T.
 * x is read for SIM_GATE_SIGMOID only, y only if dgate is wanted (either may be NULL otherwise).
 * The gradient of a broadcast input is the sum over the dimension it is broadcast along of what is
 * written here, which is left to the caller.                                              */
int gated_scan_grad_work(const sim_scan* s, size_t* bytes);
int gated_scan_grad(sim_ctx* ctx, const sim_scan* s, const sim_seq* gate, const sim_seq* x,
                    const sim_seq* y, const sim_seq* dy, const int32_t* d_len, const void* d_h0,
                    const void* d_dstate, const sim_seq* dgate, const sim_seq* dx, void* d_dh0,
                    void* d_work, size_t work_bytes);

/* Clipped policy loss with a KL term over logits of any network, and its gradient: the
 * surrogate of ppo_minibatch_grad (Sec. 4.3) without its network.
 *  N, A         samples (below 2^31) and actions (below 2^30)
 *  dtype        of logits and gradient (not SIM_DT_F64)
 *  action_type  SIM_IT_*;  adv_type  SIM_DT_F32 or SIM_DT_F64 (as returns_gae writes them)
 *  clip         in (0, 1); c_kl, c_entropy >= 0                                          */
typedef struct sim_policy_loss {
  int64_t N;
  int32_t A, dtype, action_type, adv_type;
  float clip, c_kl, c_entropy;
} sim_policy_loss;

/* With p the softmax of a sample's logits over its allowed actions, logp that of the taken
 * action, rho = exp(logp - logp_old), d = logp_ref - logp and H the entropy of p:
 *   L = sum_n w_n (-min(rho adv, clip(rho, 1-clip, 1+clip) adv) + c_kl (e^d - d - 1) - c_entropy H)
 * (e^d - d - 1: an estimate of KL(p || reference) at the taken action, never negative).
 * mask [N][A] bytes (NULL: all allowed; any strides, stride_n = 0 to share a row): 0 forbids
 * an action, whatever its logit holds, and so does a logit of -inf. d_weight [N] (NULL:
 * 1/N each): samples of weight 0 are not looked at. d_logp_old NULL: logp itself (the first step
 * after a rollout: rho = 1). d_logp_ref may be NULL if c_kl = 0; then it gives d_loss[2] alone,
 * and no part of L or grad, infinite or not. Outputs: grad dL/dlogits (may be
 * NULL, or the logits themselves: same pointer and strides), d_logp [N] (may be NULL), d_loss [4]
 * fp32: L and its policy, KL and entropy terms (sums of w times each, without the c's; summed in
 * fp64). A sample of weight 0, or with no allowed action, gives nothing: gradient 0, logp 0. So
 * does one whose action is out of range or forbidden, which also latches SIM_ESTATE.       */
int policy_loss_work(const sim_policy_loss* c, size_t* bytes);
int policy_loss(sim_ctx* ctx, const sim_policy_loss* c, const sim_mat* logits, const sim_mat* mask,
                const void* d_actions, const float* d_weight, const float* d_logp_old,
                const float* d_logp_ref, const void* d_adv, const sim_mat* grad, float* d_logp,
                float* d_loss, void* d_work, size_t work_bytes);

/* Balance loss of a router (a policy that sends each request to one of several servers, Sec. 4.1,
 * or each token to k of A experts), its counts and its gradient.
 *  N, A, k      rows (below 2^31), columns (below 2^30), choices per row (N k below 2^31)
 *  group        consecutive columns that count as one target: 1, or 6 for this simulator's
 *               actions (server a/6); divides A, A/group <= 4096
 *  dtype        of logits and gradient (not SIM_DT_F64);  index_type  SIM_IT_*
 *  coef         the loss's factor                                                        */
typedef struct sim_balance {
  int64_t N;
  int32_t A, k, group, dtype, index_type;
  float coef;
} sim_balance;

/* With W live rows (d_live [N] bytes, NULL: all), G = A/group targets, p the softmax of a row's
 * logits: f_g = counts_g / (k W), P_g the mean over live rows of p summed over g's columns,
 *   L = coef G sum_g f_g P_g,   dL/dlogit_nj = coef G / W p_nj (f_g(j) - sum_i f_g(i) p_ni)
 * (f held constant). d_index [N][k]: the chosen columns; -1 (not with SIM_IT_U8) is no choice, any
 * other value outside [0, A) latches SIM_ESTATE and counts for nothing. Outputs: d_counts
 * [G] int64, the live rows' choices; d_loss [1] fp32 (summed in fp64); grad (may be NULL, or the
 * logits themselves). Rows that are not live, or whose logits are all -inf, add nothing to P
 * and have gradient 0; W = 0 gives L = 0.                                                  */
int balance_loss_work(const sim_balance* c, size_t* bytes);
int balance_loss(sim_ctx* ctx, const sim_balance* c, const sim_mat* logits, const void* d_index,
                 const uint8_t* d_live, const sim_mat* grad, int64_t* d_counts, float* d_loss,
                 void* d_work, size_t work_bytes);

/* ---- a sequence layer, log-probabilities and updates of the caller's own network ------------
 * Linear attention with a decay for each head: a state that is a matrix, beside gated_scan's vector.
 * An array over sequences, steps, heads and channels: element (b, t, h, d) at b*stride_b +
 * t*stride_t + h*stride_h + d.                                                             */
typedef struct sim_heads {
  void* data;
  int64_t stride_b, stride_t, stride_h;
} sim_heads;

/*  B, T    sequences, steps (below 2^30)
 *  H, Hk   heads of q and y, heads of k and v: Hk divides H, and heads [i H/Hk, (i+1) H/Hk) share
 *          the keys and values i (B H below 2^21, B T H below 2^40)
 *  Dk, Dv  channels of q and k, of v and y: 1 to 256 each
 *  dtype   of q, k, v, y and their gradients (not SIM_DT_F64); states are fp32
 *  scale   finite                                                                         */
typedef struct sim_linear_attn {
  int64_t B, T;
  int32_t H, Hk, Dk, Dv, dtype;
  float scale;
} sim_linear_attn;

/* Per sequence b and head h, from S = d_s0[b][h] ([B][H][Dk][Dv] contiguous fp32, NULL: 0), with l =
 * d_decay[h] (fp32, in [0, 1]):
 *   S = l S + k_t v_t^T,   y_t = scale S^T q_t,     t = 0, 1, ..
 * d_state [B][H][Dk][Dv] (NULL: not wanted) receives S after the last step and may be d_s0 itself
 * (serving: T = 1, the state updated in place). y may be NULL (only the state is wanted). d_len [B]
 * int32 (NULL: all T): steps t >= d_len[b] are padding, whatever they hold: they leave S as it is and
 * their y is 0; a length outside [0, T] latches SIM_ESTATE and is taken as the nearer bound, and so
 * does a decay outside [0, 1] (NaN as 0).
 * Up to T = 16 steps are taken one after another. With more, a run of steps is taken at once: the
 * products q_t k_s, weighted by l^(t-s), and the state between runs are held in fp32 and multiplied, for y
 * alone, as bf16 parts that add up to them (two for 16-bit types, 16 bits of the value; three for fp32, all
 * 24), and results differ from a step-by-step sum by rounding. What the formulas make infinite or NaN, for
 * an infinity or NaN of a live step or because fp32 (or bf16's largest, 3.39e38) is passed on the way, is
 * infinite or NaN, not always the same of the two; what they make without it is not touched by it. */
int linear_attn_work(const sim_linear_attn* s, size_t* bytes);
int linear_attn(sim_ctx* ctx, const sim_linear_attn* s, const sim_heads* q, const sim_heads* k,
                const sim_heads* v, const float* d_decay, const int32_t* d_len, const float* d_s0,
                const sim_heads* y, float* d_state, void* d_work, size_t work_bytes);

/* Its gradient: from dy and d_dstate [B][H][Dk][Dv] (gradient of the last state, NULL: 0) those of q, k,
 * v and s0 (each may be NULL; d_ds0 may be d_dstate). With G the gradient of S after a step,
 *   G_t = scale q_t dy_t^T + l G_{t+1} (after the last step + dstate),
 *   dq_t = scale S_t dy_t,  dk_t = sum over the heads that share it of G_t v_t,  dv_t = .. of G_t^T k_t
 * and ds0 = l G_0. The decays are constants of the layer and get no gradient. Padding gets 0. The
 * states are formed again from q, k and v: nothing is kept of the forward call.               */
int linear_attn_grad_work(const sim_linear_attn* s, size_t* bytes);
int linear_attn_grad(sim_ctx* ctx, const sim_linear_attn* s, const sim_heads* q, const sim_heads* k,
                     const sim_heads* v, const float* d_decay, const sim_heads* dy,
                     const int32_t* d_len, const float* d_s0, const float* d_dstate,
                     const sim_heads* dq, const sim_heads* dk, const sim_heads* dv, float* d_ds0,
                     void* d_work, size_t work_bytes);

/* Log-probabilities of given tokens (actions) over the logits of any network, the entropy and the
 * likeliest columns: what policy_loss takes as d_logp_old and d_logp_ref, and what is told of a choice.
 *  N, A        rows (below 2^31), columns (below 2^30)
 *  top         alternatives per row, 0 to 64
 *  dtype       of logits and gradient (not SIM_DT_F64);  token_type  SIM_IT_*             */
typedef struct sim_logprobs {
  int64_t N;
  int32_t A, top, dtype, token_type;
} sim_logprobs;

/* With p the softmax of a row's logits over its allowed columns (mask [N][A] bytes as for policy_loss,
 * NULL: all; a logit of -inf is forbidden too): d_logp [N] = log p of the given token (-inf if it is
 * forbidden), d_entropy [N] = -sum p log p, d_top_index [N][top] int64 the columns of the largest logits,
 * largest first and of equal ones the lowest column first (a NaN counts as the largest), and d_top_logp
 * [N][top] their log p. Where a row allows fewer than top columns the rest is -1 and -inf. Each output may be
 * NULL; d_tokens may be NULL if d_logp is. A token of -1 (not with SIM_IT_U8) is none: its logp is 0; any
 * other outside [0, A) latches SIM_ESTATE and is taken as none. Rows with d_live [N] bytes (NULL: all) 0
 * are not looked at; they, and rows that allow no column, give nothing: logp 0, entropy 0, no
 * alternatives. Alternatives are best had of rows of adjacent columns, or of up to 960 columns.  */
int token_logprobs_work(const sim_logprobs* c, size_t* bytes);
int token_logprobs(sim_ctx* ctx, const sim_logprobs* c, const sim_mat* logits, const sim_mat* mask,
                   const void* d_tokens, const uint8_t* d_live, float* d_logp, float* d_entropy,
                   int64_t* d_top_index, float* d_top_logp, void* d_work, size_t work_bytes);

/* The gradient over the logits of sum_n (d_dlogp[n] logp_n + d_dentropy[n] H_n) (either may be NULL: 0):
 *   dl_j = dlogp (1[j = token] - p_j) - dentropy p_j (log p_j + H)
 * Forbidden columns, and rows that give nothing, get 0; of a row whose token is none or forbidden only the
 * entropy's part is left. grad may be the logits themselves (same pointer and strides). top is not looked at. */
int token_logprobs_grad_work(const sim_logprobs* c, size_t* bytes);
int token_logprobs_grad(sim_ctx* ctx, const sim_logprobs* c, const sim_mat* logits, const sim_mat* mask,
                        const void* d_tokens, const uint8_t* d_live, const float* d_dlogp,
                        const float* d_dentropy, const sim_mat* grad, void* d_work, size_t work_bytes);

/* Matrices: element (i, r, c) at i*stride_i + r*stride_r + c*stride_c. */
typedef struct sim_mats {
  void* data;
  int64_t stride_i, stride_r, stride_c;
} sim_mats;

/* An update orthogonalised by Newton-Schulz products, for the matrices of a network beside adam_update's
 * step: a polynomial that takes the singular values of U / |U| towards 1 and leaves the singular vectors.
 *  n, M, N   matrices, rows and columns (up to 65536 each, n below 2^16)
 *  steps     0 to 32;  dtype  of U and the result (not SIM_DT_F64)
 *  a, b, c   the polynomial's coefficients;  eps >= 0;  scale  of the result             */
typedef struct sim_ortho {
  int64_t n, M, N;
  int32_t steps, dtype;
  float a, b, c, eps, scale;
} sim_ortho;

/* X = U / (|U|_F + eps), then `steps` times, with A = X X^T (X^T X for M > N, which comes to the same),
 *   X = a X + (b A + c A A) X
 * and out = scale X. The norm is summed in fp64, sums of products in fp32; between products X, A and
 * b A + c A A are held as two fp16 parts (22 bits) of the value times 2^10, in steps of 2^-34 at the
 * finest (an update whose norm lies far below eps keeps fewer bits). So singular values, and A's and the
 * polynomial's, must stay below 60 (with the usual coefficients they stay below 4). U and out may have
 * any strides and be the same memory; a matrix of zeros gives zeros, one that holds an infinity or NaN
 * gives NaN.                                                                               */
int orthogonalize_work(const sim_ortho* c, size_t* bytes);
int orthogonalize(sim_ctx* ctx, const sim_ortho* c, const sim_mats* update, const sim_mats* out,
                  void* d_work, size_t work_bytes);

/* Per-environment counters [2][SIM_NCNT][E] int64 and sums [2][SIM_NSUM][E] fp64 into
 * device buffers (either may be NULL).                                                  */
int sim_counters(sim_ctx* ctx, int64_t* d_cnt, double* d_sum);

/* Per-environment integer-state checksums [2][E] (learned, shadow) into d_chk.          */
int sim_checksums(sim_ctx* ctx, uint64_t* d_chk);

/* Totals of the counters over all environments, reduced on the device, into h_out.
 * Synchronises the stream.                                                              */
int sim_stats(sim_ctx* ctx, sim_totals* h_out);

/* Waits for the stream; returns SIM_ESTATE if a device-side error was latched (and
 * clears it), with the reason in sim_last_error().                                     */
int sim_sync(sim_ctx* ctx);

/* Checkpoint and resume of the simulation: a snapshot holds every environment's state of both
 * systems (queues and timestamp rings, servers, counters, sums and checksums, arrival
 * processes, arrival-rate averages, the current observation, latched error flags) and the
 * context's tick counter and seed, behind a 256-byte header. sim_get_state with buf = NULL
 * stores the snapshot size in *bytes; otherwise *bytes must be at least that size and buf
 * (device or host memory) receives the snapshot after the work already enqueued on the
 * stream; the copy is complete when the call returns. sim_set_state restores a snapshot
 * into a context whose configuration has the same layout (n_envs, n_servers, n_classes,
 * queue_cap, obs_dim, shadow; SIM_EINVAL otherwise, or for a buffer that is not a snapshot
 * of this library version). Trace arrivals (sim_set_trace) are caller memory and not part
 * of the snapshot: set the same trace again before resuming. Continuing from a restored
 * snapshot reproduces the original continuation bit for bit (the counter-based random
 * draws depend only on the seed, the environment and the tick).                          */
int sim_get_state(sim_ctx* ctx, void* buf, size_t* bytes);
int sim_set_state(sim_ctx* ctx, const void* buf, size_t bytes);

/* Diagnostics: one of the library's device primitives evaluated elementwise on n inputs, so
 * that its bit identity with a host implementation can be checked directly (the parity of
 * whole rollouts depends on it). All arrays are device memory owned by the caller; the work
 * is enqueued on hip_stream (NULL: the default stream) and complete after it synchronizes.
 *   SIM_PRIM_PHILOX  d_in uint32 [n][4] counters, d_out uint32 [n][4]: the Philox4x32-10
 *                    block of each counter under the 64-bit key (low word first) (R13)
 *   SIM_PRIM_LOG, SIM_PRIM_EXP, SIM_PRIM_COS  fp64 [n] -> fp64 [n]: the deterministic
 *                    logarithm, exponential and cosine of the arrival and service draws (R14)
 *   SIM_PRIM_SQRT    fp64 [n] -> fp64 [n], correctly rounded square root
 *   SIM_PRIM_DIV     fp64 [n][2] -> fp64 [n], the first of each pair divided by the second
 * SIM_EINVAL for an unknown kind, n < 0 or NULL arrays with n > 0.                          */
enum { SIM_PRIM_PHILOX = 0, SIM_PRIM_LOG = 1, SIM_PRIM_EXP = 2, SIM_PRIM_COS = 3,
       SIM_PRIM_SQRT = 4, SIM_PRIM_DIV = 5 };
int sim_device_primitive(int32_t kind, int64_t n, uint64_t key, const void* d_in, void* d_out,
                         void* hip_stream);

/* Kernel classes for tracing. */
enum sim_kernel_class {
  SIM_KC_POLICY = 0,  /* policy MLP + sampler */
  SIM_KC_STEP = 1,    /* learned system, one tick */
  SIM_KC_STATIC = 2,  /* static shadow system, one tick */
  SIM_KC_GAE = 3,     /* returns / GAE, gated_scan, linear_attn and their gradients */
  SIM_KC_RESET = 4,   /* reset */
  SIM_KC_OTHER = 5,   /* weight repack / init, observation packing, counters, totals */
  SIM_KC_PPO = 6,     /* policy update: minibatch gradients, Adam, policy_loss, balance_loss,
                         token_logprobs and its gradient, orthogonalize */
  SIM_KC_ROLLOUT = 7, /* fused rollout: every tick's policy and learned tick in one launch */
  SIM_KC_COUNT = 8
};

/* Tracing: with `on` != 0 every kernel launch of the context is bracketed by a pair of
 * HIP events recorded on the context's stream. sim_get_timing synchronises the stream
 * and adds the elapsed time of every completed pair to per-class totals, then writes the
 * totals (milliseconds) and launch counts to h_ms[SIM_KC_COUNT] and
 * h_launches[SIM_KC_COUNT]; `clear` != 0 zeroes the totals afterwards.               */
int sim_set_timing(sim_ctx* ctx, int32_t on);
int sim_get_timing(sim_ctx* ctx, double* h_ms, int64_t* h_launches, int32_t clear);

#ifdef __cplusplus
}
#endif
#endif /* BATCHSIM_H */
