// ops.cpp -- entry points of the operators for the caller's own networks (include/batchsim.h):
// checks of sizes, strides and work memory on the host, then their launches on the context's
// stream and device. Nothing is allocated.
#include <algorithm>
#include <utility>

#include "ops.hpp"

using namespace bsim;

namespace {

constexpr int64_t kMax31 = 0x7FFFFFFF;

int elem_bytes(int dtype) { return dtype == SIM_DT_F64 ? 8 : (dtype == SIM_DT_F32 ? 4 : 2); }

// The context's device as the current one while an operator launches.
struct OnDevice {
  int prev = -1, want;
  hipError_t e = hipSuccess;
  explicit OnDevice(int d) : want(d) {
    e = hipGetDevice(&prev);
    if (e == hipSuccess && prev != want) e = hipSetDevice(want);
  }
  ~OnDevice() {
    if (e == hipSuccess && prev != want) (void)hipSetDevice(prev);
  }
};

template <class F>
int on_ctx(sim_ctx* x, int cls, const char* who, F f) try {
  OnDevice dev(op_ctx(x).device);
  hipError_t e = dev.e;
  if (e == hipSuccess)
    e = op_timed(x, cls, [](void* p) { return (*static_cast<F*>(p))(); }, &f);
  if (e != hipSuccess) return op_fail(SIM_EDEVICE, "%s: kernel launch: %s", who, hipGetErrorString(e));
  return SIM_OK;
} catch (...) {
  return op_fail(SIM_ENOMEM, "%s: host allocation failed", who);
}

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// whether n0 x n1 elements at these strides, in runs of `run`, fit 63-bit byte offsets
bool fits(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t run, int eb) {
  const __int128 last = (__int128)std::max<int64_t>(n0 - 1, 0) * s0 +
                        (__int128)std::max<int64_t>(n1 - 1, 0) * s1 + run;
  return last * eb <= ((__int128)1 << 62);
}
// whether runs of `run` elements at n0 x n1 places share no element: the inner of the two
// dimensions steps over a run, the outer one over all of the inner
bool distinct(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t run) {
  if (!n0 || !n1) return true;
  std::pair<int64_t, int64_t> d[2] = {{s0, n0}, {s1, n1}};
  if (d[1].first < d[0].first) std::swap(d[0], d[1]);
  __int128 span = run;
  for (const auto& [s, n] : d) {
    if (n <= 1) continue;
    if (s < span) return false;
    span += (__int128)s * (n - 1);
  }
  return true;
}

int check_scan(const sim_scan* s, const char* who) {
  if (!s) return op_fail(SIM_EINVAL, "%s: sizes are NULL", who);
  if (s->dtype < SIM_DT_F64 || s->dtype > SIM_DT_F16) return op_fail(SIM_EINVAL, "%s: unknown dtype %d", who, s->dtype);
  if (s->kind != SIM_GATE_LINEAR && s->kind != SIM_GATE_SIGMOID)
    return op_fail(SIM_EINVAL, "%s: unknown kind %d", who, s->kind);
  if (s->reverse != 0 && s->reverse != 1) return op_fail(SIM_EINVAL, "%s: reverse must be 0 or 1", who);
  if (s->B < 0 || s->T < 0 || s->D < 0) return op_fail(SIM_EINVAL, "%s: B, T and D must be >= 0", who);
  if (s->T >= (1 << 30) || s->B > kMax31 || s->D > kMax31 || s->B * s->D > kMax31)
    return op_fail(SIM_EUNSUPPORTED, "%s: T must stay below 2^30, B*D below 2^31", who);
  return SIM_OK;
}

// one array over steps; `need`: it may not be absent, `out`: its elements are written
int check_seq(const sim_scan& c, const sim_seq* q, bool need, bool out, const char* who, const char* name,
              sim_seq* got) {
  *got = sim_seq{nullptr, 0, 0};
  if (!q || !q->data) {
    if (need && c.B && c.T && c.D) return op_fail(SIM_EINVAL, "%s: %s is NULL", who, name);
    return SIM_OK;
  }
  if (q->stride_b < 0 || q->stride_t < 0) return op_fail(SIM_EINVAL, "%s: negative stride of %s", who, name);
  if (!fits(c.B, q->stride_b, c.T, q->stride_t, c.D, elem_bytes(c.dtype)))
    return op_fail(SIM_EINVAL, "%s: strides of %s pass 2^62 bytes", who, name);
  if (!aligned(q->data, elem_bytes(c.dtype))) return op_fail(SIM_EINVAL, "%s: %s is not aligned to its type", who, name);
  if (out && c.D && !distinct(c.B, q->stride_b, c.T, q->stride_t, c.D))
    return op_fail(SIM_EINVAL, "%s: elements of %s share memory", who, name);
  *got = *q;
  return SIM_OK;
}

int check_work(const void* work, size_t have, size_t need, const char* who) {
  if (have < need || (need && !work))
    return op_fail(SIM_EINVAL, "%s: needs %zu bytes of work memory, has %zu", who, need, work ? have : (size_t)0);
  if (need && !aligned(work, 16)) return op_fail(SIM_EINVAL, "%s: work memory must be 16-byte aligned", who);
  return SIM_OK;
}

int check_mat(int64_t N, int64_t A, const sim_mat* m, int eb, bool strided, bool out, const char* who,
              const char* name) {
  if (m->stride_n < 0 || m->stride_a < 0) return op_fail(SIM_EINVAL, "%s: negative stride of %s", who, name);
  if (strided && m->stride_n != 1 && m->stride_a != 1 && N > 1 && A > 1)
    return op_fail(SIM_EUNSUPPORTED, "%s: one stride of %s must be 1", who, name);
  if (!fits(N, m->stride_n, A, m->stride_a, 1, eb)) return op_fail(SIM_EINVAL, "%s: strides of %s pass 2^62 bytes", who, name);
  if (!aligned(m->data, eb)) return op_fail(SIM_EINVAL, "%s: %s is not aligned to its type", who, name);
  if (out && !distinct(N, m->stride_n, A, m->stride_a, 1))
    return op_fail(SIM_EINVAL, "%s: elements of %s share memory", who, name);
  return SIM_OK;
}

// logits and gradient of either loss
int check_logits(int64_t N, int32_t A, int32_t dtype, const sim_mat* logits, const sim_mat* grad,
                 const char* who, sim_mat* l, sim_mat* g) {
  *l = *g = sim_mat{nullptr, 0, 0};
  if (N > 0 && (!logits || !logits->data)) return op_fail(SIM_EINVAL, "%s: logits is NULL", who);
  int rc = SIM_OK;
  if (logits && logits->data) {
    rc = check_mat(N, A, logits, elem_bytes(dtype), true, false, who, "logits");
    if (rc) return rc;
    *l = *logits;
  }
  if (grad && grad->data) {
    rc = check_mat(N, A, grad, elem_bytes(dtype), true, true, who, "grad");
    if (rc) return rc;
    if (grad->data == l->data && ((N > 1 && grad->stride_n != l->stride_n) || (A > 1 && grad->stride_a != l->stride_a)))
      return op_fail(SIM_EINVAL, "%s: grad is the logits' memory with other strides", who);
    *g = *grad;
  }
  return SIM_OK;
}

int check_policy(const sim_policy_loss* c, const char* who) {
  if (!c) return op_fail(SIM_EINVAL, "%s: sizes are NULL", who);
  if (c->N < 0 || c->N > kMax31) return op_fail(SIM_EINVAL, "%s: N must lie in [0, 2^31)", who);
  if (c->A < 1) return op_fail(SIM_EINVAL, "%s: A must be >= 1", who);
  if (c->A >= (1 << 30)) return op_fail(SIM_EUNSUPPORTED, "%s: A must stay below 2^30", who);
  if (c->dtype < SIM_DT_F32 || c->dtype > SIM_DT_F16) return op_fail(SIM_EINVAL, "%s: logits of type %d", who, c->dtype);
  if (c->action_type < SIM_IT_U8 || c->action_type > SIM_IT_I64)
    return op_fail(SIM_EINVAL, "%s: unknown action type %d", who, c->action_type);
  if (c->adv_type != SIM_DT_F64 && c->adv_type != SIM_DT_F32)
    return op_fail(SIM_EINVAL, "%s: advantages are fp32 or fp64", who);
  if (!(c->clip > 0.0f && c->clip < 1.0f)) return op_fail(SIM_EINVAL, "%s: clip must lie in (0, 1)", who);
  if (!(c->c_kl >= 0.0f && c->c_entropy >= 0.0f))
    return op_fail(SIM_EINVAL, "%s: c_kl and c_entropy must be >= 0", who);
  return SIM_OK;
}

int check_balance(const sim_balance* c, const char* who) {
  if (!c) return op_fail(SIM_EINVAL, "%s: sizes are NULL", who);
  if (c->N < 0 || c->N > kMax31) return op_fail(SIM_EINVAL, "%s: N must lie in [0, 2^31)", who);
  if (c->A < 1 || c->k < 1) return op_fail(SIM_EINVAL, "%s: A and k must be >= 1", who);
  if (c->A >= (1 << 30)) return op_fail(SIM_EUNSUPPORTED, "%s: A must stay below 2^30", who);
  if (c->N * c->k > kMax31) return op_fail(SIM_EUNSUPPORTED, "%s: N*k must stay below 2^31", who);
  if (c->group < 1 || c->A % c->group) return op_fail(SIM_EINVAL, "%s: group must divide A", who);
  if (c->A / c->group > 4096) return op_fail(SIM_EUNSUPPORTED, "%s: at most 4096 targets", who);
  if (c->dtype < SIM_DT_F32 || c->dtype > SIM_DT_F16) return op_fail(SIM_EINVAL, "%s: logits of type %d", who, c->dtype);
  if (c->index_type < SIM_IT_U8 || c->index_type > SIM_IT_I64)
    return op_fail(SIM_EINVAL, "%s: unknown index type %d", who, c->index_type);
  return SIM_OK;
}

// three strided dimensions and runs of adjacent elements: the offsets stay below 2^62 bytes, and of an
// output no two elements are the same
struct Dim { int64_t stride, n; };
int check_box(const void* data, const Dim (&dims)[3], int64_t run, int eb, bool out, const char* who,
              const char* name) {
  __int128 last = run;
  bool some = run > 0;
  for (const Dim& d : dims) {
    if (d.stride < 0) return op_fail(SIM_EINVAL, "%s: negative stride of %s", who, name);
    last += (__int128)std::max<int64_t>(d.n - 1, 0) * d.stride;
    some = some && d.n > 0;
  }
  if (last * eb > ((__int128)1 << 62)) return op_fail(SIM_EINVAL, "%s: strides of %s pass 2^62 bytes", who, name);
  if (!aligned(data, eb)) return op_fail(SIM_EINVAL, "%s: %s is not aligned to its type", who, name);
  if (out && some) {
    Dim s[3] = {dims[0], dims[1], dims[2]};
    std::sort(s, s + 3, [](const Dim& p, const Dim& q) { return p.stride < q.stride; });
    __int128 span = run;
    for (const Dim& d : s) {
      if (d.n <= 1) continue;
      if (d.stride < span) return op_fail(SIM_EINVAL, "%s: elements of %s share memory", who, name);
      span += (__int128)d.stride * (d.n - 1);
    }
  }
  return SIM_OK;
}

int check_attn(const sim_linear_attn* s, const char* who) {
  if (!s) return op_fail(SIM_EINVAL, "%s: sizes are NULL", who);
  if (s->dtype < SIM_DT_F32 || s->dtype > SIM_DT_F16) return op_fail(SIM_EINVAL, "%s: arrays of type %d", who, s->dtype);
  if (s->B < 0 || s->T < 0) return op_fail(SIM_EINVAL, "%s: B and T must be >= 0", who);
  if (s->H < 1 || s->Hk < 1 || s->H % s->Hk) return op_fail(SIM_EINVAL, "%s: Hk must be >= 1 and divide H", who);
  if (s->Dk < 1 || s->Dv < 1) return op_fail(SIM_EINVAL, "%s: Dk and Dv must be >= 1", who);
  if (s->Dk > 256 || s->Dv > 256) return op_fail(SIM_EUNSUPPORTED, "%s: Dk and Dv go up to 256", who);
  if (!(s->scale - s->scale == 0.0f)) return op_fail(SIM_EINVAL, "%s: scale must be finite", who);
  if (s->T >= (1 << 30) || s->B >= (1 << 21) || s->B * s->H >= (1 << 21) ||
      (__int128)s->B * s->T * s->H >= ((__int128)1 << 40))
    return op_fail(SIM_EUNSUPPORTED, "%s: T must stay below 2^30, B*H below 2^21, B*T*H below 2^40", who);
  return SIM_OK;
}

// one array over steps and heads; `need`: it may not be absent, `out`: its elements are written
int check_heads(const sim_linear_attn& c, const sim_heads* x, int H, int D, bool need, bool out, const char* who,
                const char* name, sim_heads* got) {
  *got = sim_heads{nullptr, 0, 0, 0};
  if (!x || !x->data) {
    if (need && c.B && c.T) return op_fail(SIM_EINVAL, "%s: %s is NULL", who, name);
    return SIM_OK;
  }
  const Dim dims[3] = {{x->stride_b, c.B}, {x->stride_t, c.T}, {x->stride_h, H}};
  *got = *x;
  return check_box(x->data, dims, D, elem_bytes(c.dtype), out, who, name);
}

int check_logprobs(const sim_logprobs* c, const char* who) {
  if (!c) return op_fail(SIM_EINVAL, "%s: sizes are NULL", who);
  if (c->N < 0 || c->N > kMax31) return op_fail(SIM_EINVAL, "%s: N must lie in [0, 2^31)", who);
  if (c->A < 1) return op_fail(SIM_EINVAL, "%s: A must be >= 1", who);
  if (c->A >= (1 << 30)) return op_fail(SIM_EUNSUPPORTED, "%s: A must stay below 2^30", who);
  if (c->top < 0) return op_fail(SIM_EINVAL, "%s: top must be >= 0", who);
  if (c->top > 64) return op_fail(SIM_EUNSUPPORTED, "%s: at most 64 alternatives", who);
  if (c->dtype < SIM_DT_F32 || c->dtype > SIM_DT_F16) return op_fail(SIM_EINVAL, "%s: logits of type %d", who, c->dtype);
  if (c->token_type < SIM_IT_U8 || c->token_type > SIM_IT_I64)
    return op_fail(SIM_EINVAL, "%s: unknown token type %d", who, c->token_type);
  return SIM_OK;
}

int check_ortho(const sim_ortho* c, const char* who) {
  if (!c) return op_fail(SIM_EINVAL, "%s: sizes are NULL", who);
  if (c->n < 0 || c->M < 0 || c->N < 0) return op_fail(SIM_EINVAL, "%s: n, M and N must be >= 0", who);
  if (c->M > 65536 || c->N > 65536 || c->n >= 65536)
    return op_fail(SIM_EUNSUPPORTED, "%s: M and N go up to 65536, n below 65536", who);
  if (c->steps < 0 || c->steps > 32) return op_fail(SIM_EINVAL, "%s: steps must lie in [0, 32]", who);
  if (c->dtype < SIM_DT_F32 || c->dtype > SIM_DT_F16) return op_fail(SIM_EINVAL, "%s: matrices of type %d", who, c->dtype);
  for (const float v : {c->a, c->b, c->c, c->eps, c->scale})
    if (!(v - v == 0.0f)) return op_fail(SIM_EINVAL, "%s: coefficients, eps and scale must be finite", who);
  if (c->eps < 0.0f) return op_fail(SIM_EINVAL, "%s: eps must be >= 0", who);
  return SIM_OK;
}

int int_bytes(int t) { return t == SIM_IT_U8 ? 1 : (t == SIM_IT_I32 ? 4 : 8); }

}  // namespace

extern "C" {

int gated_scan_work(const sim_scan* s, size_t* bytes) {
  int rc = check_scan(s, "gated_scan_work");
  if (rc) return rc;
  if (!bytes) return op_fail(SIM_EINVAL, "gated_scan_work: bytes is NULL");
  *bytes = scan_work_bytes(*s, false);
  return SIM_OK;
}

int gated_scan(sim_ctx* x, const sim_scan* s, const sim_seq* gate, const sim_seq* xs, const int32_t* d_len,
               const void* d_h0, const sim_seq* y, void* d_state, void* d_work, size_t work_bytes) {
  const char* who = "gated_scan";
  if (!x) return op_fail(SIM_EINVAL, "%s: ctx is NULL", who);
  int rc = check_scan(s, who);
  if (rc) return rc;
  ScanArgs a{};
  a.c = *s;
  if ((rc = check_seq(*s, gate, true, false, who, "gate", &a.g))) return rc;
  if ((rc = check_seq(*s, xs, true, false, who, "x", &a.x))) return rc;
  if ((rc = check_seq(*s, y, false, true, who, "y", &a.y))) return rc;
  const size_t wide = s->dtype == SIM_DT_F64 ? 8 : 4;
  if (!aligned(d_len, 4) || !aligned(d_h0, wide) || !aligned(d_state, wide))
    return op_fail(SIM_EINVAL, "%s: lengths and states must be aligned to their type", who);
  if ((rc = check_work(d_work, work_bytes, scan_work_bytes(*s, false), who))) return rc;
  if (s->B * s->D == 0 || (!a.y.data && !d_state)) return SIM_OK;
  a.len = d_len; a.h0 = d_h0; a.state = d_state; a.work = d_work;
  const OpCtx o = op_ctx(x);
  a.err = o.err;
  return on_ctx(x, SIM_KC_GAE, who, [&] { return launch_scan(a, false, o.stream); });
}

int gated_scan_grad_work(const sim_scan* s, size_t* bytes) {
  int rc = check_scan(s, "gated_scan_grad_work");
  if (rc) return rc;
  if (!bytes) return op_fail(SIM_EINVAL, "gated_scan_grad_work: bytes is NULL");
  *bytes = scan_work_bytes(*s, true);
  return SIM_OK;
}

int gated_scan_grad(sim_ctx* x, const sim_scan* s, const sim_seq* gate, const sim_seq* xs, const sim_seq* y,
                    const sim_seq* dy, const int32_t* d_len, const void* d_h0, const void* d_dstate,
                    const sim_seq* dgate, const sim_seq* dx, void* d_dh0, void* d_work, size_t work_bytes) {
  const char* who = "gated_scan_grad";
  if (!x) return op_fail(SIM_EINVAL, "%s: ctx is NULL", who);
  int rc = check_scan(s, who);
  if (rc) return rc;
  ScanArgs a{};
  a.c = *s;
  if ((rc = check_seq(*s, dgate, false, true, who, "dgate", &a.dg))) return rc;
  if ((rc = check_seq(*s, dx, false, true, who, "dx", &a.dx))) return rc;
  if ((rc = check_seq(*s, gate, true, false, who, "gate", &a.g))) return rc;
  if ((rc = check_seq(*s, dy, true, false, who, "dy", &a.dy))) return rc;
  if ((rc = check_seq(*s, xs, a.dg.data && s->kind == SIM_GATE_SIGMOID, false, who, "x", &a.x))) return rc;
  if ((rc = check_seq(*s, y, a.dg.data, false, who, "y", &a.y))) return rc;
  const size_t wide = s->dtype == SIM_DT_F64 ? 8 : 4;
  if (!aligned(d_len, 4) || !aligned(d_h0, wide) || !aligned(d_dstate, wide) || !aligned(d_dh0, wide))
    return op_fail(SIM_EINVAL, "%s: lengths and states must be aligned to their type", who);
  if ((rc = check_work(d_work, work_bytes, scan_work_bytes(*s, true), who))) return rc;
  if (s->B * s->D == 0 || (!a.dg.data && !a.dx.data && !d_dh0)) return SIM_OK;
  a.len = d_len; a.h0 = d_h0; a.ds = d_dstate; a.state = d_dh0; a.work = d_work;
  const OpCtx o = op_ctx(x);
  a.err = o.err;
  return on_ctx(x, SIM_KC_GAE, who, [&] { return launch_scan(a, true, o.stream); });
}

int policy_loss_work(const sim_policy_loss* c, size_t* bytes) {
  int rc = check_policy(c, "policy_loss_work");
  if (rc) return rc;
  if (!bytes) return op_fail(SIM_EINVAL, "policy_loss_work: bytes is NULL");
  *bytes = policy_loss_bytes(*c);
  return SIM_OK;
}

int policy_loss(sim_ctx* x, const sim_policy_loss* c, const sim_mat* logits, const sim_mat* mask,
                const void* d_actions, const float* d_weight, const float* d_logp_old,
                const float* d_logp_ref, const void* d_adv, const sim_mat* grad, float* d_logp,
                float* d_loss, void* d_work, size_t work_bytes) {
  const char* who = "policy_loss";
  if (!x) return op_fail(SIM_EINVAL, "%s: ctx is NULL", who);
  int rc = check_policy(c, who);
  if (rc) return rc;
  PolicyLossArgs a{};
  a.c = *c;
  if ((rc = check_logits(c->N, c->A, c->dtype, logits, grad, who, &a.l, &a.grad))) return rc;
  if (mask && mask->data) {
    if ((rc = check_mat(c->N, c->A, mask, 1, false, false, who, "mask"))) return rc;
    a.mask = *mask;
  }
  if (!d_loss || (c->N > 0 && (!d_actions || !d_adv))) return op_fail(SIM_EINVAL, "%s: NULL argument", who);
  if (c->c_kl > 0.0f && !d_logp_ref && c->N > 0)
    return op_fail(SIM_EINVAL, "%s: c_kl > 0 needs reference log-probabilities", who);
  if (!aligned(d_actions, int_bytes(c->action_type)) || !aligned(d_adv, elem_bytes(c->adv_type)) ||
      !aligned(d_weight, 4) || !aligned(d_logp_old, 4) || !aligned(d_logp_ref, 4) || !aligned(d_logp, 4) ||
      !aligned(d_loss, 4))
    return op_fail(SIM_EINVAL, "%s: an array is not aligned to its type", who);
  if ((rc = check_work(d_work, work_bytes, policy_loss_bytes(*c), who))) return rc;
  a.act = d_actions; a.w = d_weight; a.logp_old = d_logp_old; a.logp_ref = d_logp_ref; a.adv = d_adv;
  a.logp = d_logp; a.loss = d_loss; a.work = d_work;
  const OpCtx o = op_ctx(x);
  a.err = o.err;
  return on_ctx(x, SIM_KC_PPO, who, [&] { return launch_policy_loss(a, o.stream); });
}

int balance_loss_work(const sim_balance* c, size_t* bytes) {
  int rc = check_balance(c, "balance_loss_work");
  if (rc) return rc;
  if (!bytes) return op_fail(SIM_EINVAL, "balance_loss_work: bytes is NULL");
  *bytes = balance_bytes(*c);
  return SIM_OK;
}

int balance_loss(sim_ctx* x, const sim_balance* c, const sim_mat* logits, const void* d_index,
                 const uint8_t* d_live, const sim_mat* grad, int64_t* d_counts, float* d_loss, void* d_work,
                 size_t work_bytes) {
  const char* who = "balance_loss";
  if (!x) return op_fail(SIM_EINVAL, "%s: ctx is NULL", who);
  int rc = check_balance(c, who);
  if (rc) return rc;
  BalanceArgs a{};
  a.c = *c;
  if ((rc = check_logits(c->N, c->A, c->dtype, logits, grad, who, &a.l, &a.grad))) return rc;
  if (!d_loss || !d_counts || (c->N > 0 && !d_index)) return op_fail(SIM_EINVAL, "%s: NULL argument", who);
  if (!aligned(d_index, int_bytes(c->index_type)) || !aligned(d_counts, 8) || !aligned(d_loss, 4))
    return op_fail(SIM_EINVAL, "%s: an array is not aligned to its type", who);
  if ((rc = check_work(d_work, work_bytes, balance_bytes(*c), who))) return rc;
  a.idx = d_index; a.live = d_live; a.counts = d_counts; a.loss = d_loss; a.work = d_work;
  const OpCtx o = op_ctx(x);
  a.err = o.err;
  return on_ctx(x, SIM_KC_PPO, who, [&] { return launch_balance(a, o.stream); });
}

int linear_attn_work(const sim_linear_attn* s, size_t* bytes) {
  int rc = check_attn(s, "linear_attn_work");
  if (rc) return rc;
  if (!bytes) return op_fail(SIM_EINVAL, "linear_attn_work: bytes is NULL");
  *bytes = attn_work_bytes(*s, false);
  return SIM_OK;
}

int linear_attn(sim_ctx* x, const sim_linear_attn* s, const sim_heads* q, const sim_heads* k, const sim_heads* v,
                const float* d_decay, const int32_t* d_len, const float* d_s0, const sim_heads* y,
                float* d_state, void* d_work, size_t work_bytes) {
  const char* who = "linear_attn";
  if (!x) return op_fail(SIM_EINVAL, "%s: ctx is NULL", who);
  int rc = check_attn(s, who);
  if (rc) return rc;
  AttnArgs a{};
  a.c = *s;
  if ((rc = check_heads(*s, y, s->H, s->Dv, false, true, who, "y", &a.y))) return rc;
  if ((rc = check_heads(*s, q, s->H, s->Dk, a.y.data, false, who, "q", &a.q))) return rc;
  if ((rc = check_heads(*s, k, s->Hk, s->Dk, true, false, who, "k", &a.k))) return rc;
  if ((rc = check_heads(*s, v, s->Hk, s->Dv, true, false, who, "v", &a.v))) return rc;
  if (!d_decay && s->B) return op_fail(SIM_EINVAL, "%s: decay is NULL", who);
  if (!aligned(d_decay, 4) || !aligned(d_len, 4) || !aligned(d_s0, 4) || !aligned(d_state, 4))
    return op_fail(SIM_EINVAL, "%s: decays, lengths and states must be aligned to their type", who);
  if ((rc = check_work(d_work, work_bytes, attn_work_bytes(*s, false), who))) return rc;
  if (s->B == 0 || ((!a.y.data || s->T == 0) && !d_state)) return SIM_OK;
  a.decay = d_decay; a.len = d_len; a.s0 = d_s0; a.state = d_state; a.work = d_work;
  const OpCtx o = op_ctx(x);
  a.err = o.err;
  return on_ctx(x, SIM_KC_GAE, who, [&] { return launch_attn(a, false, o.stream); });
}

int linear_attn_grad_work(const sim_linear_attn* s, size_t* bytes) {
  int rc = check_attn(s, "linear_attn_grad_work");
  if (rc) return rc;
  if (!bytes) return op_fail(SIM_EINVAL, "linear_attn_grad_work: bytes is NULL");
  *bytes = attn_work_bytes(*s, true);
  return SIM_OK;
}

int linear_attn_grad(sim_ctx* x, const sim_linear_attn* s, const sim_heads* q, const sim_heads* k,
                     const sim_heads* v, const float* d_decay, const sim_heads* dy, const int32_t* d_len,
                     const float* d_s0, const float* d_dstate, const sim_heads* dq, const sim_heads* dk,
                     const sim_heads* dv, float* d_ds0, void* d_work, size_t work_bytes) {
  const char* who = "linear_attn_grad";
  if (!x) return op_fail(SIM_EINVAL, "%s: ctx is NULL", who);
  int rc = check_attn(s, who);
  if (rc) return rc;
  AttnArgs a{};
  a.c = *s;
  if ((rc = check_heads(*s, dq, s->H, s->Dk, false, true, who, "dq", &a.dq))) return rc;
  if ((rc = check_heads(*s, dk, s->Hk, s->Dk, false, true, who, "dk", &a.dk))) return rc;
  if ((rc = check_heads(*s, dv, s->Hk, s->Dv, false, true, who, "dv", &a.dv))) return rc;
  const bool some = a.dq.data || a.dk.data || a.dv.data;
  if ((rc = check_heads(*s, q, s->H, s->Dk, a.dk.data || a.dv.data || d_ds0, false, who, "q", &a.q))) return rc;
  if ((rc = check_heads(*s, k, s->Hk, s->Dk, a.dq.data || a.dv.data, false, who, "k", &a.k))) return rc;
  if ((rc = check_heads(*s, v, s->Hk, s->Dv, a.dq.data || a.dk.data, false, who, "v", &a.v))) return rc;
  if ((rc = check_heads(*s, dy, s->H, s->Dv, true, false, who, "dy", &a.dy))) return rc;
  if (!d_decay && s->B) return op_fail(SIM_EINVAL, "%s: decay is NULL", who);
  if (!aligned(d_decay, 4) || !aligned(d_len, 4) || !aligned(d_s0, 4) || !aligned(d_dstate, 4) || !aligned(d_ds0, 4))
    return op_fail(SIM_EINVAL, "%s: decays, lengths and states must be aligned to their type", who);
  if ((rc = check_work(d_work, work_bytes, attn_work_bytes(*s, true), who))) return rc;
  if (s->B == 0 || ((!some || s->T == 0) && !d_ds0)) return SIM_OK;
  a.decay = d_decay; a.len = d_len; a.s0 = d_s0; a.ds = d_dstate; a.state = d_ds0; a.work = d_work;
  const OpCtx o = op_ctx(x);
  a.err = o.err;
  return on_ctx(x, SIM_KC_GAE, who, [&] { return launch_attn(a, true, o.stream); });
}

int token_logprobs_work(const sim_logprobs* c, size_t* bytes) {
  int rc = check_logprobs(c, "token_logprobs_work");
  if (rc) return rc;
  if (!bytes) return op_fail(SIM_EINVAL, "token_logprobs_work: bytes is NULL");
  *bytes = logprob_bytes(*c, false);
  return SIM_OK;
}

int token_logprobs(sim_ctx* x, const sim_logprobs* c, const sim_mat* logits, const sim_mat* mask,
                   const void* d_tokens, const uint8_t* d_live, float* d_logp, float* d_entropy,
                   int64_t* d_top_index, float* d_top_logp, void* d_work, size_t work_bytes) {
  const char* who = "token_logprobs";
  if (!x) return op_fail(SIM_EINVAL, "%s: ctx is NULL", who);
  int rc = check_logprobs(c, who);
  if (rc) return rc;
  LogprobArgs a{};
  a.c = *c;
  if ((rc = check_logits(c->N, c->A, c->dtype, logits, nullptr, who, &a.l, &a.grad))) return rc;
  if (mask && mask->data) {
    if ((rc = check_mat(c->N, c->A, mask, 1, false, false, who, "mask"))) return rc;
    a.mask = *mask;
  }
  if (c->N > 0 && d_logp && !d_tokens) return op_fail(SIM_EINVAL, "%s: logp needs tokens", who);
  if (!aligned(d_tokens, int_bytes(c->token_type)) || !aligned(d_logp, 4) || !aligned(d_entropy, 4) ||
      !aligned(d_top_index, 8) || !aligned(d_top_logp, 4))
    return op_fail(SIM_EINVAL, "%s: an array is not aligned to its type", who);
  if ((rc = check_work(d_work, work_bytes, logprob_bytes(*c, false), who))) return rc;
  a.tokens = d_tokens; a.live = d_live; a.logp = d_logp; a.entropy = d_entropy;
  if (c->top) { a.top_index = d_top_index; a.top_logp = d_top_logp; }
  if (c->N == 0 || (!a.logp && !a.entropy && !a.top_index && !a.top_logp)) return SIM_OK;
  a.work = d_work;
  const OpCtx o = op_ctx(x);
  a.err = o.err;
  return on_ctx(x, SIM_KC_PPO, who, [&] { return launch_logprobs(a, o.stream); });
}

int token_logprobs_grad_work(const sim_logprobs* c, size_t* bytes) {
  int rc = check_logprobs(c, "token_logprobs_grad_work");
  if (rc) return rc;
  if (!bytes) return op_fail(SIM_EINVAL, "token_logprobs_grad_work: bytes is NULL");
  *bytes = logprob_bytes(*c, true);
  return SIM_OK;
}

int token_logprobs_grad(sim_ctx* x, const sim_logprobs* c, const sim_mat* logits, const sim_mat* mask,
                        const void* d_tokens, const uint8_t* d_live, const float* d_dlogp,
                        const float* d_dentropy, const sim_mat* grad, void* d_work, size_t work_bytes) {
  const char* who = "token_logprobs_grad";
  if (!x) return op_fail(SIM_EINVAL, "%s: ctx is NULL", who);
  int rc = check_logprobs(c, who);
  if (rc) return rc;
  LogprobArgs a{};
  a.c = *c;
  if ((rc = check_logits(c->N, c->A, c->dtype, logits, grad, who, &a.l, &a.grad))) return rc;
  if (mask && mask->data) {
    if ((rc = check_mat(c->N, c->A, mask, 1, false, false, who, "mask"))) return rc;
    a.mask = *mask;
  }
  if (c->N > 0 && !a.grad.data) return op_fail(SIM_EINVAL, "%s: grad is NULL", who);
  if (c->N > 0 && d_dlogp && !d_tokens) return op_fail(SIM_EINVAL, "%s: dlogp needs tokens", who);
  if (!aligned(d_tokens, int_bytes(c->token_type)) || !aligned(d_dlogp, 4) || !aligned(d_dentropy, 4))
    return op_fail(SIM_EINVAL, "%s: an array is not aligned to its type", who);
  if ((rc = check_work(d_work, work_bytes, logprob_bytes(*c, true), who))) return rc;
  if (c->N == 0) return SIM_OK;
  a.tokens = d_tokens; a.live = d_live; a.dlogp = d_dlogp; a.dentropy = d_dentropy; a.work = d_work;
  const OpCtx o = op_ctx(x);
  a.err = o.err;
  return on_ctx(x, SIM_KC_PPO, who, [&] { return launch_logprobs(a, o.stream); });
}

int orthogonalize_work(const sim_ortho* c, size_t* bytes) {
  int rc = check_ortho(c, "orthogonalize_work");
  if (rc) return rc;
  if (!bytes) return op_fail(SIM_EINVAL, "orthogonalize_work: bytes is NULL");
  *bytes = ortho_bytes(*c);
  return SIM_OK;
}

int orthogonalize(sim_ctx* x, const sim_ortho* c, const sim_mats* update, const sim_mats* out, void* d_work,
                  size_t work_bytes) {
  const char* who = "orthogonalize";
  if (!x) return op_fail(SIM_EINVAL, "%s: ctx is NULL", who);
  int rc = check_ortho(c, who);
  if (rc) return rc;
  OrthoArgs a{};
  a.c = *c;
  if (c->n && c->M && c->N) {
    const sim_mats* both[2] = {update, out};
    for (int i = 0; i < 2; ++i) {
      const char* name = i ? "out" : "update";
      if (!both[i] || !both[i]->data) return op_fail(SIM_EINVAL, "%s: %s is NULL", who, name);
      const Dim dims[3] = {{both[i]->stride_i, c->n}, {both[i]->stride_r, c->M}, {both[i]->stride_c, c->N}};
      if ((rc = check_box(both[i]->data, dims, 1, elem_bytes(c->dtype), i, who, name))) return rc;
    }
    a.u = *update;
    a.out = *out;
  }
  if ((rc = check_work(d_work, work_bytes, ortho_bytes(*c), who))) return rc;
  if (!a.u.data) return SIM_OK;
  a.work = d_work;
  const OpCtx o = op_ctx(x);
  return on_ctx(x, SIM_KC_PPO, who, [&] { return launch_ortho(a, o.stream); });
}

}  // extern "C"
