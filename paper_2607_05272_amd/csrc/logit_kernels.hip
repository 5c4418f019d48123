// logit_kernels.hip -- losses over the logits of the caller's network, with their gradients: the
// clipped policy loss with a KL term, and a router's balance loss.
//
// Both need a row's softmax first (its maximum m and S = sum exp(l - m)) and then write a gradient
// per logit, so the logits are read, reduced and written out again: bound by HBM.
#include "ops_dev.hpp"

namespace bsim {
namespace {

constexpr int kRows = 4;            // rows per workgroup, one wave each
constexpr int kMaxBlocks = 2048;    // workgroups of a loss, each with its partial sums

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
template <class W>
__device__ __forceinline__ W wave_sum(W v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// A sample's loss terms and the derivative q of its loss with respect to logp (without weight).
struct Terms { float pol, kl, q; };
__device__ __forceinline__ Terms policy_terms(const sim_policy_loss& c, float logp, const float* old,
                                              const float* ref, double adv64, int64_t n) {
  const float adv = (float)adv64;
  Terms r{0.f, 0.f, 0.f};
  const float rho = old ? expf(logp - old[n]) : 1.0f;
  const float lo = 1.0f - c.clip, hi = 1.0f + c.clip;
  const float rc = fminf(fmaxf(rho, lo), hi);
  const float s1 = rho * adv, s2 = rc * adv;
  r.pol = s1 <= s2 ? -s1 : -s2;   // NaN if either is: rc alone may have lost it
  if (!(s1 == s1)) r.pol = s1;
  const bool slope = s1 <= s2 || (rho > lo && rho < hi) || !(s1 == s1);
  r.q = slope ? -s1 : 0.0f;
  if (ref) {
    const float d = ref[n] - logp, e = expm1f(d);
    r.kl = e - d;
    r.q -= c.c_kl * e;
  }
  return r;
}

template <class E>
__global__ __launch_bounds__(64 * kRows) void policy_row_k(PolicyLossArgs s) {
  typedef typename E::T T;
  __shared__ double part[kRows][3];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T* l = static_cast<const T*>(s.l.data);
  T* g = static_cast<T*>(s.grad.data);
  const uint8_t* mk = static_cast<const uint8_t*>(s.mask.data);
  double pol = 0.0, kl = 0.0, ent = 0.0;
  for (int64_t n = (int64_t)blockIdx.x * kRows + wave; n < s.c.N; n += (int64_t)gridDim.x * kRows) {
    const float w = s.w ? s.w[n] : 1.0f / (float)s.c.N;
    auto logit = [&](int64_t j) {
      if (mk && !mk[n * s.mask.stride_n + j * s.mask.stride_a]) return -INFINITY;
      return (float)l[n * s.l.stride_n + j * s.l.stride_a];
    };
    bool on = w != 0.0f;
    float m = -INFINITY, S = 0.f, X = 0.f, logp = 0.f, logS = 0.f, H = 0.f;
    Terms tm{0.f, 0.f, 0.f};
    int64_t act = -1;
    if (on) {
      bool some = false;
      for (int j = lane; j < s.c.A; j += 64) {
        const float v = logit(j);
        some = some || !(v == -INFINITY);
        m = fmaxf(m, v);
      }
      on = __ballot(some) != 0ull;
      m = wave_max(m);
    }
    if (on) {
      act = load_int(s.act, s.c.action_type, n);
      const bool ok = act >= 0 && act < s.c.A && !(logit(act) == -INFINITY);
      if (!ok) {
        if (lane == 0) atomicOr(s.err, ERR_ACTION);
        on = false;
      }
    }
    if (on) {
      for (int j = lane; j < s.c.A; j += 64) {
        const float v = logit(j);
        const float e = v == -INFINITY ? 0.0f : expf(v - m);
        S += e;
        if (e != 0.0f) X += e * (v - m);
      }
      S = wave_sum(S);
      X = wave_sum(X);
      logS = logf(S);
      logp = (logit(act) - m) - logS;
      H = logS - X / S;
      const double adv = s.c.adv_type == SIM_DT_F64 ? static_cast<const double*>(s.adv)[n]
                                                    : (double)static_cast<const float*>(s.adv)[n];
      tm = policy_terms(s.c, logp, s.logp_old, s.logp_ref, adv, n);
      pol += (double)w * tm.pol;
      kl += (double)w * tm.kl;
      ent += (double)w * H;
    }
    if (lane == 0 && s.logp) s.logp[n] = logp;
    if (!g) continue;
    for (int j = lane; j < s.c.A; j += 64) {
      float o = 0.0f;
      if (on) {
        const float v = logit(j);
        if (!(v == -INFINITY)) {
          const float lp = (v - m) - logS, p = expf(lp);
          o = tm.q * ((j == act ? 1.0f : 0.0f) - p);
          if (s.c.c_entropy > 0.0f && p > 0.0f) o += s.c.c_entropy * (p * (lp + H));
          o *= w;
        }
      }
      g[n * s.grad.stride_n + j * s.grad.stride_a] = (T)o;
    }
  }
  if (lane == 0) { part[wave][0] = pol; part[wave][1] = kl; part[wave][2] = ent; }
  __syncthreads();
  if (threadIdx.x < 3) {
    double v = 0.0;
    for (int i = 0; i < kRows; ++i) v += part[i][threadIdx.x];
    static_cast<double*>(s.work)[3 * blockIdx.x + threadIdx.x] = v;
  }
}

// the workgroups' sums, in a fixed order
__global__ __launch_bounds__(64) void policy_finish_k(PolicyLossArgs s, int nb) {
  const double* w = static_cast<const double*>(s.work);
  double v[3] = {0.0, 0.0, 0.0};
  for (int b = threadIdx.x; b < nb; b += 64)
    for (int i = 0; i < 3; ++i) v[i] += w[3 * b + i];
  for (int i = 0; i < 3; ++i) v[i] = wave_sum(v[i]);
  if (threadIdx.x == 0) {
    s.loss[0] = (float)(v[0] + (double)s.c.c_kl * v[1] - (double)s.c.c_entropy * v[2]);
    for (int i = 0; i < 3; ++i) s.loss[1 + i] = (float)v[i];
  }
}

int loss_blocks(int64_t N) {
  const int64_t b = (N + kRows - 1) / kRows;
  return (int)(b < 1 ? 1 : (b > kMaxBlocks ? kMaxBlocks : b));
}

// ---- balance loss ----------------------------------------------------------------------------
// work: per-workgroup sums [kMaxBlocks] fp64, then the live rows (one 64-bit integer)
__device__ __forceinline__ unsigned long long* live_count(const BalanceArgs& s) {
  return reinterpret_cast<unsigned long long*>(static_cast<double*>(s.work) + kMaxBlocks);
}

__global__ __launch_bounds__(256) void balance_zero_k(BalanceArgs s, int G) {
  for (int i = threadIdx.x; i < G; i += 256) s.counts[i] = 0;
  if (threadIdx.x == 0) *live_count(s) = 0ull;
}

__global__ __launch_bounds__(256) void balance_count_k(BalanceArgs s) {
  for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < s.c.N; n += (int64_t)gridDim.x * 256) {
    if (s.live && !s.live[n]) continue;
    atomicAdd(live_count(s), 1ull);
    for (int i = 0; i < s.c.k; ++i) {
      const int64_t a = load_int(s.idx, s.c.index_type, n * s.c.k + i);
      if (a >= 0 && a < s.c.A)
        atomicAdd(reinterpret_cast<unsigned long long*>(s.counts) + a / s.c.group, 1ull);
      else if (a != -1)
        atomicOr(s.err, ERR_ACTION);
    }
  }
}

template <class E>
__global__ __launch_bounds__(64 * kRows) void balance_row_k(BalanceArgs s) {
  typedef typename E::T T;
  __shared__ double part[kRows];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T* l = static_cast<const T*>(s.l.data);
  T* g = static_cast<T*>(s.grad.data);
  const double W = (double)*live_count(s);
  const float scale = W > 0.0 ? (float)((double)s.c.coef * (s.c.A / s.c.group) / W) : 0.0f;
  const float fk = W > 0.0 ? (float)(1.0 / (W * s.c.k)) : 0.0f;
  double acc = 0.0;
  for (int64_t n = (int64_t)blockIdx.x * kRows + wave; n < s.c.N; n += (int64_t)gridDim.x * kRows) {
    bool on = !s.live || s.live[n];
    float m = -INFINITY, S = 0.f, X = 0.f;
    if (on) {
      bool some = false;
      for (int j = lane; j < s.c.A; j += 64) {
        const float v = (float)l[n * s.l.stride_n + j * s.l.stride_a];
        some = some || !(v == -INFINITY);
        m = fmaxf(m, v);
      }
      on = __ballot(some) != 0ull;
      m = wave_max(m);
    }
    if (on) {
      for (int j = lane; j < s.c.A; j += 64) {
        const float v = (float)l[n * s.l.stride_n + j * s.l.stride_a];
        const float e = v == -INFINITY ? 0.0f : expf(v - m);
        S += e;
        X += e * (fk * (float)s.counts[j / s.c.group]);
      }
      S = wave_sum(S);
      X = wave_sum(X) / S;
      acc += (double)X;
    }
    if (!g) continue;
    for (int j = lane; j < s.c.A; j += 64) {
      float o = 0.0f;
      if (on) {
        const float v = (float)l[n * s.l.stride_n + j * s.l.stride_a];
        const float p = v == -INFINITY ? 0.0f : expf(v - m) / S;
        o = scale * p * (fk * (float)s.counts[j / s.c.group] - X);
      }
      g[n * s.grad.stride_n + j * s.grad.stride_a] = (T)o;
    }
  }
  if (lane == 0) part[wave] = acc;
  __syncthreads();
  if (threadIdx.x == 0) {
    double v = 0.0;
    for (int i = 0; i < kRows; ++i) v += part[i];
    static_cast<double*>(s.work)[blockIdx.x] = v;
  }
}

__global__ __launch_bounds__(64) void balance_finish_k(BalanceArgs s, int nb) {
  const double* w = static_cast<const double*>(s.work);
  double v = 0.0;
  for (int b = threadIdx.x; b < nb; b += 64) v += w[b];
  v = wave_sum(v);
  const double W = (double)*live_count(s);
  if (threadIdx.x == 0)
    s.loss[0] = W > 0.0 ? (float)(v * ((double)s.c.coef * (s.c.A / s.c.group) / W)) : 0.0f;
}

}  // namespace

size_t policy_loss_bytes(const sim_policy_loss&) { return (size_t)kMaxBlocks * 3 * sizeof(double); }

hipError_t launch_policy_loss(const PolicyLossArgs& a, hipStream_t st) {
  const int nb = loss_blocks(a.c.N);
  const dim3 grid(nb), block(64 * kRows);
  switch (a.c.dtype) {
    case SIM_DT_F32: hipLaunchKernelGGL(policy_row_k<F32>, grid, block, 0, st, a); break;
    case SIM_DT_BF16: hipLaunchKernelGGL(policy_row_k<BF16>, grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL(policy_row_k<F16>, grid, block, 0, st, a); break;
  }
  hipLaunchKernelGGL(policy_finish_k, dim3(1), dim3(64), 0, st, a, nb);
  return hipGetLastError();
}

size_t balance_bytes(const sim_balance&) { return (size_t)kMaxBlocks * sizeof(double) + 16; }

hipError_t launch_balance(const BalanceArgs& a, hipStream_t st) {
  const int nb = loss_blocks(a.c.N), G = a.c.A / a.c.group;
  const dim3 grid(nb), block(64 * kRows);
  hipLaunchKernelGGL(balance_zero_k, dim3(1), dim3(256), 0, st, a, G);
  if (a.c.N > 0)
    hipLaunchKernelGGL(balance_count_k, dim3((unsigned)((a.c.N + 255) / 256 > 1024 ? 1024 : (a.c.N + 255) / 256)),
                       dim3(256), 0, st, a);
  switch (a.c.dtype) {
    case SIM_DT_F32: hipLaunchKernelGGL(balance_row_k<F32>, grid, block, 0, st, a); break;
    case SIM_DT_BF16: hipLaunchKernelGGL(balance_row_k<BF16>, grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL(balance_row_k<F16>, grid, block, 0, st, a); break;
  }
  hipLaunchKernelGGL(balance_finish_k, dim3(1), dim3(64), 0, st, a, nb);
  return hipGetLastError();
}

}  // namespace bsim
