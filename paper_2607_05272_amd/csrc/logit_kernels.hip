// logit_kernels.hip -- losses over the logits of the caller's network, with their gradients: the
// clipped policy loss with a KL term, and a router's balance loss (rows, sums and forms: logit_dev.hpp).
#include "logit_dev.hpp"

namespace bsim {
namespace {
// e^d - 1 and, in `rest`, e^d - 1 - d: both lose all their digits to the subtractions where d is small, so
// the second is summed as a series up to |d| = 0.35 (its first term left out is d^9/9!, 2e-9 of d^2/2).
__device__ __forceinline__ float grow(float d, float& rest) {
  float t = fmaf(d, 1.0f / 40320.0f, 1.0f / 5040.0f);
  t = fmaf(d, t, 1.0f / 720.0f);
  t = fmaf(d, t, 1.0f / 120.0f);
  t = fmaf(d, t, 1.0f / 24.0f);
  t = fmaf(d, t, 1.0f / 6.0f);
  t = fmaf(d, t, 0.5f) * (d * d);
  const float e = exp_of(d) - 1.0f;
  const bool small = fabsf(d) < 0.35f;
  rest = small ? t : e - d;
  return small ? d + t : e;
}

// ---- the two losses ----------------------------------------------------------------------------
struct PolicyOp {
  static constexpr bool kBal = false, kSums = true, kClosed = false;
  static constexpr int kTargets = 1;
  typedef PolicyLossArgs Args;
  struct Row { float w, adv, old, ref; int64_t act; };

  // what the row has besides its logits; false: it is not looked at
  __device__ static __forceinline__ bool open(const Args& s, int64_t n, Row& r) {
    r.w = s.w ? s.w[n] : 1.0f / (float)s.c.N;
    r.act = load_int(s.act, s.c.action_type, n);
    r.adv = s.c.adv_type == SIM_DT_F64 ? (float)static_cast<const double*>(s.adv)[n]
                                       : static_cast<const float*>(s.adv)[n];
    r.old = s.logp_old ? s.logp_old[n] : 0.0f;
    r.ref = s.logp_ref ? s.logp_ref[n] : 0.0f;
    return r.w != 0.0f;
  }
  // the taken action's logit, -inf if it is out of range or forbidden
  template <class T>
  __device__ static __forceinline__ float taken(const Args& s, int64_t n, const Row& r) {
    if (r.act < 0 || r.act >= s.c.A) return -INFINITY;
    const uint8_t* mk = static_cast<const uint8_t*>(s.mask.data);
    if (mk && !mk[n * s.mask.stride_n + r.act * s.mask.stride_a]) return -INFINITY;
    return (float)static_cast<const T*>(s.l.data)[n * s.l.stride_n + r.act * s.l.stride_a];
  }
  // the row's terms and gradient; false: it gives nothing. `first`: this thread keeps its sums
  __device__ static __forceinline__ bool close(const Args& s, int64_t n, const Row& r, const Part& p, float la,
                                               bool first, Sums& sums, RowOut& o) {
    if (p.m == -INFINITY) return false;          // no allowed action
    if (la == -INFINITY) {
      if (first) atomicOr(s.err, ERR_ACTION);
      return false;
    }
    const float logS = log_of(p.S), logp = (la - p.m) - logS, rS = __builtin_amdgcn_rcpf(p.S);
    const float H = fmaf(-p.X, rS, logS);
    const float rho = s.logp_old ? exp_of(logp - r.old) : 1.0f;
    const float lo = 1.0f - s.c.clip, hi = 1.0f + s.c.clip;
    const float s1 = rho * r.adv, s2 = fminf(fmaxf(rho, lo), hi) * r.adv;
    const bool nan = !(s1 == s1);                // the clipped one alone may have lost it
    const float pol = s1 <= s2 || nan ? -s1 : -s2;
    float q = s1 <= s2 || nan || (rho > lo && rho < hi) ? -s1 : 0.0f, kl = 0.0f;
    if (s.logp_ref) {
      const float slope = grow(r.ref - logp, kl);
      if (s.c.c_kl > 0.0f) q -= s.c.c_kl * slope;   // 0 times an infinite slope is not 0
    }
    const float wr = r.w * rS, ch = s.c.c_entropy;
    o.alpha = ch > 0.0f ? wr * fmaf(ch, H - logS, -q) : -wr * q;
    o.beta = wr * ch;
    o.delta = r.w * q;
    if (first) {
      sums.a += (double)r.w * pol;
      sums.b += (double)r.w * kl;
      sums.c += (double)r.w * H;
      if (s.logp) s.logp[n] = logp;
    }
    return true;
  }
  __device__ static __forceinline__ void shut(const Args& s, int64_t n) {   // a row that gives nothing
    if (s.logp) s.logp[n] = 0.0f;
  }
  __device__ static __forceinline__ void fill(const Args&, int, float*) {}
  __device__ static __forceinline__ float target(const Args&, const float*, int) { return 0.0f; }
  __device__ static __forceinline__ void finish(const Args& s, const Sums& v) {
    // a term without a coefficient is told apart, but is no part of the loss, infinite or not
    s.loss[0] = (float)(v.a + (s.c.c_kl > 0.0f ? (double)s.c.c_kl * v.b : 0.0) -
                        (s.c.c_entropy > 0.0f ? (double)s.c.c_entropy * v.c : 0.0));
    s.loss[1] = (float)v.a;
    s.loss[2] = (float)v.b;
    s.loss[3] = (float)v.c;
  }
};

// f of a target: coef G / W times its share of the live rows' choices, so that a row's term of the
// loss is s and its gradient p (f - s). Every workgroup holds it in LDS.
constexpr int kMaxTargets = 4096;
// Choices are counted by workgroups that each write a row of counts, which a second launch adds up; few
// enough of them are counted by every workgroup of the rows itself.
constexpr int kCountBlocks = 256, kCountThreads = 512, kCountAhead = 4, kCountSelf = 4096;
// the work memory: sums [kMaxBlocks][3] fp64, f [G], live rows [kCountBlocks], counts [kCountBlocks][G]
__device__ __forceinline__ float* targets(const BalanceArgs& s) {
  return reinterpret_cast<float*>(static_cast<double*>(s.work) + 3 * kMaxBlocks);
}
__device__ __forceinline__ uint32_t* live_parts(const BalanceArgs& s) {
  return reinterpret_cast<uint32_t*>(targets(s) + s.c.A / s.c.group);
}
int count_blocks(int64_t N, int k) {
  if (N * k <= kCountSelf) return 0;
  constexpr int each = kCountThreads * kCountAhead;
  return (int)std::min<int64_t>(kCountBlocks, (N * k + each - 1) / each);
}
// A target's factor f_g coef G / W, less that of an even share, coef / W: only differences of the factors
// matter to the gradient, and near balance (or with one target) those of the factors themselves would be
// rounding. The loss gets the even share back at its end.
__device__ __forceinline__ float target_of(const BalanceArgs& s, uint32_t W, uint32_t count) {
  if (W == 0) return 0.0f;
  const double G = s.c.A / s.c.group, all = (double)W * s.c.k;
  return (float)((double)s.c.coef / W * ((double)count * G - all) / all);
}

__device__ void fill_targets(const BalanceArgs& s, int nb, float* f);
__device__ float target(const BalanceArgs& s, const float* f, int j);

struct BalanceOp {
  static constexpr bool kBal = true, kSums = true, kClosed = false;
  static constexpr int kTargets = kMaxTargets;
  typedef BalanceArgs Args;
  struct Row { int64_t act; };
  __device__ static __forceinline__ bool open(const Args& s, int64_t n, Row& r) {
    r.act = -1;
    return !s.live || s.live[n];
  }
  template <class T>
  __device__ static __forceinline__ float taken(const Args&, int64_t, const Row&) { return 0.0f; }
  __device__ static __forceinline__ bool close(const Args&, int64_t, const Row&, const Part& p, float, bool first,
                                               Sums& sums, RowOut& o) {
    if (first) sums.c += 1.0;   // live rows, and those that have a probability
    if (p.m == -INFINITY) return false;
    const float rS = __builtin_amdgcn_rcpf(p.S), si = p.X * rS;
    o.beta = rS;
    o.alpha = -si * rS;
    o.delta = 0.0f;
    if (first) {
      sums.a += (double)si;
      sums.b += 1.0;
    }
    return true;
  }
  __device__ static __forceinline__ void shut(const Args&, int64_t) {}
  __device__ static __forceinline__ void fill(const Args& s, int nb, float* f) { fill_targets(s, nb, f); }
  __device__ static __forceinline__ float target(const Args& s, const float* f, int j) { return bsim::target(s, f, j); }
  __device__ static __forceinline__ void finish(const Args& s, const Sums& v) {
    s.loss[0] = v.c > 0.0 ? (float)(v.a + (double)s.c.coef * v.b / v.c) : 0.0f;
  }
};

// Adds choices first, first + step, ... of the live rows to hist (cleared by the caller) and the live rows
// to *live; the loads of several choices fly together.
__device__ __forceinline__ void count_choices(const BalanceArgs& s, uint32_t first, uint32_t step, uint32_t* hist,
                                              uint32_t* live, bool tell) {
  const uint32_t k = (uint32_t)s.c.k, total = (uint32_t)(s.c.N * s.c.k);   // below 2^31
  uint32_t mine = 0;
  for (uint32_t i0 = first; i0 < total; i0 += kCountAhead * step) {
    int64_t a[kCountAhead];
    bool on[kCountAhead];
#pragma unroll
    for (int u = 0; u < kCountAhead; ++u) {
      const uint32_t i = i0 + u * step;
      on[u] = i < total;
      a[u] = on[u] ? load_int(s.idx, s.c.index_type, i) : -1;
      const uint32_t n = k == 1 ? i : i / k;
      if (on[u] && s.live) on[u] = s.live[n];
      if (on[u] && n * k == i) ++mine;
    }
#pragma unroll
    for (int u = 0; u < kCountAhead; ++u) {
      if (!on[u] || a[u] == -1) continue;
      if (a[u] >= 0 && a[u] < s.c.A)
        atomicAdd(&hist[s.c.group == 1 ? (uint32_t)a[u] : (uint32_t)a[u] / (uint32_t)s.c.group], 1u);
      else if (tell) atomicOr(s.err, ERR_ACTION);
    }
  }
  if (mine) atomicAdd(live, mine);
}

// The groups' choices, in LDS of up to 256 workgroups; their counts are added up by balance_targets_k, or
// where they are few by each workgroup of the next launch. Bound by latency: a chain of index, atomic and
// barrier (65536 choices 7.3 us, 1048576 of 8 bytes 7.1 us).
__global__ __launch_bounds__(kCountThreads) void balance_count_k(BalanceArgs s) {
  __shared__ uint32_t hist[kMaxTargets];
  __shared__ uint32_t live;
  const int G = s.c.A / s.c.group;
  for (int g = threadIdx.x; g < G; g += kCountThreads) hist[g] = 0;
  if (threadIdx.x == 0) live = 0;
  __syncthreads();
  count_choices(s, blockIdx.x * kCountThreads + threadIdx.x, gridDim.x * kCountThreads, hist, &live, true);
  __syncthreads();
  uint32_t* o = live_parts(s);
  if (threadIdx.x == 0) o[blockIdx.x] = live;
  for (int g = threadIdx.x; g < G; g += kCountThreads) o[kCountBlocks + blockIdx.x * G + g] = hist[g];
}

// 32 targets a workgroup, 8 threads each (128 targets of 256 workgroups 4.7 us)
__global__ __launch_bounds__(256) void balance_targets_k(BalanceArgs s, int nb) {
  __shared__ uint32_t part[8][32], live[4];
  const int G = s.c.A / s.c.group, g = blockIdx.x * 32 + (threadIdx.x & 31), sl = threadIdx.x >> 5;
  const uint32_t* lp = live_parts(s);
  const uint32_t* cnt = lp + kCountBlocks;
  uint32_t w = threadIdx.x < nb ? lp[threadIdx.x] : 0, c = 0;
  if (g < G) {
#pragma unroll 8
    for (int b = sl; b < nb; b += 8) c += cnt[b * G + g];
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) w += __shfl_xor(w, o);
  if ((threadIdx.x & 63) == 0) live[threadIdx.x >> 6] = w;
  part[sl][threadIdx.x & 31] = c;
  __syncthreads();
  if (sl == 0 && g < G) {
    c = 0;
    for (int i = 0; i < 8; ++i) c += part[i][threadIdx.x];
    s.counts[g] = c;
    targets(s)[g] = target_of(s, live[0] + live[1] + live[2] + live[3], c);
  }
}
static_assert(kCountBlocks <= 256, "a thread per counting workgroup");

// Fills f [G] in LDS: from the launch that added up nb workgroups' counts, by adding them up here where
// there are few, or (nb = 0) by counting.
__host__ __device__ bool few_counts(int nb, int G) { return nb * G <= 4096; }
__device__ __forceinline__ void fill_targets(const BalanceArgs& s, int nb, float* f) {
  const int G = s.c.A / s.c.group;
  if (nb && !few_counts(nb, G)) {
    for (int g = threadIdx.x; g < G; g += blockDim.x) f[g] = targets(s)[g];
  } else {
    __shared__ uint32_t live;
    uint32_t* hist = reinterpret_cast<uint32_t*>(f);
    for (int g = threadIdx.x; g < G; g += blockDim.x) hist[g] = 0;
    if (threadIdx.x == 0) live = 0;
    __syncthreads();
    if (nb) {
      const uint32_t* lp = live_parts(s);
      const uint32_t* cnt = lp + kCountBlocks;
      for (int b = threadIdx.x; b < nb; b += blockDim.x) atomicAdd(&live, lp[b]);
#pragma unroll 4
      for (int i = threadIdx.x; i < nb * G; i += blockDim.x) atomicAdd(&hist[i % G], cnt[i]);
    } else {
      count_choices(s, threadIdx.x, blockDim.x, hist, &live, blockIdx.x == 0);
    }
    __syncthreads();
    for (int g = threadIdx.x; g < G; g += blockDim.x) {
      const uint32_t c = hist[g];
      if (blockIdx.x == 0) s.counts[g] = c;
      f[g] = target_of(s, live, c);
    }
  }
  __syncthreads();
}
__device__ __forceinline__ float target(const BalanceArgs& s, const float* f, int j) {
  return f[s.c.group == 1 ? (uint32_t)j : (uint32_t)j / (uint32_t)s.c.group];
}


}  // namespace

size_t policy_loss_bytes(const sim_policy_loss&) {
  return (size_t)kMaxBlocks * 3 * sizeof(double) + kSplitMost * (sizeof(Part) + sizeof(float));
}

hipError_t launch_policy_loss(const PolicyLossArgs& a, hipStream_t st) { return launch_loss<PolicyOp>(a, 0, st); }

size_t balance_bytes(const sim_balance& c) {
  const size_t G = c.A / c.group;
  return (size_t)kMaxBlocks * 3 * sizeof(double) + (G + kCountBlocks * (1 + G)) * sizeof(uint32_t);
}

hipError_t launch_balance(const BalanceArgs& a, hipStream_t st) {
  const int nb = count_blocks(a.c.N, a.c.k);
  if (nb) {
    hipLaunchKernelGGL(balance_count_k, dim3(nb), dim3(kCountThreads), 0, st, a);
    const int G = a.c.A / a.c.group;
    if (!few_counts(nb, G)) hipLaunchKernelGGL(balance_targets_k, dim3((G + 31) / 32), dim3(256), 0, st, a, nb);
  }
  return launch_loss<BalanceOp>(a, nb, st);
}

}  // namespace bsim
