// logprob_kernels.hip -- log-probabilities of given tokens over the logits of the caller's network, the
// entropy, the likeliest columns, and the gradient of the first two (rows, sums and forms: logit_dev.hpp).
//
// With x = l - m and S = sum e^x as there: log p_j = x_j - log S, H = log S - sum(e x) / S, and of
// g log p_a + h H
//   dl_j = p_j (-g - h (H - log S) - h x_j) + g [j = a].
#include "logit_dev.hpp"

namespace bsim {
namespace {

struct LogprobOp {
  static constexpr bool kBal = false, kSums = false;
  static constexpr int kTargets = 1;
  typedef LogprobArgs Args;
  struct Row { float g, h; int64_t act; };

  __device__ static __forceinline__ bool open(const Args& s, int64_t n, Row& r) {
    r.act = s.tokens ? load_int(s.tokens, s.c.token_type, n) : -1;
    r.g = s.dlogp ? s.dlogp[n] : 0.0f;
    r.h = s.dentropy ? s.dentropy[n] : 0.0f;
    return !s.live || s.live[n];
  }
  // the given token's logit, -inf if there is none or it is forbidden
  template <class T>
  __device__ static __forceinline__ float taken(const Args& s, int64_t n, const Row& r) {
    if (r.act < 0 || r.act >= s.c.A) return -INFINITY;
    const uint8_t* mk = static_cast<const uint8_t*>(s.mask.data);
    if (mk && !mk[n * s.mask.stride_n + r.act * s.mask.stride_a]) return -INFINITY;
    return (float)static_cast<const T*>(s.l.data)[n * s.l.stride_n + r.act * s.l.stride_a];
  }
  __device__ static __forceinline__ bool close(const Args& s, int64_t n, const Row& r, const Part& p, float la,
                                               bool first, Sums&, RowOut& o) {
    const bool none = r.act < 0 || r.act >= s.c.A;
    if (first && none && r.act != -1) atomicOr(s.err, ERR_ACTION);
    if (p.m == -INFINITY) return false;          // no allowed column
    const float logS = log_of(p.S), rS = __builtin_amdgcn_rcpf(p.S);
    const float H = fmaf(-p.X, rS, logS);
    if (first) {
      if (s.logp) s.logp[n] = none ? 0.0f : (la == -INFINITY ? la : (la - p.m) - logS);
      if (s.entropy) s.entropy[n] = H;
    }
    const float g = la == -INFINITY ? 0.0f : r.g;   // none or forbidden
    o.alpha = -rS * fmaf(r.h, H - logS, g);
    o.beta = -rS * r.h;
    o.delta = g;
    return true;
  }
  __device__ static __forceinline__ void shut(const Args& s, int64_t n) {
    if (s.logp) s.logp[n] = 0.0f;
    if (s.entropy) s.entropy[n] = 0.0f;
  }
  __device__ static __forceinline__ void fill(const Args&, int, float*) {}
  __device__ static __forceinline__ float target(const Args&, const float*, int) { return 0.0f; }
  __device__ static __forceinline__ void finish(const Args&, const Sums&) {}
};

// The order of alternatives as whole numbers: the logit's (a NaN above all, -0 as 0), then the lowest
// column first. 0: not an alternative.
__device__ __forceinline__ uint64_t key_of(float v, uint32_t j) {
  if (v == -INFINITY) return 0;
  const uint32_t u = __float_as_uint(v + 0.0f);
  const uint32_t o = v == v ? ((int32_t)u < 0 ? ~u : u | 0x80000000u) : 0xFFFFFFFFu;
  return (uint64_t)o << 32 | (uint32_t)~j;
}

// One workgroup per row, one look over the row per alternative.
constexpr int kTop = 256;
template <class E>
__global__ __launch_bounds__(kTop) void logprob_top_k(LogprobArgs s) {
  typedef typename E::T T;
  __shared__ Part parts[kTop / 64];
  __shared__ uint64_t best[kTop / 64];
  const int A = s.c.A, top = s.c.top;
  for (int64_t n = blockIdx.x; n < s.c.N; n += gridDim.x) {
    const bool on = !s.live || s.live[n];
    const T* l = static_cast<const T*>(s.l.data) + n * s.l.stride_n;
    const uint8_t* mk = s.mask.data ? static_cast<const uint8_t*>(s.mask.data) + n * s.mask.stride_n : nullptr;
    auto logit = [&](int j) {
      return mk && !mk[j * s.mask.stride_a] ? -INFINITY : (float)l[j * s.l.stride_a];
    };
    Part p{-INFINITY, 0.0f, 0.0f};
    if (on) {
      for (int j = threadIdx.x; j < A; j += kTop) {
        const float v = logit(j), M = max_nan(p.m, v);
        if (M == -INFINITY) continue;
        p = against<false>(p, M);
        p.S += exp_of(max_nan(v - M, kLowest));
      }
      __syncthreads();
      p = join_threads<false, kTop / 64>(p, parts);
    }
    uint64_t last = ~0ull;
    for (int i = 0; i < top; ++i) {
      uint64_t k = 0;
      if (on && last) {
        for (int j = threadIdx.x; j < A; j += kTop) {
          const uint64_t c = key_of(logit(j), j);
          if (c < last && c > k) k = c;
        }
      }
      for (int o = 1; o < 64; o <<= 1) {
        const uint64_t c = __shfl_xor(k, o);
        if (c > k) k = c;
      }
      __syncthreads();
      if ((threadIdx.x & 63) == 0) best[threadIdx.x >> 6] = k;
      __syncthreads();
      for (int w = 0; w < kTop / 64; ++w)
        if (best[w] > k) k = best[w];
      last = k;
      if (threadIdx.x == 0) {
        const int j = k ? (int)~(uint32_t)k : -1;
        if (s.top_index) s.top_index[n * top + i] = j;
        if (s.top_logp) s.top_logp[n * top + i] = k ? (logit(j) - p.m) - log_of(p.S) : -INFINITY;
      }
    }
  }
}

}  // namespace

size_t logprob_bytes(const sim_logprobs&, bool) {
  return (size_t)kMaxBlocks * 3 * sizeof(double) + kSplitMost * (sizeof(Part) + sizeof(float));
}

hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t st) {
  if (a.logp || a.entropy || a.grad.data) {
    const hipError_t e = launch_loss<LogprobOp>(a, 0, st);
    if (e != hipSuccess) return e;
  }
  if (a.top_index || a.top_logp) {
    const dim3 grid(blocks_for(a.c.N, 1, 1 << 20)), block(kTop);
    if (a.c.dtype == SIM_DT_F32) hipLaunchKernelGGL(logprob_top_k<F32>, grid, block, 0, st, a);
    else if (a.c.dtype == SIM_DT_BF16) hipLaunchKernelGGL(logprob_top_k<BF16>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(logprob_top_k<F16>, grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace bsim
