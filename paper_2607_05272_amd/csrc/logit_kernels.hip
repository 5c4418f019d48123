// logit_kernels.hip -- losses over the logits of the caller's network, with their gradients: the
// clipped policy loss with a KL term, and a router's balance loss.
//
// With x = l - m of a row's maximum m, e = exp(x) and S = sum e, both gradients are p = e / S times an
// affine function of something known per element, and their terms follow from S and one more sum:
//   policy   H = log S - sum(e x) / S,   dl_j = p_j (alpha + beta x_j) + delta [j = action]
//   balance  s = sum(e f) / S,           dl_j = p_j (f_j - s)
// So a row is read, reduced once and written: bound by HBM as long as it stays in registers in
// between. An x below -1000 is taken as -1000: its e is 0 either way, and 0 times a finite number
// is 0, so -inf logits and masked ones need no case of their own. Maxima keep NaN.
#include <algorithm>

#include "ops_dev.hpp"

namespace bsim {
namespace {

constexpr int kMaxBlocks = 4096;    // workgroups of a loss, each with its partial sums
constexpr float kLowest = -1000.0f;

__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

__device__ __forceinline__ float log_of(float x) { return __builtin_amdgcn_logf(x) * 0.69314718055994531f; }
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

// A part of a row: its maximum m, S = sum e and X = sum e x (policy) or sum e f (balance), with x and e
// against m. A part of nothing has m = -inf, S = X = 0.
struct Part { float m, S, X; };
// the same against the maximum m of a larger part
template <bool BAL>
__device__ __forceinline__ Part against(const Part& a, float m) {
  const float d = m == -INFINITY ? 0.0f : max_nan(a.m - m, kLowest), f = exp_of(d);
  return Part{m, f * a.S, BAL ? f * a.X : f * fmaf(d, a.S, a.X)};
}
// Over a wave, in every lane, by DPP moves within the vector unit (a step of a few cycles, where one
// through LDS takes over a hundred): sums along each row of 16 lanes, then from row to row.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp(float none, float v) {
  return __uint_as_float(
      __builtin_amdgcn_update_dpp(__float_as_uint(none), __float_as_uint(v), CTRL, ROWS, 0xf, false));
}
template <class F>
__device__ __forceinline__ float wave_reduce(float v, F f, bool keep) {
  // lanes without a source take their own value (keep: maxima) or 0 (sums)
  v = f(v, dpp<0x111, 0xf>(keep ? v : 0.0f, v));   // row_shr 1, 2, 4, 8
  v = f(v, dpp<0x112, 0xf>(keep ? v : 0.0f, v));
  v = f(v, dpp<0x114, 0xf>(keep ? v : 0.0f, v));
  v = f(v, dpp<0x118, 0xf>(keep ? v : 0.0f, v));
  v = f(v, dpp<0x142, 0xa>(keep ? v : 0.0f, v));   // row_bcast 15 into rows 1 and 3
  v = f(v, dpp<0x143, 0xc>(keep ? v : 0.0f, v));   // row_bcast 31 into rows 2 and 3
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_reduce(v, [](float a, float b) { return max_nan(a, b); }, true);
}
__device__ __forceinline__ float wave_add(float v) {
  return wave_reduce(v, [](float a, float b) { return a + b; }, false);
}

// over 1 << lg adjacent lanes, in every lane
__device__ __forceinline__ float max_lanes(float m, int lg) {
  for (int o = 1; o < (1 << lg); o <<= 1) m = max_nan(m, __shfl_xor(m, o));
  return m;
}
__device__ __forceinline__ void add_lanes(float& S, float& X, int lg) {
  for (int o = 1; o < (1 << lg); o <<= 1) {
    S += __shfl_xor(S, o);
    X += __shfl_xor(X, o);
  }
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp(double v) {   // 0 where there is no source
  const uint64_t u = __double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0u, (uint32_t)u, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0u, (uint32_t)(u >> 32), CTRL, ROWS, 0xf, false);
  return __longlong_as_double((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double v) {   // in lane 63
  v += dpp<0x111, 0xf>(v);
  v += dpp<0x112, 0xf>(v);
  v += dpp<0x114, 0xf>(v);
  v += dpp<0x118, 0xf>(v);
  v += dpp<0x142, 0xa>(v);
  v += dpp<0x143, 0xc>(v);
  return v;
}

struct RowOut { float alpha, beta, delta; };
struct Sums { double a, b, c; };   // a thread's sums over its rows

// ---- the two losses ----------------------------------------------------------------------------
struct PolicyOp {
  static constexpr bool kBal = false;
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

struct BalanceOp {
  static constexpr bool kBal = true;
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
__device__ __forceinline__ void fill_targets(const PolicyLossArgs&, int, float*) {}
__device__ __forceinline__ float target(const BalanceArgs& s, const float* f, int j) {
  return f[s.c.group == 1 ? (uint32_t)j : (uint32_t)j / (uint32_t)s.c.group];
}
__device__ __forceinline__ float target(const PolicyLossArgs&, const float*, int) { return 0.0f; }

// A workgroup's sums, in a fixed order: to the work memory, or with one workgroup the loss itself.
// lds: [waves][3]
template <class OP>
__device__ __forceinline__ void leave(const typename OP::Args& s, Sums v, double (*lds)[3]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
  v.a = wave_sum(v.a);
  v.b = wave_sum(v.b);
  v.c = wave_sum(v.c);
  if (lane == 63) { lds[wave][0] = v.a; lds[wave][1] = v.b; lds[wave][2] = v.c; }
  __syncthreads();
  if (wave == 0) {
    Sums t{0.0, 0.0, 0.0};
    if (lane < nw) t = Sums{lds[lane][0], lds[lane][1], lds[lane][2]};
    t.a = wave_sum(t.a);
    t.b = wave_sum(t.b);
    t.c = wave_sum(t.c);
    if (lane == 63) {
      if (gridDim.x * gridDim.y == 1) {
        OP::finish(s, t);
      } else {
        double* o = static_cast<double*>(s.work) + 3 * (blockIdx.x * gridDim.y + blockIdx.y);
        o[0] = t.a; o[1] = t.b; o[2] = t.c;
      }
    }
  }
}
// The workgroups' sums, in a fixed order: one launch more (4.5 us) for a result that is the same each time.
constexpr int kFinish = 1024;
template <class OP>
__global__ __launch_bounds__(kFinish) void loss_finish_k(typename OP::Args s, int nb) {
  __shared__ double lds[kFinish / 64][3];
  const double* w = static_cast<const double*>(s.work);
  Sums v{0.0, 0.0, 0.0};
#pragma unroll 4
  for (int b = threadIdx.x; b < nb; b += kFinish) {
    v.a += w[3 * b];
    v.b += w[3 * b + 1];
    v.c += w[3 * b + 2];
  }
  leave<OP>(s, v, lds);
}

// ---- rows of adjacent logits -----------------------------------------------------------------
// N elements of a row, at any alignment of the element type
template <class E, int N>
struct Chunk {
  typedef typename E::T T;
  typedef T Raw __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  typedef T Val __attribute__((ext_vector_type(N)));
  typedef float Wide __attribute__((ext_vector_type(N)));
  Val v;
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (N == 1) v[0] = p[0];
    else v = __builtin_bit_cast(Val, *reinterpret_cast<const Raw*>(p));
  }
  __device__ __forceinline__ float get(int i) const { return (float)v[i]; }
  // Keeps the compiler from holding the widened elements of one pass for the next one: they would
  // take twice the registers (and spill) where the chunks just fit.
  __device__ __forceinline__ void forget() {
    if constexpr (N * sizeof(T) == 16) hide(v);
  }
  __device__ __forceinline__ static void store(T* p, const Wide& w) {
    if constexpr (N == 1) p[0] = (T)w[0];
    else *reinterpret_cast<Raw*>(p) = __builtin_bit_cast(Raw, __builtin_convertvector(w, Val));
  }
};
// their mask bytes, at any stride
template <int N>
struct MaskBytes {
  uint32_t w[(N + 3) / 4];
  __device__ __forceinline__ void load(const uint8_t* p, int64_t stride) {
    if (N > 1 && stride == 1) {
      __builtin_memcpy(w, p, N);
    } else {
#pragma unroll
      for (int i = 0; i < (N + 3) / 4; ++i) w[i] = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) w[i / 4] |= (uint32_t)p[i * stride] << (8 * (i % 4));
    }
  }
  __device__ __forceinline__ bool open(int i) const { return (w[i / 4] >> (8 * (i % 4))) & 0xffu; }
};

// Chunk c of a row of A >= N logits starts at j0. The last one ends with the row: its first `skip`
// elements belong to the chunk before it too (both write the same values there, but only one adds
// them up). Chunks past the row's end are all skip, and not written.
template <int N>
__device__ __forceinline__ void place(int c, int A, int& j0, int& skip) {
  const int at = c * N;
  j0 = at < A - N ? at : A - N;
  skip = at - j0 < N ? at - j0 : N;
}

// Rows of up to 4 KB: 1 << lg lanes take a row, R chunks each; joined by lane moves, without a barrier. Bound
// by HBM (policy fp32 65536 x 512 51 us, 5.3 TB/s), short rows by what each row takes besides its elements
// (bf16 131072 x 128 22 us, 3.2 TB/s; balance 17 us for the same).
template <class OP, class E, int N, int R>
__global__ __launch_bounds__(256) void loss_wave_k(typename OP::Args s, int lg, int nb) {
  typedef typename E::T T;
  typedef Chunk<E, N> Ch;
  __shared__ double lds[4][3];
  __shared__ float f[OP::kBal ? kMaxTargets : 1];
  fill_targets(s, nb, f);
  const int A = s.c.A, gl = threadIdx.x & ((1 << lg) - 1), per = 256 >> lg;
  int j0[R], skip[R];
#pragma unroll
  for (int r = 0; r < R; ++r) place<N>(gl + (r << lg), A, j0[r], skip[r]);
  float fj[OP::kBal ? R : 1][OP::kBal ? N : 1];
  if constexpr (OP::kBal) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int i = 0; i < N; ++i) fj[r][i] = target(s, f, j0[r] + i);
    }
  }
  Sums sums{0.0, 0.0, 0.0};
  for (int64_t n0 = (int64_t)blockIdx.x * per; n0 < s.c.N; n0 += (int64_t)gridDim.x * per) {
    const int64_t n = n0 + (threadIdx.x >> lg);
    const bool in = n < s.c.N;
    typename OP::Row row;
    bool on = in && OP::open(s, n, row);
    Ch ch[R];
    float la = 0.0f;
    if (on) {
      const T* l = static_cast<const T*>(s.l.data) + n * s.l.stride_n;
#pragma unroll
      for (int r = 0; r < R; ++r) ch[r].load(l + j0[r]);
      la = OP::template taken<T>(s, n, row);
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r) ch[r].v = typename Ch::Val{};
    }
    float x[R][N];
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[r][i] = ch[r].get(i);
    }
    if constexpr (!OP::kBal) {
      if (s.mask.data && on) {
        const uint8_t* mk = static_cast<const uint8_t*>(s.mask.data) + n * s.mask.stride_n;
        MaskBytes<N> mb[R];
#pragma unroll
        for (int r = 0; r < R; ++r) mb[r].load(mk + j0[r] * s.mask.stride_a, s.mask.stride_a);
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
          for (int i = 0; i < N; ++i) x[r][i] = mb[r].open(i) ? x[r][i] : -INFINITY;
        }
      }
    }
    Part p{-INFINITY, 0.0f, 0.0f};
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int i = 0; i < N; ++i) p.m = max_nan(p.m, x[r][i]);
    }
    p.m = max_lanes(p.m, lg);
    const float m = p.m == -INFINITY ? 0.0f : p.m;
    float e[R][N];
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[r][i] = max_nan(x[r][i] - m, kLowest);
        e[r][i] = exp_of(x[r][i]);
        const float add = i >= skip[r] ? e[r][i] : 0.0f;
        p.S += add;
        p.X = fmaf(add, OP::kBal ? fj[OP::kBal ? r : 0][OP::kBal ? i : 0] : x[r][i], p.X);
      }
    }
    add_lanes(p.S, p.X, lg);
    RowOut o{0.0f, 0.0f, 0.0f};
    on = on && OP::close(s, n, row, p, la, gl == 0, sums, o);
    if (in && !on && gl == 0) OP::shut(s, n);
    if (s.grad.data && in) {
      T* g = static_cast<T*>(s.grad.data) + n * s.grad.stride_n;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        typename Ch::Wide w;
#pragma unroll
        for (int i = 0; i < N; ++i)
          w[i] = e[r][i] * fmaf(o.beta, OP::kBal ? fj[OP::kBal ? r : 0][OP::kBal ? i : 0] : x[r][i], o.alpha);
        if constexpr (!OP::kBal) {
          const int64_t at = row.act - j0[r];
          if (at >= 0 && at < N) {
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] += at == i ? o.delta : 0.0f;
          }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = on ? w[i] : 0.0f;
        if (skip[r] < N) Ch::store(g + j0[r], w);
      }
    }
  }
  leave<OP>(s, sums, lds);
}

// A row's part per wave, joined over the workgroup's NW waves; lds: two uses one after the other take
// different buffers.
template <bool BAL, int NW>
__device__ __forceinline__ Part join_waves(Part p, Part* lds) {
  if (NW == 1) return p;
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) lds[wave] = p;
  __syncthreads();
  const Part q = lds[(threadIdx.x & 63) % NW];   // a lane holds each wave's part
  constexpr int lg = NW == 2 ? 1 : (NW == 4 ? 2 : (NW == 8 ? 3 : 4));
  Part r = against<BAL>(q, max_lanes(q.m, lg));
  add_lanes(r.S, r.X, lg);
  return r;
}

// a thread's part joined over its workgroup
template <bool BAL, int NW>
__device__ __forceinline__ Part join_threads(Part p, Part* lds) {
  p = against<BAL>(p, wave_max(p.m));
  p.S = wave_add(p.S);
  p.X = wave_add(p.X);
  return join_waves<BAL, NW>(p, lds);
}

// Longer rows: a workgroup takes a row and holds it as it was read, R chunks a thread; while a chunk's
// gradient goes out the same chunk of the workgroup's next row comes in. Places past the row's end hold
// -inf. One read and one write: bf16 4096 x 131072 492 us, 4.4 TB/s; of odd length, off the cache lines, 2048 x
// 50257 106 us, 3.9 TB/s. A row's chain (loads, two joins, gradient) is hidden by the other workgroups of the
// CU alone, 4 waves per SIMD of 128 registers; 8 chunks a thread instead of 16 are slower.
template <class E, int NT, int R, bool MASK>
__global__ __launch_bounds__(NT, 4) void policy_block_k(PolicyLossArgs s) {
  typedef PolicyOp OP;
  typedef typename E::T T;
  constexpr int N = 16 / sizeof(T), NW = NT / 64;
  typedef Chunk<E, N> Ch;
  __shared__ double lds[NW][3];
  __shared__ Part parts[2][NW];
  __shared__ float taken[2];
  const int A = s.c.A;
  T* g = static_cast<T*>(s.grad.data);
  Ch ch[R];
  MaskBytes<N> mb[MASK ? R : 1];
  const T none = (T)-INFINITY;
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int i = 0; i < N; ++i) ch[r].v[i] = none;
  }
  // chunk r of row n; at: its first element
  auto fetch = [&](int r, int at, int64_t n) {
    const T* l = static_cast<const T*>(s.l.data) + n * s.l.stride_n;
    const uint8_t* mk = nullptr;
    if constexpr (MASK) mk = static_cast<const uint8_t*>(s.mask.data) + n * s.mask.stride_n;
    if (at + N <= A) {
      ch[r].load(l + (uint32_t)at);
      if constexpr (MASK) mb[r].load(mk + at * s.mask.stride_a, s.mask.stride_a);
    } else if (at < A) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        ch[r].v[i] = at + i < A ? l[at + i] : none;
        if constexpr (MASK) {
          if (i % 4 == 0) mb[r].w[i / 4] = 0;
          if (at + i < A) mb[r].w[i / 4] |= (uint32_t)mk[(at + i) * s.mask.stride_a] << (8 * (i % 4));
        }
      }
    }
  };
  auto value = [&](int r, int i) {
    const float v = ch[r].get(i);
    if constexpr (MASK) return mb[r].open(i) ? v : -INFINITY;
    else return v;
  };
  Sums sums{0.0, 0.0, 0.0};
  OP::Row row, next;
  bool on = false, on_next = false;
  const int64_t step = gridDim.x;
  if (blockIdx.x < s.c.N) on_next = OP::open(s, blockIdx.x, next);
  if (on_next) {
#pragma unroll
    for (int r = 0; r < R; ++r) fetch(r, (threadIdx.x + r * NT) * N, blockIdx.x);
  }
  int use = 0;
  for (int64_t n = blockIdx.x; n < s.c.N; n += step) {
    row = next;
    on = on_next;
    on_next = n + step < s.c.N && OP::open(s, n + step, next);
    RowOut o{0.0f, 0.0f, 0.0f};
    float m = 0.0f;
    if (on) {   // the same in the whole workgroup
      float la = 0.0f;   // one wave reads it itself
      if (NW == 1) la = OP::template taken<T>(s, n, row);
      else if (threadIdx.x == 0) taken[use] = OP::template taken<T>(s, n, row);
      // 16 elements at a time, as they come in, against the thread's maximum so far
      constexpr int K = 16 / N;
      Part p{-INFINITY, 0.0f, 0.0f};
#pragma unroll
      for (int r0 = 0; r0 < R; r0 += K) {
        if (r0 * NT * N < A) {
          float M = p.m;
#pragma unroll
          for (int r = r0; r < r0 + K; ++r) {
#pragma unroll
            for (int i = 0; i < N; ++i) M = max_nan(M, value(r, i));
          }
          p = against<false>(p, M);
          const float from = M == -INFINITY ? 0.0f : M;
#pragma unroll
          for (int r = r0; r < r0 + K; ++r) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
              const float x = max_nan(value(r, i) - from, kLowest), e = exp_of(x);
              p.S += e;
              p.X = fmaf(e, x, p.X);
            }
          }
        }
      }
      p = join_threads<false, NW>(p, parts[use]);
      on = OP::close(s, n, row, p, NW == 1 ? la : taken[use], threadIdx.x == 0, sums, o);
      m = p.m;
      use ^= 1;   // only a row with a barrier between frees the other buffer
    }
    if (!on && threadIdx.x == 0) OP::shut(s, n);
    int at0 = threadIdx.x * N;
    fresh(at0);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int at = at0 + r * NT * N;
      if (g && at < A) {
        ch[r].forget();
        T* out = g + n * s.grad.stride_n;
        typename Ch::Wide w;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float x = max_nan(value(r, i) - m, kLowest);
          w[i] = exp_of(x) * fmaf(o.beta, x, o.alpha);
        }
        const int64_t hit = row.act - at;
        if (hit >= 0 && hit < N) {
#pragma unroll
          for (int i = 0; i < N; ++i) w[i] += hit == i ? o.delta : 0.0f;
        }
        if (!on) w = typename Ch::Wide{};
        if (at + N <= A) {
          Ch::store(out + (uint32_t)at, w);
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (at + i < A) out[at + i] = (T)w[i];
        }
      }
      if (on_next) fetch(r, at, n + step);
    }
  }
  leave<OP>(s, sums, lds);
}

// A run of a row's logits, read where it lies: chunks [c0, c1) and, if `tail`, the elements past the whole
// chunks, by NT threads.
template <class OP, class E, int NT>
struct Run {
  typedef typename E::T T;
  static constexpr int N = 16 / sizeof(T), U = 4;
  typedef Chunk<E, N> Ch;
  const typename OP::Args& s;
  const float* f;
  const T* l;
  const uint8_t* mk = nullptr;
  int64_t ms = 0;
  int c0, c1, whole;
  bool tail;

  __device__ __forceinline__ Run(const typename OP::Args& s_, const float* f_, int64_t n, int c0_, int c1_, bool tail_)
      : s(s_), f(f_), l(static_cast<const T*>(s_.l.data) + n * s_.l.stride_n), c0(c0_), c1(c1_),
        whole(s_.c.A / N), tail(tail_) {
    if constexpr (!OP::kBal) {
      if (s.mask.data) mk = static_cast<const uint8_t*>(s.mask.data) + n * s.mask.stride_n;
      ms = s.mask.stride_a;
    }
  }
  __device__ __forceinline__ float factor(int j, float x) const { return OP::kBal ? target(s, f, j) : x; }
  __device__ __forceinline__ float logit(int j) const { return !mk || mk[j * ms] ? (float)l[j] : -INFINITY; }
  __device__ __forceinline__ void fetch(int c, Ch (&ch)[U], MaskBytes<N> (&mb)[U]) const {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (c + u * NT < c1) {
        ch[u].load(l + (int64_t)(c + u * NT) * N);
        if (mk) mb[u].load(mk + (int64_t)(c + u * NT) * N * ms, ms);
      }
    }
  }
  // the thread's part
  __device__ __forceinline__ Part part() const {
    Part p{-INFINITY, 0.0f, 0.0f};
    for (int at = c0 + threadIdx.x; at < c1; at += U * NT) {
      Ch ch[U];
      MaskBytes<N> mb[U];
      fetch(at, ch, mb);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = at + u * NT;
        if (c >= c1) continue;
        float v[N], M = p.m;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          v[i] = !mk || mb[u].open(i) ? ch[u].get(i) : -INFINITY;
          M = max_nan(M, v[i]);
        }
        if (M == -INFINITY) continue;
        p = against<OP::kBal>(p, M);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float x = max_nan(v[i] - M, kLowest), e = exp_of(x);
          p.S += e;
          p.X = fmaf(e, factor(c * N + i, x), p.X);
        }
      }
    }
    for (int j = whole * N + threadIdx.x; tail && j < s.c.A; j += NT) {
      const float v = logit(j), M = max_nan(p.m, v);
      if (M == -INFINITY) continue;
      p = against<OP::kBal>(p, M);
      const float x = max_nan(v - M, kLowest), e = exp_of(x);
      p.S += e;
      p.X = fmaf(e, factor(j, x), p.X);
    }
    return p;
  }
  // the gradient, 0 if the row is not on
  __device__ __forceinline__ void slopes(T* out, bool on, float m, const RowOut& o, int64_t act) const {
    auto slope = [&](int j, float v) {
      const float x = max_nan(v - m, kLowest), w = exp_of(x) * fmaf(o.beta, factor(j, x), o.alpha);
      return act == j ? w + o.delta : w;
    };
    for (int at = c0 + threadIdx.x; at < c1; at += U * NT) {
      Ch ch[U];
      MaskBytes<N> mb[U];
      if (on) fetch(at, ch, mb);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = at + u * NT;
        if (c >= c1) continue;
        typename Ch::Wide w{};
        if (on) {
#pragma unroll
          for (int i = 0; i < N; ++i) w[i] = slope(c * N + i, !mk || mb[u].open(i) ? ch[u].get(i) : -INFINITY);
        }
        Ch::store(out + (int64_t)c * N, w);
      }
    }
    for (int j = whole * N + threadIdx.x; tail && j < s.c.A; j += NT) out[j] = (T)(on ? slope(j, logit(j)) : 0.0f);
  }
};
// Rows that no workgroup's registers hold: a workgroup reads a row twice (bf16 512 x 300000 197 us, 4.7 TB/s
// counting both reads). Masked rows of more than 8192 chunks and all of more than 16384 come here (bf16 65536 and
// 131072 logits, fp32 half as many) but for few rows: a mask's bytes take as many registers again.
constexpr int kStream = 1024;
template <class OP, class E>
__global__ __launch_bounds__(kStream) void loss_stream_k(typename OP::Args s, int nb) {
  typedef typename E::T T;
  constexpr int NW = kStream / 64;
  __shared__ double lds[NW][3];
  __shared__ Part parts[2][NW];
  __shared__ float taken[2];
  __shared__ float f[OP::kBal ? kMaxTargets : 1];
  fill_targets(s, nb, f);
  T* g = static_cast<T*>(s.grad.data);
  Sums sums{0.0, 0.0, 0.0};
  int use = 0;
  for (int64_t n = blockIdx.x; n < s.c.N; n += gridDim.x) {
    typename OP::Row row;
    bool on = OP::open(s, n, row);
    const Run<OP, E, kStream> run(s, f, n, 0, s.c.A / Run<OP, E, kStream>::N, true);
    RowOut o{0.0f, 0.0f, 0.0f};
    float m = 0.0f;
    if (on) {
      if (threadIdx.x == 0) taken[use] = OP::template taken<T>(s, n, row);
      const Part p = join_threads<OP::kBal, NW>(run.part(), parts[use]);
      on = OP::close(s, n, row, p, taken[use], threadIdx.x == 0, sums, o);
      m = p.m;
      use ^= 1;   // only a row with a barrier between frees the other buffer
    }
    if (!on && threadIdx.x == 0) OP::shut(s, n);
    if (g) run.slopes(g + n * s.grad.stride_n, on, m, o, row.act);
  }
  leave<OP>(s, sums, lds);
}

// Few long rows: gridDim.y workgroups share each, in two launches. The work memory past the sums holds
// their parts [N][gridDim.y] and the taken actions' logits [N] (the gradient may overwrite them).
constexpr int kSplit = 256, kSplitMost = 1024;
__device__ __forceinline__ Part* split_parts(const PolicyLossArgs& s) {
  return reinterpret_cast<Part*>(static_cast<double*>(s.work) + 3 * kMaxBlocks);
}
template <class E>
__device__ __forceinline__ Run<PolicyOp, E, kSplit> split_run(const PolicyLossArgs& s) {
  const int whole = s.c.A / Run<PolicyOp, E, kSplit>::N, k = gridDim.y, i = blockIdx.y;
  return Run<PolicyOp, E, kSplit>(s, nullptr, blockIdx.x, (int)((int64_t)whole * i / k),
                                  (int)((int64_t)whole * (i + 1) / k), i + 1 == k);
}
template <class E>
__global__ __launch_bounds__(kSplit) void policy_parts_k(PolicyLossArgs s) {
  __shared__ Part lds[kSplit / 64];
  PolicyOp::Row row;
  if (!PolicyOp::open(s, blockIdx.x, row)) return;   // the same in the whole workgroup
  float la = 0.0f;
  if (blockIdx.y == 0 && threadIdx.x == 0) la = PolicyOp::taken<typename E::T>(s, blockIdx.x, row);
  const Part p = join_threads<false, kSplit / 64>(split_run<E>(s).part(), lds);
  if (threadIdx.x != 0) return;
  split_parts(s)[blockIdx.x * gridDim.y + blockIdx.y] = p;
  if (blockIdx.y == 0) reinterpret_cast<float*>(split_parts(s) + kSplitMost)[blockIdx.x] = la;
}
template <class E>
__global__ __launch_bounds__(kSplit) void policy_slopes_k(PolicyLossArgs s) {
  typedef typename E::T T;
  __shared__ double lds[kSplit / 64][3];
  const int64_t n = blockIdx.x;
  Sums sums{0.0, 0.0, 0.0};
  PolicyOp::Row row;
  bool on = PolicyOp::open(s, n, row);
  const bool first = blockIdx.y == 0 && threadIdx.x == 0;
  RowOut o{0.0f, 0.0f, 0.0f};
  float m = 0.0f;
  if (on) {
    const Part* parts = split_parts(s) + n * gridDim.y;
    float M = -INFINITY;
    for (int i = 0; i < gridDim.y; ++i) M = max_nan(M, parts[i].m);
    Part p{M, 0.0f, 0.0f};
    for (int i = 0; i < gridDim.y; ++i) {
      const Part q = against<false>(parts[i], M);
      p.S += q.S;
      p.X += q.X;
    }
    on = PolicyOp::close(s, n, row, p, reinterpret_cast<const float*>(split_parts(s) + kSplitMost)[n], first, sums, o);
    m = p.m;
  }
  if (!on && first) PolicyOp::shut(s, n);
  if (s.grad.data) split_run<E>(s).slopes(static_cast<T*>(s.grad.data) + n * s.grad.stride_n, on, m, o, row.act);
  leave<PolicyOp>(s, sums, lds);
}

// The place of a workgroup among all: in turn, or each XCD with a run of neighbours, where a wave's piece of a
// row is 512 bytes (us in turn and so, masked: fp32 131072 x 96 34.7, 33.0; 131072 x 72 30.7, 28.8; 66904 x 72
// 24.5, 23.7; pieces of 256, bf16 131072 x 72 28.8, 29.1; one workgroup a CU, fp32 40000 x 160 21.8, 24.5).
// Over fp32 samples and actions, both losses: 0.99 to 1.08 of the other way's speed with up to 12 actions and
// around 131072 samples (balance 131072 x 24 22.7, 21.0; policy 131072 x 12 10.4, 9.7), 0.92 to 1.01 with few
// samples of more actions (65536 x 24 8.5, 9.2; 16384 x 72 8.3, 8.7), 0.93 to 1.05 with 262144 (x 72 masked 56.6,
// 60.8; balance x 24 26.8, 25.4).
template <bool RUNS>
__device__ __forceinline__ int64_t first_of() {
  if constexpr (RUNS) {
    const uint32_t each = gridDim.x >> 3, rest = gridDim.x & 7, xcd = blockIdx.x & 7;
    return xcd * each + (xcd < rest ? xcd : rest) + (blockIdx.x >> 3);
  }
  return blockIdx.x;
}

// ---- logits of adjacent samples: [A][N] --------------------------------------------------------
// A lane takes two adjacent samples; W waves share them, each with up to R of their actions, and one
// thread a sample joins the waves' parts and closes it. GR such groups make a workgroup. Bound by HBM and the
// two barriers (policy fp32 131072 x 96 masked 30 us, 3.9 TB/s; balance 65536 x 48 11.4 us): more waves with 6
// actions each hold fewer loads (43 us for 35, with the sum's launch), fewer registers for more waves spill (40).
template <class OP, class E, int W, int GR, int R>
__global__ __launch_bounds__(64 * W * GR) void loss_cols_k(typename OP::Args s, int nb) {
  typedef typename E::T T;
  typedef T Raw __attribute__((ext_vector_type(2), aligned(sizeof(T))));
  typedef T Val __attribute__((ext_vector_type(2)));
  typedef uint8_t Bytes __attribute__((ext_vector_type(2), aligned(1)));
  struct Closed { float m, alpha, beta, delta; int act; };   // act -2: the sample gives nothing
  constexpr bool kShare = W > 1;
  // parts joined at once: two, or they and 24 logits spill (policy 40000 x 300 columns 40 -> 35 us); with 12
  // all of them (balance 30000 x 162 22.3 us, two at a time 23.2)
  constexpr int kJoin = R > 12 ? 2 : W;
  __shared__ double lds[W * GR][3];
  __shared__ Part parts[kShare ? W * GR : 1][128];
  __shared__ Closed closed[kShare ? GR : 1][128];
  __shared__ float f[OP::kBal ? kMaxTargets : 1];
  fill_targets(s, nb, f);
  const int A = s.c.A, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // the same in all of a wave's lanes
  const int wa = wave % W, grp = wave / W, mine = (A - wa + W - 1) / W;
  const T* l0 = static_cast<const T*>(s.l.data);
  T* g0 = static_cast<T*>(s.grad.data);
  const int64_t N = s.c.N, ls = s.l.stride_n, gs = s.grad.stride_n;
  Sums sums{0.0, 0.0, 0.0};
  for (int64_t n0 = first_of<sizeof(T) == 4 && W <= 8>() * 128 * GR; n0 < N; n0 += (int64_t)gridDim.x * 128 * GR) {
    // every lane has both samples, side by side: pairs at a lane's offset from the row's address
    const bool fits = n0 + 128 * GR <= N && ls == 1 && (!g0 || gs == 1);
    either(fits, [&](auto ALL) {
    constexpr bool WHOLE = decltype(ALL)::value;
    int64_t base = n0 + grp * 128;
    int64_t la = s.l.stride_a, ma = 0, ga = s.grad.stride_a;
    if constexpr (!OP::kBal) ma = s.mask.stride_a;
    fresh(base);
    fresh(la);
    fresh(ma);
    fresh(ga);
    const int64_t n = base + 2 * lane;
    const bool in0 = n < N, in1 = n + 1 < N;
    // what a sample has besides its logits, read ahead of them by the thread that will close it
    constexpr int OWN = kShare ? 1 : 2;
    typename OP::Row rows[OWN];
    bool on[OWN];
    float taken[OWN];
#pragma unroll
    for (int v = 0; v < OWN; ++v) {
      const int64_t t = kShare ? n0 + threadIdx.x : n + v;
      on[v] = (!kShare || threadIdx.x < 128 * GR) && t < N && OP::open(s, t, rows[v]);
      taken[v] = on[v] ? OP::template taken<T>(s, t, rows[v]) : 0.0f;
    }
    float x[R][2];
    if constexpr (WHOLE) {
      const T* row = l0 + base + wa * la;
#pragma unroll
      for (int i = 0; i < R; ++i, row += W * la) {
        x[i][0] = x[i][1] = -INFINITY;
        if (i < mine) {
          const Raw v = *reinterpret_cast<const Raw*>(row + 2u * lane);
          x[i][0] = (float)v[0];
          x[i][1] = (float)v[1];
        }
      }
    } else {
      const int64_t at[2] = {(in0 ? n : N - 1) * ls, (in1 ? n + 1 : N - 1) * ls};
      const T* row = l0 + wa * la;
#pragma unroll
      for (int i = 0; i < R; ++i, row += W * la) {
#pragma unroll
        for (int v = 0; v < 2; ++v) x[i][v] = i < mine ? (float)row[at[v]] : -INFINITY;
      }
    }
    if constexpr (!OP::kBal) {
      if (s.mask.data) {
        const int64_t ms = s.mask.stride_n;
        const uint8_t* row = static_cast<const uint8_t*>(s.mask.data) + wa * ma;
        if (WHOLE && ms == 1) {
          Bytes open[R];
          row += base;
#pragma unroll
          for (int i = 0; i < R; ++i, row += W * ma)
            open[i] = i < mine ? *reinterpret_cast<const Bytes*>(row + 2u * lane) : Bytes{0, 0};
#pragma unroll
          for (int i = 0; i < R; ++i) {
#pragma unroll
            for (int v = 0; v < 2; ++v) x[i][v] = open[i][v] ? x[i][v] : -INFINITY;
          }
        } else {
          const int64_t at[2] = {(in0 ? n : N - 1) * ms, (in1 ? n + 1 : N - 1) * ms};
#pragma unroll
          for (int i = 0; i < R; ++i, row += W * ma) {
#pragma unroll
            for (int v = 0; v < 2; ++v) x[i][v] = i < mine && row[at[v]] ? x[i][v] : -INFINITY;
          }
        }
      }
    }
    Part p[2];
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      p[v] = Part{-INFINITY, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < R; ++i) p[v].m = max_nan(p[v].m, x[i][v]);
      const float m = p[v].m == -INFINITY ? 0.0f : p[v].m;
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const float d = max_nan(x[i][v] - m, kLowest), e = exp_of(d);
        p[v].S += e;
        p[v].X = fmaf(e, OP::kBal ? (i < mine ? target(s, f, wa + W * i) : 0.0f) : d, p[v].X);
      }
    }
    Closed c[2];
    auto close = [&](int64_t t, int v, const Part& whole) {
      RowOut o{0.0f, 0.0f, 0.0f};
      const bool gives = on[v] && OP::close(s, t, rows[v], whole, taken[v], true, sums, o);
      if (!gives) OP::shut(s, t);
      return Closed{whole.m == -INFINITY ? 0.0f : whole.m, o.alpha, o.beta, o.delta, gives ? (int)rows[v].act : -2};
    };
    if constexpr (kShare) {
      static_assert(W >= 2, "a thread for each sample");
#pragma unroll
      for (int v = 0; v < 2; ++v) parts[wave][2 * lane + v] = p[v];
      __syncthreads();
      const int kg = threadIdx.x / 128, ks = threadIdx.x % 128;
      if (kg < GR && n0 + threadIdx.x < N) {
        float M = parts[kg * W][ks].m;
#pragma unroll kJoin
        for (int w = 1; w < W; ++w) M = max_nan(M, parts[kg * W + w][ks].m);
        Part whole{M, 0.0f, 0.0f};
#pragma unroll kJoin
        for (int w = 0; w < W; ++w) {
          const Part q = against<OP::kBal>(parts[kg * W + w][ks], M);
          whole.S += q.S;
          whole.X += q.X;
        }
        closed[kg][ks] = close(n0 + threadIdx.x, 0, whole);
      }
      __syncthreads();
      c[0] = closed[grp][2 * lane];
      c[1] = closed[grp][2 * lane + 1];
    } else {
      c[0] = c[1] = Closed{0.0f, 0.0f, 0.0f, 0.0f, -2};
      if (in0) c[0] = close(n, 0, p[0]);
      if (in1) c[1] = close(n + 1, OWN - 1, p[1]);
    }
    if (g0) {
      T* row = g0 + wa * ga;
      const int64_t at = n * gs;
#pragma unroll
      for (int i = 0; i < R; ++i, row += W * ga) {
        if (i < mine) {
          const int a = wa + W * i;
          float w[2];
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const float d = max_nan(x[i][v] - c[v].m, kLowest);
            w[v] = exp_of(d) * fmaf(c[v].beta, OP::kBal ? target(s, f, a) : d, c[v].alpha);
            if (!OP::kBal) w[v] += c[v].act == a ? c[v].delta : 0.0f;
            w[v] = c[v].act == -2 ? 0.0f : w[v];
          }
          if constexpr (WHOLE) {
            typedef float Two __attribute__((ext_vector_type(2)));
            *reinterpret_cast<Raw*>(row + base + 2u * lane) =
                __builtin_bit_cast(Raw, __builtin_convertvector((Two{w[0], w[1]}), Val));
          } else {
            if (in0) row[at] = (T)w[0];
            if (in1) row[at + gs] = (T)w[1];
          }
        }
      }
    }
    });
  }
  __syncthreads();
  leave<OP>(s, sums, lds);
}

// More actions than the waves of a workgroup hold: a lane takes a sample, kLaneWaves waves share its actions
// and read them twice (policy fp32 65536 x 500 81 us, 4.9 TB/s counting both reads; balance 87; few samples of
// many actions leave most of the chip empty: bf16 2048 x 50257 2.5 ms, by rows 106 us).
constexpr int kLaneWaves = 16;
template <class OP, class E>
__global__ __launch_bounds__(64 * kLaneWaves) void loss_lane_k(typename OP::Args s, int nb) {
  typedef typename E::T T;
  constexpr int U = 8;   // loads that fly together
  struct Closed { float m, alpha, beta, delta; int64_t act; bool on; };
  __shared__ double lds[kLaneWaves][3];
  __shared__ Part parts[kLaneWaves][64];
  __shared__ Closed closed[64];
  __shared__ float f[OP::kBal ? kMaxTargets : 1];
  fill_targets(s, nb, f);
  const int A = s.c.A, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // the same in all of a wave's lanes
  Sums sums{0.0, 0.0, 0.0};
  for (int64_t n0 = (int64_t)blockIdx.x * 64; n0 < s.c.N; n0 += (int64_t)gridDim.x * 64) {
    const bool in = n0 + lane < s.c.N;
    const int64_t n = in ? n0 + lane : s.c.N - 1;
    const T* l = static_cast<const T*>(s.l.data) + n * s.l.stride_n;
    // logits a0, a0 + kLaneWaves, ...: those past the last one and masked ones are -inf
    auto read = [&](int a0, float (&v)[U]) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int a = a0 + u * kLaneWaves;
        v[u] = a < A ? (float)l[a * s.l.stride_a] : -INFINITY;
      }
      if constexpr (!OP::kBal) {
        if (s.mask.data) {
          const uint8_t* mk = static_cast<const uint8_t*>(s.mask.data) + n * s.mask.stride_n;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int a = a0 + u * kLaneWaves;
            if (a < A && !mk[a * s.mask.stride_a]) v[u] = -INFINITY;
          }
        }
      }
    };
    Part p{-INFINITY, 0.0f, 0.0f};
    for (int a0 = wave; a0 < A; a0 += U * kLaneWaves) {
      float v[U], M = p.m;
      read(a0, v);
#pragma unroll
      for (int u = 0; u < U; ++u) M = max_nan(M, v[u]);
      p = against<OP::kBal>(p, M);
      const float m = M == -INFINITY ? 0.0f : M;
      // a round's terms are added up among themselves: a lane's sums take A / 128 additions one after
      // another, as few as the other forms'
      float e[U], ex[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int a = a0 + u * kLaneWaves;
        const float x = max_nan(v[u] - m, kLowest);
        e[u] = exp_of(x);
        ex[u] = e[u] * (OP::kBal ? (a < A ? target(s, f, a) : 0.0f) : x);
      }
#pragma unroll
      for (int h = U / 2; h; h /= 2) {
#pragma unroll
        for (int u = 0; u < h; ++u) {
          e[u] += e[u + h];
          ex[u] += ex[u + h];
        }
      }
      p.S += e[0];
      p.X += ex[0];
    }
    parts[wave][lane] = p;
    __syncthreads();
    if (wave == 0) {
      Closed c{0.0f, 0.0f, 0.0f, 0.0f, -1, false};
      typename OP::Row row;
      if (in && OP::open(s, n, row)) {
        float M = parts[0][lane].m;
#pragma unroll 4
        for (int w = 1; w < kLaneWaves; ++w) M = max_nan(M, parts[w][lane].m);
        Part whole{M, 0.0f, 0.0f};
#pragma unroll 4
        for (int w = 0; w < kLaneWaves; ++w) {
          const Part q = against<OP::kBal>(parts[w][lane], M);
          whole.S += q.S;
          whole.X += q.X;
        }
        RowOut o{0.0f, 0.0f, 0.0f};
        c.on = OP::close(s, n, row, whole, OP::template taken<T>(s, n, row), true, sums, o);
        c = Closed{M, o.alpha, o.beta, o.delta, (int64_t)row.act, c.on};
      }
      if (in && !c.on) OP::shut(s, n);
      closed[lane] = c;
    }
    __syncthreads();
    if (s.grad.data && in) {
      const Closed c = closed[lane];
      T* g = static_cast<T*>(s.grad.data) + n * s.grad.stride_n;
      for (int a0 = wave; a0 < A; a0 += U * kLaneWaves) {
        float v[U];
        read(a0, v);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int a = a0 + u * kLaneWaves;
          if (a >= A) continue;
          const float x = max_nan(v[u] - c.m, kLowest);
          float w = exp_of(x) * fmaf(c.beta, OP::kBal ? target(s, f, a) : x, c.alpha);
          if (!OP::kBal && c.act == a) w += c.delta;
          g[a * s.grad.stride_a] = (T)(c.on ? w : 0.0f);
        }
      }
    }
  }
  __syncthreads();
  leave<OP>(s, sums, lds);
}

// ---- choice of the form -------------------------------------------------------------------------
int ceil_log2(int64_t x) {
  int r = 0;
  while (((int64_t)1 << r) < x) ++r;
  return r;
}
int blocks_for(int64_t N, int per, int most) {
  const int64_t b = (N + per - 1) / per;
  return (int)(b < 1 ? 1 : (b > most ? most : b));
}

constexpr int kHeld = 16;             // chunks of a row that a thread holds
constexpr int kSplitFrom = 4, kSplitChunks = 4096;   // workgroups that share a row, from which length
constexpr int kFill = 256 * 1024;     // threads that fill the chip while they hold a row (128 registers each)

// samples whose 193 to 384 actions are held
template <class OP>
constexpr int64_t kHold24 = OP::kBal ? 65536 : 32768;

// Launches the form for these sizes and strides; the workgroups that left sums.
template <class OP, class E>
int launch_rows(const typename OP::Args& a, int nb, hipStream_t st) {
  constexpr int N = 16 / sizeof(typename E::T);
  const int A = a.c.A;
  const int64_t rows = a.c.N;
  const bool adjacent = (a.l.stride_a == 1 || A == 1) && (!a.grad.data || a.grad.stride_a == 1 || A == 1);
  if (!adjacent) {
    // Waves that share a sample, each with at most 12 of its actions, or 24 with the most waves and samples:
    // they leave little room beside them, which reading the samples twice does (us held and read twice, fp32:
    // policy 2000 x 200 16.5, 11.6; 40000 x 380 42.3, 41.3, masked 68, 83; 100000 x 200 63, 73; with 12 8000 x
    // 160 11.5, 12.5; balance 2000 x 200 23.6, 15.7; 40000 x 380 61, 49; 100000 x 200 50, 67).
    const int lw = ceil_log2((A + 11) / 12), each = 128 * (lw < 2 ? 4 >> lw : 1);
    if (A > 16 * 24 || (A > 16 * 12 && rows < kHold24<OP>)) {
      const int g = blocks_for(rows, 64, kMaxBlocks);
      hipLaunchKernelGGL((loss_lane_k<OP, E>), dim3(g), dim3(64 * kLaneWaves), 0, st, a, nb);
      return g;
    }
    const int g = blocks_for(rows, each, kMaxBlocks);
    const dim3 grid(g), block(lw < 2 ? 256 : std::min(1024, 64 << lw));
    if (A <= 6) hipLaunchKernelGGL((loss_cols_k<OP, E, 1, 4, 6>), grid, block, 0, st, a, nb);
    else if (lw == 0) hipLaunchKernelGGL((loss_cols_k<OP, E, 1, 4, 12>), grid, block, 0, st, a, nb);
    else if (lw == 1) hipLaunchKernelGGL((loss_cols_k<OP, E, 2, 2, 12>), grid, block, 0, st, a, nb);
    else if (lw == 2) hipLaunchKernelGGL((loss_cols_k<OP, E, 4, 1, 12>), grid, block, 0, st, a, nb);
    else if (lw == 3) hipLaunchKernelGGL((loss_cols_k<OP, E, 8, 1, 12>), grid, block, 0, st, a, nb);
    else if (lw == 4) hipLaunchKernelGGL((loss_cols_k<OP, E, 16, 1, 12>), grid, block, 0, st, a, nb);
    else hipLaunchKernelGGL((loss_cols_k<OP, E, 16, 1, 24>), grid, block, 0, st, a, nb);
    return g;
  }
  const int chunks = (A + N - 1) / N;
  if (A < N || chunks <= 256) {
    // four chunks a lane: what a row takes besides its elements is shared by the most rows of a wave
    const int lg = A < N ? ceil_log2(A) : ceil_log2((chunks + 3) / 4);
    const int need = A < N ? 1 : (chunks + (1 << lg) - 1) >> lg;
    const int g = blocks_for(rows, 256 >> lg, kMaxBlocks);
    const dim3 grid(g), block(256);
    if (A < N) hipLaunchKernelGGL((loss_wave_k<OP, E, 1, 1>), grid, block, 0, st, a, lg, nb);
    else if (need == 1) hipLaunchKernelGGL((loss_wave_k<OP, E, N, 1>), grid, block, 0, st, a, lg, nb);
    else if (need == 2) hipLaunchKernelGGL((loss_wave_k<OP, E, N, 2>), grid, block, 0, st, a, lg, nb);
    else hipLaunchKernelGGL((loss_wave_k<OP, E, N, 4>), grid, block, 0, st, a, lg, nb);
    return g;
  }
  if constexpr (!OP::kBal) {
    // Few long rows are shared by as many workgroups as fill the chip and have a chunk a thread; the second
    // launch takes about 3 us (us shared and not, bf16: 16 x 16000 12.0, 11.1; 16 x 50000 14.2, 16.4; 16 x
    // 150000 15.8, 36.8; 60 x 73246 18.5, 21.3; 100 x 20000 13.8, 12.4; fp32 308 x 27036 by two 26.0, 23.0).
    const int share = (int)std::min<int64_t>((2 * 256 + rows - 1) / std::max<int64_t>(rows, 1), chunks / kSplit);
    if (rows > 0 && share >= kSplitFrom && chunks >= kSplitChunks && rows * share <= kSplitMost) {
      const dim3 grid((unsigned)rows, (unsigned)share), block(kSplit);
      hipLaunchKernelGGL(policy_parts_k<E>, grid, block, 0, st, a);
      hipLaunchKernelGGL(policy_slopes_k<E>, grid, block, 0, st, a);
      return (int)rows * share;
    }
    // the fewest threads that hold a row, more where there are too few rows to fill the chip
    int nt = 64;
    while (nt < 1024 && (chunks > kHeld * nt || (nt < 512 && rows * nt < kFill && chunks > nt))) nt *= 2;
    if (chunks <= kHeld * nt && !(a.mask.data && nt == 1024)) {
      const int g = blocks_for(rows, 1, std::min(kMaxBlocks, kFill / nt));
      const dim3 grid(g), block(nt);
      if (a.mask.data) {
        if (nt == 64) hipLaunchKernelGGL((policy_block_k<E, 64, kHeld, true>), grid, block, 0, st, a);
        else if (nt == 128) hipLaunchKernelGGL((policy_block_k<E, 128, kHeld, true>), grid, block, 0, st, a);
        else if (nt == 256) hipLaunchKernelGGL((policy_block_k<E, 256, kHeld, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((policy_block_k<E, 512, kHeld, true>), grid, block, 0, st, a);
      } else {
        if (nt == 64) hipLaunchKernelGGL((policy_block_k<E, 64, kHeld, false>), grid, block, 0, st, a);
        else if (nt == 128) hipLaunchKernelGGL((policy_block_k<E, 128, kHeld, false>), grid, block, 0, st, a);
        else if (nt == 256) hipLaunchKernelGGL((policy_block_k<E, 256, kHeld, false>), grid, block, 0, st, a);
        else if (nt == 512) hipLaunchKernelGGL((policy_block_k<E, 512, kHeld, false>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((policy_block_k<E, 1024, kHeld, false>), grid, block, 0, st, a);
      }
      return g;
    }
  }
  const int g = blocks_for(rows, 1, 512);
  hipLaunchKernelGGL((loss_stream_k<OP, E>), dim3(g), dim3(kStream), 0, st, a, nb);
  return g;
}
template <class OP>
hipError_t launch_loss(const typename OP::Args& a, int nb, hipStream_t st) {
  const int g = a.c.dtype == SIM_DT_F32 ? launch_rows<OP, F32>(a, nb, st)
                : a.c.dtype == SIM_DT_BF16 ? launch_rows<OP, BF16>(a, nb, st) : launch_rows<OP, F16>(a, nb, st);
  if (g > 1) hipLaunchKernelGGL(loss_finish_k<OP>, dim3(1), dim3(kFinish), 0, st, a, g);
  return hipGetLastError();
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
