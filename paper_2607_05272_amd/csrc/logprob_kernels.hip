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
  static constexpr bool kBal = false, kSums = false, kClosed = true;
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
    const float logS = p.m == INFINITY ? NAN : log_of(p.S), rS = __builtin_amdgcn_rcpf(p.S);
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

// ---- with alternatives -------------------------------------------------------------------------
// The order of logits as signed whole numbers (a NaN above all, -0 as 0), kNone for those that are no alternative; and
// back.
constexpr int kNone = INT32_MIN;
__device__ __forceinline__ int order_of(float v) {
  const int u = __float_as_int(v + 0.0f), o = u ^ ((u >> 31) & 0x7FFFFFFF);
  return v == v ? (v == -INFINITY ? kNone : o) : INT32_MAX;
}
__device__ __forceinline__ float value_of(int o) { return __int_as_float(o ^ ((o >> 31) & 0x7FFFFFFF)); }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_of(uint32_t v) { return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false); }
// over 16 or 64 adjacent lanes, in every one: rotations within 16 lanes, then across
template <int LG, class F>
__device__ __forceinline__ int group(int v, F f) {
  v = f(v, dpp_of<0x128>(v));   // row_ror 8, 4, 2, 1
  v = f(v, dpp_of<0x124>(v));
  v = f(v, dpp_of<0x122>(v));
  v = f(v, dpp_of<0x121>(v));
  if constexpr (LG == 6) {
    v = f(v, __shfl_xor(v, 16));
    v = f(v, __shfl_xor(v, 32));
  }
  return v;
}
template <int LG, class F>
__device__ __forceinline__ float group_f(float v, F f) {
  return __int_as_float(group<LG>(__float_as_int(v), [&](int a, int b) { return __float_as_int(f(__int_as_float(a), __int_as_float(b))); }));
}

// Rows of up to 1024: 1 << LG lanes take a row, V logits each, in registers; an alternative is the largest that is left,
// found by a round over the lanes. Of adjacent samples (COLS) a workgroup first turns S of them in LDS. Bound by the
// rounds' chains (some 40 instructions per alternative and 4 rows): fp32 16384 x 96 by columns, six alternatives, 12.1 us for
// 1.6 of HBM.
constexpr int kGroups = 256;
template <class E, int LG, int V, bool COLS>
__global__ __launch_bounds__(kGroups) void logprob_short_k(LogprobArgs s, int S) {
  typedef typename E::T T;
  extern __shared__ float tile[];
  const int A = s.c.A, top = s.c.top, gl = threadIdx.x & ((1 << LG) - 1), per = kGroups >> LG;
  const int64_t N = s.c.N, each = COLS ? S : per;
  const T* l = static_cast<const T*>(s.l.data);
  const uint8_t* mk = static_cast<const uint8_t*>(s.mask.data);
  Sums sums;
  for (int64_t n0 = blockIdx.x * each; n0 < N; n0 += gridDim.x * each) {
    if (COLS) {
      __syncthreads();
      const int k = threadIdx.x % S;
      if (n0 + k < N) {
        const int64_t n = n0 + k;
#pragma unroll 4
        for (int j = threadIdx.x / S; j < A; j += kGroups / S) {
          const float v = (float)l[n * s.l.stride_n + j * s.l.stride_a];
          tile[j * (S + 1) + k] = mk && !mk[n * s.mask.stride_n + j * s.mask.stride_a] ? -INFINITY : v;
        }
      }
      __syncthreads();
    }
    for (int k0 = 0; k0 < each; k0 += per) {
      const int k = k0 + (threadIdx.x >> LG);
      const int64_t n = n0 + k;
      const bool in = n < N && k < each;
      LogprobOp::Row row{0.0f, 0.0f, -1};
      bool on = in && LogprobOp::open(s, n, row);
      float x[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int j = gl + (i << LG);
        x[i] = -INFINITY;
        if (on && j < A) {
          if (COLS) x[i] = tile[j * (S + 1) + k];
          else x[i] = mk && !mk[n * s.mask.stride_n + j * s.mask.stride_a] ? -INFINITY : (float)l[n * s.l.stride_n + j];
        }
      }
      const float la = on && gl == 0 ? LogprobOp::taken<T>(s, n, row) : 0.0f;
      Part p{-INFINITY, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < V; ++i) p.m = max_nan(p.m, x[i]);
      p.m = group_f<LG>(p.m, [](float a, float b) { return max_nan(a, b); });
      const float m = p.m == -INFINITY ? 0.0f : p.m;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = max_nan(x[i] - m, kLowest), e = exp_of(d);
        p.S += e;
        p.X = fmaf(e, d, p.X);
      }
      p.S = group_f<LG>(p.S, [](float a, float b) { return a + b; });
      p.X = group_f<LG>(p.X, [](float a, float b) { return a + b; });
      RowOut o;
      if (gl == 0 && in && !(on && LogprobOp::close(s, n, row, p, la, true, sums, o))) LogprobOp::shut(s, n);
      const float logS = log_of(p.S);
      int q[V];
#pragma unroll
      for (int i = 0; i < V; ++i) q[i] = order_of(x[i]);
      for (int t = 0; t < top; ++t) {
        int best = kNone, at = 0;
#pragma unroll
        for (int i = V - 1; i >= 0; --i) {   // of equal ones the first
          at = q[i] >= best ? i : at;
          best = q[i] >= best ? q[i] : best;
        }
        const int most = group<LG>(best, [](int a, int b) { return a > b ? a : b; });
        const int j = gl + (at << LG);
        const int first = group<LG>(best == most ? j : INT32_MAX, [](int a, int b) { return a < b ? a : b; });
        if (first == j && most != kNone) {
#pragma unroll
          for (int i = 0; i < V; ++i) q[i] = i == at ? kNone : q[i];
        }
        if (in && gl == (t & ((1 << LG) - 1))) {
          if (s.top_index) s.top_index[n * top + t] = most == kNone ? -1 : first;
          if (s.top_logp) s.top_logp[n * top + t] = most == kNone ? -INFINITY : (value_of(most) - p.m) - logS;
        }
      }
    }
  }
}

// A key orders alternatives as one whole number: the logit's order, then the lower column. 0: none.
__device__ __forceinline__ uint64_t key_of(int order, int j) {
  return order == kNone ? 0 : (uint64_t)((uint32_t)order ^ 0x80000000u) << 32 | (uint32_t)~j;
}
__device__ __forceinline__ int order_in(uint64_t key) { return (int)((uint32_t)(key >> 32) ^ 0x80000000u); }
__device__ __forceinline__ int column_in(uint64_t key) { return (int)~(uint32_t)key; }

// lane ^ X, within the vector unit
template <int X>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  if constexpr (X == 1) return dpp_of<0xB1>(v);         // quad_perm 1 0 3 2
  else if constexpr (X == 2) return dpp_of<0x4E>(v);    // 2 3 0 1
  else if constexpr (X == 3) return dpp_of<0x1B>(v);    // 3 2 1 0
  else if constexpr (X == 7) return dpp_of<0x141>(v);   // row_half_mirror
  else if constexpr (X == 15) return dpp_of<0x140>(v);  // row_mirror
  else if constexpr (X == 4) return lane_xor<3>(lane_xor<7>(v));
  else if constexpr (X == 8) return dpp_of<0x128>(v);   // row_ror 8
  else if constexpr (X == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);   // rows 0 0 2 2 and 1 1 3 3
    return threadIdx.x & 16 ? r[0] : r[1];
  } else if constexpr (X == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  } else if constexpr (X == 31) return lane_xor<16>(lane_xor<15>(v));
  else return lane_xor<32>(lane_xor<31>(v));
}
// the larger of the keys of lane and lane ^ X to the lanes without bit B, the smaller one to the others
template <int X, int B>
__device__ __forceinline__ void exchange(uint64_t& k) {
  const uint64_t o = (uint64_t)lane_xor<X>((uint32_t)(k >> 32)) << 32 | lane_xor<X>((uint32_t)k);
  const bool low = threadIdx.x & B;
  k = (o > k) != low ? o : k;
}
// halves that rise and fall, into falling order over 64 lanes
template <int D>
__device__ __forceinline__ void settle(uint64_t& k) {
  exchange<D, D>(k);
  if constexpr (D > 1) settle<D / 2>(k);
}
// 64 keys into falling order: runs of 2, 4, .., each turned against its neighbour and settled
__device__ __forceinline__ void sort_keys(uint64_t& k) {
  exchange<1, 1>(k);
  exchange<3, 2>(k); settle<1>(k);
  exchange<7, 4>(k); settle<2>(k);
  exchange<15, 8>(k); settle<4>(k);
  exchange<31, 16>(k); settle<8>(k);
  exchange<63, 32>(k); settle<16>(k);
}
// the 64 largest of two falling runs
__device__ __forceinline__ uint64_t join_keys(uint64_t a, uint64_t b) {
  const uint64_t o = (uint64_t)lane_xor<63>((uint32_t)(b >> 32)) << 32 | lane_xor<63>((uint32_t)b);
  uint64_t k = o > a ? o : a;
  settle<32>(k);
  return k;
}
__device__ __forceinline__ uint64_t key_at(uint64_t k, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(k >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((uint32_t)k, lane);
}

// Longer rows: a workgroup takes a row or one of gridDim.y parts of it, its waves every fourth stretch of 512 logits. A wave
// keeps its 64 largest keys, one a lane, and collects in LDS what could be among the row's largest `top`: logits not
// below the least of the `top` that any wave has kept (at first, of its lanes' largest ones). 64 of them are sorted and
// joined at once, by moves within the vector unit: after the first stretches few logits are collected at all. Many rows
// are bound by what is done with each logit and by loads that a wave waits for two chunks at a time, not by HBM: twenty
// alternatives of 4096 x 50257 take 193 us in bf16 (2.1 TB/s) as in fp32 (4.3 TB/s), five of fp32 1000 x 20000 34 us (2.4 TB/s).
// Few rows are bound by the chains of all that: bf16 32 x 131072, twenty alternatives, 15.8 us and 4.0 for the parts, for
// 1.7 of HBM.
constexpr int kLong = 256, kLongWaves = kLong / 64;
struct LongPart {
  Part p;
  uint32_t pad;
  uint64_t keys[64];
};
template <class E>
__global__ __launch_bounds__(kLong) void logprob_long_k(LogprobArgs s) {
  typedef typename E::T T;
  constexpr int N = 8, U = 2;   // logits of a lane that are compared together, and chunks that fly together
  typedef Chunk<E, N> Ch;
  __shared__ Part parts[kLongWaves];
  __shared__ uint64_t found[kLongWaves][128];
  __shared__ float taken;
  __shared__ int shared;   // the largest of the waves' least ones that they keep: what is below is none of the row's
  const int A = s.c.A, top = s.c.top, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int units = (A + N - 1) / N, c0 = (int)((int64_t)units * blockIdx.y / gridDim.y),
            c1 = (int)((int64_t)units * (blockIdx.y + 1) / gridDim.y);
  for (int64_t n = blockIdx.x; n < s.c.N; n += gridDim.x) {
    LogprobOp::Row row;
    const bool on = LogprobOp::open(s, n, row);
    Part p{-INFINITY, 0.0f, 0.0f};
    uint64_t best = 0;
    if (on) {
      if (threadIdx.x == 0) {
        taken = LogprobOp::taken<T>(s, n, row);
        shared = kNone;
      }
      __syncthreads();   // a row before may still be read until here
      const T* l = static_cast<const T*>(s.l.data) + n * s.l.stride_n;
      const uint8_t* mk = s.mask.data ? static_cast<const uint8_t*>(s.mask.data) + n * s.mask.stride_n : nullptr;
      int own = kNone, others = kNone, have = 0;   // the least that is kept here and elsewhere; collected keys
      float bound = -INFINITY;
      auto take = [&](uint64_t k) {   // 64 keys join; the bounds rise
        sort_keys(k);
        best = join_keys(best, k);
        own = order_in(key_at(best, top - 1));
        if (lane == 0 && own > others) __hip_atomic_fetch_max(&shared, own, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      };
      auto flush = [&]() {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const uint64_t k = found[wave][lane], rest = found[wave][64 + lane];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        found[wave][lane] = rest;
        take(lane < have ? k : 0);
        have = have > 64 ? have - 64 : 0;
      };
      const int enough = top > 8 ? top : 8;
      for (int at = c0 + threadIdx.x; at - lane < c1; at += U * kLong) {
        Ch ch[U];
        MaskBytes<N> mb[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int j = (at + u * kLong) * N;
          if (at + u * kLong < c1) {
            if (j + N <= A) {
              ch[u].load(l + j);
              if (mk) mb[u].load(mk + j * s.mask.stride_a, s.mask.stride_a);
            } else {
#pragma unroll
              for (int i = 0; i < N; ++i) {
                ch[u].v[i] = j + i < A ? l[j + i] : (T)-INFINITY;
                if (i % 4 == 0) mb[u].w[i / 4] = 0;
                if (mk && j + i < A) mb[u].w[i / 4] |= (uint32_t)mk[(j + i) * s.mask.stride_a] << (8 * (i % 4));
              }
            }
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float x[N], M = -INFINITY;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            x[i] = at + u * kLong < c1 ? ch[u].get(i) : -INFINITY;
            if (mk) x[i] = at + u * kLong < c1 && mb[u].open(i) ? x[i] : -INFINITY;
            M = max_nan(M, x[i]);
          }
          if (!(M == -INFINITY)) {
            p = against<false>(p, max_nan(p.m, M));
#pragma unroll
            for (int i = 0; i < N; ++i) {
              const float d = max_nan(x[i] - p.m, kLowest), e = exp_of(d);
              p.S += e;
              p.X = fmaf(e, d, p.X);
            }
          }
          if (!__any(!(M < bound || M == -INFINITY))) continue;
          others = __builtin_amdgcn_readfirstlane(__hip_atomic_load(&shared, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
          if (own == kNone && others == kNone) {   // the first stretch: `top` of its lanes' largest are a bound
            uint64_t k = key_of(order_of(M), lane);
            sort_keys(k);
            const uint64_t least = key_at(k, top - 1);
            if (least) others = order_in(least);
          }
          const int before = own;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const int q = order_of(x[i]);
            // one equal to the least that this wave kept of earlier stretches has a higher column; else it may have a lower one
            const bool in = q != kNone && q > before && q >= own && q >= others;
            const uint64_t who = __ballot(in);
            if (!who) continue;
            const int place = have + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
            if (in) found[wave][place] = key_of(q, (at + u * kLong) * N + i);
            have += __popcll(who);
            if (have >= 64) flush();
          }
          if (have >= enough) flush();   // the bound follows soon enough
          const int most = own > others ? own : others;
          bound = most == kNone ? -INFINITY : (most == INT32_MAX ? INFINITY : value_of(most));
        }
      }
      if (have) flush();
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      found[wave][lane] = best;
      p = join_threads<false, kLongWaves>(p, parts);
      __syncthreads();
      if (wave == 0) {
        for (int w = 1; w < kLongWaves; ++w) best = join_keys(best, found[w][lane]);
      }
    }
    if (wave != 0) continue;
    if (gridDim.y > 1) {
      LongPart& o = static_cast<LongPart*>(s.work)[n * gridDim.y + blockIdx.y];
      if (lane == 0) o.p = p;
      o.keys[lane] = best;
      continue;
    }
    const float logS = log_of(p.S);
    RowOut o;
    Sums sums;
    if (lane == 0 && !(on && LogprobOp::close(s, n, row, p, taken, true, sums, o))) LogprobOp::shut(s, n);
    if (lane < top) {
      if (s.top_index) s.top_index[n * top + lane] = best ? column_in(best) : -1;
      if (s.top_logp) s.top_logp[n * top + lane] = best ? (value_of(order_in(best)) - p.m) - logS : -INFINITY;
    }
  }
}
// The parts of a row, every fourth a wave.
template <class E>
__global__ __launch_bounds__(kLong) void logprob_join_k(LogprobArgs s, int parts) {
  __shared__ uint64_t lists[kLongWaves][64];
  const int64_t n = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, top = s.c.top;
  const LongPart* in = static_cast<const LongPart*>(s.work) + n * parts;
  uint64_t best = 0;
  constexpr int U = 4;   // loads that fly together
  for (int i0 = wave; i0 < parts; i0 += U * kLongWaves) {
    uint64_t k[U];
#pragma unroll
    for (int u = 0; u < U; ++u) k[u] = i0 + u * kLongWaves < parts ? in[i0 + u * kLongWaves].keys[lane] : 0;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * kLongWaves < parts) best = join_keys(best, k[u]);
  }
  lists[wave][lane] = best;
  __syncthreads();
  if (wave != 0) return;
  LogprobOp::Row row;
  const bool on = LogprobOp::open(s, n, row);
  float M = -INFINITY;
  for (int i = lane; i < parts; i += 64) M = max_nan(M, in[i].p.m);
  M = wave_max(M);
  Part p{M, 0.0f, 0.0f};
  for (int i = lane; i < parts; i += 64) {
    const Part q = against<false>(in[i].p, M);
    p.S += q.S;
    p.X += q.X;
  }
  p.S = wave_add(p.S);
  p.X = wave_add(p.X);
  for (int w = 1; w < kLongWaves; ++w) best = join_keys(best, lists[w][lane]);
  const float logS = log_of(p.S);
  RowOut o;
  Sums sums;
  if (lane == 0) {
    const float la = on ? LogprobOp::taken<typename E::T>(s, n, row) : 0.0f;
    if (!(on && LogprobOp::close(s, n, row, p, la, true, sums, o))) LogprobOp::shut(s, n);
  }
  if (lane < top) {
    if (s.top_index) s.top_index[n * top + lane] = best && on ? column_in(best) : -1;
    if (s.top_logp) s.top_logp[n * top + lane] = best && on ? (value_of(order_in(best)) - p.m) - logS : -INFINITY;
  }
}

// Many adjacent samples of more than 960 columns: one look over the row per alternative, as slow as it is rare.
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
          const uint64_t c = key_of(order_of(logit(j)), j);
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

constexpr int kShort = 1024, kTurned = 960;
// Parts of a long row: enough to fill the chip (32 x 131072: 8 parts a row 24 us, 16 20, 32 19; fp32 1000 x 20000: one 30
// us, two 39)
constexpr int kLongFill = 512, kLongLeast = 4096;
int parts_of(int64_t N, int A) {
  const int64_t want = (kLongFill + N - 1) / std::max<int64_t>(N, 1);
  return (int)std::max<int64_t>(1, std::min<int64_t>(want, A / kLongLeast));
}

template <class E, bool COLS>
void launch_short(const LogprobArgs& a, hipStream_t st) {
  // 32 samples turned at once: of 64 a wave's passes over them follow each other (16384 x 96 12.2 us against 18.6)
  const int A = a.c.A, S = A <= 480 ? 32 : 16;
  const int per = COLS ? S : (A <= 256 ? kGroups / 16 : kGroups / 64);
  const dim3 grid(blocks_for(a.c.N, per, 1 << 16)), block(kGroups);
  const size_t lds = COLS ? (size_t)A * (S + 1) * sizeof(float) : 0;
  if (A <= 64) hipLaunchKernelGGL((logprob_short_k<E, 4, 4, COLS>), grid, block, lds, st, a, S);
  else if (A <= 128) hipLaunchKernelGGL((logprob_short_k<E, 4, 8, COLS>), grid, block, lds, st, a, S);
  else if (A <= 256) hipLaunchKernelGGL((logprob_short_k<E, 4, 16, COLS>), grid, block, lds, st, a, S);
  else if (A <= 512) hipLaunchKernelGGL((logprob_short_k<E, 6, 8, COLS>), grid, block, lds, st, a, S);
  else hipLaunchKernelGGL((logprob_short_k<E, 6, 16, COLS>), grid, block, lds, st, a, S);
}

template <class E>
hipError_t launch_top(const LogprobArgs& a, hipStream_t st) {
  const bool rows = a.l.stride_a == 1 || a.c.A == 1;
  if (rows && a.c.A <= kShort) {
    launch_short<E, false>(a, st);
  } else if (rows) {
    const int parts = parts_of(a.c.N, a.c.A);
    hipLaunchKernelGGL(logprob_long_k<E>, dim3(blocks_for(a.c.N, 1, 1 << 16), parts), dim3(kLong), 0, st, a);
    if (parts > 1) hipLaunchKernelGGL(logprob_join_k<E>, dim3((unsigned)a.c.N), dim3(kLong), 0, st, a, parts);
  } else if (a.c.A <= kTurned) {
    launch_short<E, true>(a, st);
  } else {
    const hipError_t e = launch_loss<LogprobOp>(a, 0, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(logprob_top_k<E>, dim3(blocks_for(a.c.N, 1, 1 << 20)), dim3(kTop), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace

size_t logprob_bytes(const sim_logprobs& c, bool grad) {
  const size_t split = (size_t)kMaxBlocks * 3 * sizeof(double) + kSplitMost * (sizeof(Part) + sizeof(float));
  if (grad || c.top == 0) return split;
  const int parts = c.A > kShort ? parts_of(c.N, c.A) : 1;
  return std::max(split, parts > 1 ? (size_t)c.N * parts * sizeof(LongPart) : 0);
}

hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t st) {
  if (!a.top_index && !a.top_logp) return launch_loss<LogprobOp>(a, 0, st);
  return a.c.dtype == SIM_DT_F32 ? launch_top<F32>(a, st) : a.c.dtype == SIM_DT_BF16 ? launch_top<BF16>(a, st) : launch_top<F16>(a, st);
}

}  // namespace bsim
