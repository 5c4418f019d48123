// linattn_kernels.hip -- linear attention with a decay for each head, and its gradient.
//
// One run computes, per sequence and head, over its live steps in either direction, from a state S,
//   out_i = so sum_{j<=i} l^(i-j) (q_i k_j) su v_j + so l^(i+1-lag) q_i S,   S' = l^n S + su sum_j l^(n-1-j+lag) k_j v_j^T.
// The operator is the run of (q, k, v) with so = scale. Its gradient is three more, lag = 1 where the state
// is the gradient of the state behind a step (which that step's own product still joins undecayed):
//   dq  (dy, v, k) forwards from S0^T, so = scale
//   dk  (v, dy, q) backwards from dS^T, su = scale, lag = 1
//   dv  (k, q, dy) backwards from dS, su = scale, lag = 1, whose last state is dS0
#include <algorithm>

#include "ops_dev.hpp"

namespace bsim {
namespace {

struct In {
  const void* p;
  int64_t sb, st, sh;
  int share;   // heads that share one of this array's
};
struct AttnRun {
  In q, k, v;
  void* out;            // null: only the state is wanted
  int64_t ob, ot, oh;
  const float *s0, *decay;
  float* state;         // null: not wanted
  int64_t sr, sc;       // strides of a state's rows (q's channels) and columns (v's)
  const int32_t* len;
  uint32_t* err;        // null: another run tells
  int64_t T;
  int H, Dq, Dv, lag;
  bool back, wide;      // steps from the last to the first; out in fp32
  float so, su;
};

__device__ __forceinline__ float decay_of(const AttnRun& r, int h) {
  float l = r.decay[h];
  if (!(l >= 0.0f && l <= 1.0f)) {
    if (r.err && threadIdx.x == 0) atomicOr(r.err, ERR_DECAY);
    l = l > 1.0f ? 1.0f : 0.0f;
  }
  return l;
}
__device__ __forceinline__ int64_t steps_of(const AttnRun& r, int b) {
  int64_t n = r.T;
  if (r.len) {
    n = r.len[b];
    if (n < 0 || n > r.T) {
      if (r.err && threadIdx.x == 0) atomicOr(r.err, ERR_LENGTH);
      n = n < 0 ? 0 : r.T;
    }
  }
  return n;
}
template <class T>
__device__ __forceinline__ const T* row_of(const In& x, int b, int64_t t, int h) {
  return static_cast<const T*>(x.p) + b * x.sb + t * x.st + (h / x.share) * x.sh;
}

// One step after another: 64 columns of a state, in registers, 16 rows apart by 16 rows a thread. Bound by
// reading and writing the state where there are many, by a step's chain otherwise.
constexpr int kStep = 256;
template <class E, int R>
__global__ __launch_bounds__(kStep) void attn_step_k(AttnRun r) {
  typedef typename E::T T;
  __shared__ float ql[R * 16], kl[R * 16], vl[64], red[4][64];
  const int h = blockIdx.x % r.H, b = blockIdx.x / r.H, c0 = blockIdx.y * 64;
  const int rg = threadIdx.x >> 4, c = c0 + (threadIdx.x & 15) * 4;
  const float l = decay_of(r, h);
  const int64_t n = steps_of(r, b), base = (int64_t)blockIdx.x * r.Dq * r.Dv;
  float s[R][4];
  const bool quad = r.sc == 1 && (r.Dv & 3) == 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = rg + 16 * i;
#pragma unroll
    for (int u = 0; u < 4; ++u) s[i][u] = 0.0f;
    if (!r.s0 || row >= r.Dq || c >= r.Dv) continue;
    const float* p = r.s0 + base + row * r.sr + c * r.sc;
    if (quad) {
      typedef float Raw __attribute__((ext_vector_type(4), aligned(4)));
      const Raw w = *reinterpret_cast<const Raw*>(p);
#pragma unroll
      for (int u = 0; u < 4; ++u) s[i][u] = w[u];
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (c + u < r.Dv) s[i][u] = p[u * r.sc];
    }
  }
  for (int64_t i = 0; i < n; ++i) {
    const int64_t t = r.back ? n - 1 - i : i;
    if (threadIdx.x < R * 16) {
      const int j = threadIdx.x;
      ql[j] = r.out && j < r.Dq ? (float)row_of<T>(r.q, b, t, h)[j] : 0.0f;
      kl[j] = j < r.Dq ? (float)row_of<T>(r.k, b, t, h)[j] : 0.0f;
    }
    if (threadIdx.x >= kStep - 64) {
      const int j = threadIdx.x - (kStep - 64);
      vl[j] = c0 + j < r.Dv ? (float)row_of<T>(r.v, b, t, h)[c0 + j] * r.su : 0.0f;
    }
    __syncthreads();
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const float before = r.lag ? 1.0f : l, after = r.lag ? l : 1.0f;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const float kk = kl[rg + 16 * k], qq = ql[rg + 16 * k];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float w = fmaf(kk, vl[(threadIdx.x & 15) * 4 + u], before * s[k][u]);
        acc[u] = fmaf(qq, w, acc[u]);
        s[k][u] = after * w;
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      acc[u] += __shfl_xor(acc[u], 16);
      acc[u] += __shfl_xor(acc[u], 32);
    }
    if ((threadIdx.x & 48) == 0) {
#pragma unroll
      for (int u = 0; u < 4; ++u) red[threadIdx.x >> 6][(threadIdx.x & 15) * 4 + u] = acc[u];
    }
    __syncthreads();
    if (r.out && threadIdx.x < 64 && c0 + threadIdx.x < r.Dv) {
      const int j = threadIdx.x;
      const float y = ((red[0][j] + red[1][j]) + (red[2][j] + red[3][j])) * r.so;
      const int64_t at = b * r.ob + t * r.ot + h * r.oh + c0 + j;
      if (r.wide) static_cast<float*>(r.out)[at] = y;
      else static_cast<T*>(r.out)[at] = (T)y;
    }
  }
  if (r.out) {   // padding
    const int64_t cells = (r.T - n) * 64;
    for (int64_t i = threadIdx.x; i < cells; i += kStep) {
      const int j = (int)(i & 63);
      const int64_t at = b * r.ob + (n + (i >> 6)) * r.ot + h * r.oh + c0 + j;
      if (c0 + j >= r.Dv) continue;
      if (r.wide) static_cast<float*>(r.out)[at] = 0.0f;
      else static_cast<T*>(r.out)[at] = (T)0.0f;
    }
  }
  if (!r.state) return;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = rg + 16 * i;
    if (row >= r.Dq || c >= r.Dv) continue;
    float* p = r.state + base + row * r.sr + c * r.sc;
    if (quad) {
      typedef float Raw __attribute__((ext_vector_type(4), aligned(4)));
      *reinterpret_cast<Raw*>(p) = Raw{s[i][0], s[i][1], s[i][2], s[i][3]};
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (c + u < r.Dv) p[u * r.sc] = s[i][u];
    }
  }
}

// Gradients of shared keys and values: the sum over the heads that share them, in order.
template <class E>
__global__ __launch_bounds__(256) void attn_share_k(const float* w, sim_heads o, int64_t cells, int64_t T, int Hk,
                                                    int g, int D) {
  typedef typename E::T T_;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < cells; i += (int64_t)gridDim.x * 256) {
    const int d = (int)(i % D);
    const int64_t bth = i / D, h = bth % Hk, bt = bth / Hk, t = bt % T, b = bt / T;
    float v = 0.0f;
    for (int j = 0; j < g; ++j) v += w[(bth * g + j) * D + d];
    static_cast<T_*>(o.data)[b * o.stride_b + t * o.stride_t + h * o.stride_h + d] = (T_)v;
  }
}

template <class E>
void launch_run(const AttnRun& r, int64_t B, hipStream_t st) {
  const dim3 grid((unsigned)(B * r.H), (r.Dv + 63) / 64), block(kStep);
  if (r.Dq <= 64) hipLaunchKernelGGL((attn_step_k<E, 4>), grid, block, 0, st, r);
  else if (r.Dq <= 128) hipLaunchKernelGGL((attn_step_k<E, 8>), grid, block, 0, st, r);
  else hipLaunchKernelGGL((attn_step_k<E, 16>), grid, block, 0, st, r);
}

In in_of(const sim_heads& x, int share) { return In{x.data, x.stride_b, x.stride_t, x.stride_h, share}; }

template <class E>
void launch_typed(const AttnArgs& a, bool grad, hipStream_t st) {
  const sim_linear_attn& c = a.c;
  const int g = c.H / c.Hk;
  AttnRun f{};
  f.decay = a.decay; f.len = a.len; f.err = a.err; f.T = c.T; f.H = c.H;
  const In q = in_of(a.q, 1), k = in_of(a.k, g), v = in_of(a.v, g), dy = in_of(a.dy, 1);
  auto dims = [&](AttnRun& r, int Dq, int Dv, bool turned) {   // turned: states are [Dv][Dq] in memory
    r.Dq = Dq; r.Dv = Dv;
    r.sr = turned ? 1 : Dv; r.sc = turned ? Dq : 1;
  };
  auto out = [&](AttnRun& r, const sim_heads& o) {
    r.out = o.data; r.ob = o.stride_b; r.ot = o.stride_t; r.oh = o.stride_h;
  };
  if (!grad) {
    AttnRun r = f;
    r.q = q; r.k = k; r.v = v;
    dims(r, c.Dk, c.Dv, false);
    out(r, a.y);
    r.s0 = a.s0; r.state = a.state; r.so = c.scale; r.su = 1.0f;
    launch_run<E>(r, c.B, st);
    return;
  }
  // each told by the first run there is
  if (a.dq.data) {
    AttnRun r = f;
    r.q = dy; r.k = v; r.v = k;
    dims(r, c.Dv, c.Dk, true);
    out(r, a.dq);
    r.s0 = a.s0; r.so = c.scale; r.su = 1.0f;
    launch_run<E>(r, c.B, st);
    f.err = nullptr;
  }
  f.back = true; f.lag = 1; f.so = 1.0f; f.su = c.scale;
  auto shared = [&](AttnRun& r, const sim_heads& o, int D) {
    if (g == 1 || !o.data) {
      out(r, o);
      launch_run<E>(r, c.B, st);
      return;
    }
    r.out = a.work; r.wide = true;
    r.oh = D; r.ot = (int64_t)c.H * D; r.ob = c.T * r.ot;
    launch_run<E>(r, c.B, st);
    const int64_t cells = c.B * c.T * c.Hk * D;
    if (cells)
      hipLaunchKernelGGL(attn_share_k<E>, dim3((unsigned)std::min<int64_t>((cells + 255) / 256, 1 << 16)), dim3(256), 0,
                         st, static_cast<const float*>(a.work), o, cells, c.T, c.Hk, g, D);
  };
  if (a.dk.data) {
    AttnRun r = f;
    r.q = v; r.k = dy; r.v = q;
    dims(r, c.Dv, c.Dk, true);
    r.s0 = a.ds;
    shared(r, a.dk, c.Dk);
    f.err = nullptr;
  }
  if (a.dv.data || a.state) {   // the last one: ds0 may be written over dstate
    AttnRun r = f;
    r.q = k; r.k = q; r.v = dy;
    dims(r, c.Dk, c.Dv, false);
    r.s0 = a.ds; r.state = a.state;
    shared(r, a.dv, c.Dv);
  }
}

}  // namespace

size_t attn_work_bytes(const sim_linear_attn& c, bool grad) {
  return grad && c.H > c.Hk ? (size_t)c.B * c.T * c.H * std::max(c.Dk, c.Dv) * sizeof(float) : 0;
}

hipError_t launch_attn(const AttnArgs& a, bool grad, hipStream_t st) {
  if (a.c.dtype == SIM_DT_F32) launch_typed<F32>(a, grad, st);
  else if (a.c.dtype == SIM_DT_BF16) launch_typed<BF16>(a, grad, st);
  else launch_typed<F16>(a, grad, st);
  return hipGetLastError();
}

}  // namespace bsim
