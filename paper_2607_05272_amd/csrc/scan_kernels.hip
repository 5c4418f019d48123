// scan_kernels.hip -- the gated linear recurrence and its gradient over [B][T][D].
//
//   linear   h = g_t h + x_t,        sigmoid  f = 1/(1 + exp(-g_t)), h = f h + (1 - f) x_t
//
// One multiplication and one addition per element over two reads and a write: bound by HBM.
// Positions p = 0..T-1 are taken in processing order, t = p or T-1-p; padding is the
// identity, so the state passes through it on either side of a sequence.
#include "ops_dev.hpp"

namespace bsim {
namespace {

// a step's gate and the factor of its input: h = a h + r x
template <class W, bool SIG>
__device__ __forceinline__ void gate_of(W g, W& a, W& r) {
  if (SIG) {
    sigmoid_pair(g, a, r);
  } else {
    a = g;
    r = (W)1;
  }
}

__device__ __forceinline__ int64_t seq_len(const ScanArgs& s, int64_t b, bool tell) {
  if (!s.len) return s.c.T;
  int64_t n = s.len[b];
  if (n < 0 || n > s.c.T) {
    if (tell) atomicOr(s.err, ERR_LENGTH);
    n = n < 0 ? 0 : s.c.T;
  }
  return n;
}

// One lane per channel, step after step.
template <class E, bool SIG>
__global__ __launch_bounds__(256) void scan_step_k(ScanArgs s) {
  typedef typename E::T T;
  typedef typename E::W W;
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= s.c.B * s.c.D) return;
  const int64_t b = c / s.c.D, d = c % s.c.D, n = seq_len(s, b, d == 0);
  const T* g = static_cast<const T*>(s.g.data) + b * s.g.stride_b + d;
  const T* x = static_cast<const T*>(s.x.data) + b * s.x.stride_b + d;
  T* y = static_cast<T*>(s.y.data) + b * s.y.stride_b + d;
  W h = s.h0 ? static_cast<const W*>(s.h0)[c] : (W)0;
  for (int64_t p = 0; p < s.c.T; ++p) {
    const int64_t t = s.c.reverse ? s.c.T - 1 - p : p;
    W out = (W)0;
    if (t < n) {
      W a, r;
      gate_of<W, SIG>((W)g[t * s.g.stride_t], a, r);
      h = a * h + r * (W)x[t * s.x.stride_t];
      out = h;
    }
    if (s.y.data) y[t * s.y.stride_t] = (T)out;
  }
  if (s.state) static_cast<W*>(s.state)[c] = h;
}

template <class E, bool SIG>
__global__ __launch_bounds__(256) void scan_step_grad_k(ScanArgs s) {
  typedef typename E::T T;
  typedef typename E::W W;
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= s.c.B * s.c.D) return;
  const int64_t b = c / s.c.D, d = c % s.c.D, n = seq_len(s, b, d == 0);
  const T* g = static_cast<const T*>(s.g.data) + b * s.g.stride_b + d;
  const T* x = static_cast<const T*>(s.x.data) + b * s.x.stride_b + d;
  const T* y = static_cast<const T*>(s.y.data) + b * s.y.stride_b + d;
  const T* dy = static_cast<const T*>(s.dy.data) + b * s.dy.stride_b + d;
  T* dg = static_cast<T*>(s.dg.data) + b * s.dg.stride_b + d;
  T* dx = static_cast<T*>(s.dx.data) + b * s.dx.stride_b + d;
  const W h0 = s.h0 ? static_cast<const W*>(s.h0)[c] : (W)0;
  W C = s.ds ? static_cast<const W*>(s.ds)[c] : (W)0;
  for (int64_t p = s.c.T - 1; p >= 0; --p) {
    const int64_t t = s.c.reverse ? s.c.T - 1 - p : p, tp = s.c.reverse ? t + 1 : t - 1;
    W og = (W)0, ox = (W)0;
    if (t < n) {
      W a, r;
      gate_of<W, SIG>((W)g[t * s.g.stride_t], a, r);
      const W G = (W)dy[t * s.dy.stride_t] + C;
      ox = r * G;
      C = a * G;
      if (s.dg.data) {
        const W hp = tp >= 0 && tp < n ? (W)y[tp * s.y.stride_t] : h0;
        og = SIG ? G * (hp - (W)x[t * s.x.stride_t]) * a * r : G * hp;
      }
    }
    if (s.dg.data) dg[t * s.dg.stride_t] = (T)og;
    if (s.dx.data) dx[t * s.dx.stride_t] = (T)ox;
  }
  if (s.state) static_cast<W*>(s.state)[c] = C;
}

template <class E, bool SIG>
hipError_t go(const ScanArgs& a, bool grad, hipStream_t st) {
  const unsigned nb = (unsigned)((a.c.B * a.c.D + 255) / 256);
  if (grad) hipLaunchKernelGGL((scan_step_grad_k<E, SIG>), dim3(nb), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((scan_step_k<E, SIG>), dim3(nb), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <class E>
hipError_t go(const ScanArgs& a, bool grad, hipStream_t st) {
  return a.c.kind == SIM_GATE_SIGMOID ? go<E, true>(a, grad, st) : go<E, false>(a, grad, st);
}

}  // namespace

size_t scan_work_bytes(const sim_scan&, bool) { return 0; }

hipError_t launch_scan(const ScanArgs& a, bool grad, hipStream_t st) {
  switch (a.c.dtype) {
    case SIM_DT_F64: return go<F64>(a, grad, st);
    case SIM_DT_F32: return go<F32>(a, grad, st);
    case SIM_DT_BF16: return go<BF16>(a, grad, st);
    default: return go<F16>(a, grad, st);
  }
}

}  // namespace bsim
