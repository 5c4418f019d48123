// ortho_kernels.hip -- updates orthogonalised by Newton-Schulz products.
//
// X = U / (|U|_F + eps) with its shorter side as rows (U^T for more rows than columns: the polynomial is odd,
// so it commutes with transposing), then A = X X^T, B = b A + c A A, X = a X + B X.
#include <algorithm>

#include "ops_dev.hpp"

namespace bsim {
namespace {

struct OrthoDims {
  int64_t n, r, c;
  bool turned;   // U's columns are X's rows
};
OrthoDims dims_of(const sim_ortho& o) {
  const bool t = o.M > o.N;
  return OrthoDims{o.n, t ? o.N : o.M, t ? o.M : o.N, t};
}

constexpr int kNorm = 256, kNormParts = 64;
template <class E>
__global__ __launch_bounds__(kNorm) void ortho_norm_k(OrthoArgs a, double* part) {
  typedef typename E::T T;
  __shared__ double lds[kNorm / 64];
  const int64_t cells = a.c.M * a.c.N;
  const T* u = static_cast<const T*>(a.u.data) + blockIdx.y * a.u.stride_i;
  double s = 0.0;
  for (int64_t i = blockIdx.x * kNorm + threadIdx.x; i < cells; i += kNormParts * kNorm) {
    const double v = (double)(float)u[i / a.c.N * a.u.stride_r + i % a.c.N * a.u.stride_c];
    s = fma(v, v, s);
  }
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.y * kNormParts + blockIdx.x] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <class E>
__global__ __launch_bounds__(256) void ortho_load_k(OrthoArgs a, OrthoDims d, const double* part, float* x) {
  typedef typename E::T T;
  const int64_t i = blockIdx.y, cells = d.r * d.c;
  double s = 0.0;
  for (int p = 0; p < kNormParts; ++p) s += part[i * kNormParts + p];
  const float f = (float)(1.0 / (sqrt(s) + (double)a.c.eps));
  const T* u = static_cast<const T*>(a.u.data) + i * a.u.stride_i;
  const int64_t sr = d.turned ? a.u.stride_c : a.u.stride_r, sc = d.turned ? a.u.stride_r : a.u.stride_c;
  for (int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x; j < cells; j += (int64_t)gridDim.x * 256)
    x[i * cells + j] = s == 0.0 ? 0.0f : (float)u[j / d.c * sr + j % d.c * sc] * f;
}

// out [R][C] = f1 P [R][K] Q + f2 D, Q [K][C] or, TR, [C][K]; D has out's layout
template <bool TR>
__global__ __launch_bounds__(256) void ortho_mul_k(const float* P, const float* Q, const float* D, float* out, int64_t R,
                                                   int64_t C, int64_t K, float f1, float f2, int64_t sp, int64_t sq) {
  __shared__ float p[16][17], q[16][17];
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const int64_t tiles = (C + 15) / 16, all = tiles * ((R + 15) / 16);
  P += blockIdx.y * sp;
  Q += blockIdx.y * sq;
  for (int64_t tile = blockIdx.x; tile < all; tile += gridDim.x) {
  const int64_t r0 = tile / tiles * 16, c0 = tile % tiles * 16;
  float s = 0.0f;
  for (int64_t k0 = 0; k0 < K; k0 += 16) {
    p[ty][tx] = r0 + ty < R && k0 + tx < K ? P[(r0 + ty) * K + k0 + tx] : 0.0f;
    if (TR) q[tx][ty] = c0 + ty < C && k0 + tx < K ? Q[(c0 + ty) * K + k0 + tx] : 0.0f;
    else q[ty][tx] = k0 + ty < K && c0 + tx < C ? Q[(k0 + ty) * C + c0 + tx] : 0.0f;
    __syncthreads();
    for (int k = 0; k < 16; ++k) s = fmaf(p[ty][k], q[k][tx], s);
    __syncthreads();
  }
  if (r0 + ty < R && c0 + tx < C) {
    const int64_t at = blockIdx.y * R * C + (r0 + ty) * C + c0 + tx;
    out[at] = D ? fmaf(f2, D[at], f1 * s) : f1 * s;
  }
  }
}

template <class E>
__global__ __launch_bounds__(256) void ortho_store_k(OrthoArgs a, OrthoDims d, const float* x) {
  typedef typename E::T T;
  const int64_t i = blockIdx.y, cells = d.r * d.c;
  T* o = static_cast<T*>(a.out.data) + i * a.out.stride_i;
  for (int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x; j < cells; j += (int64_t)gridDim.x * 256) {
    const int64_t m = j / a.c.N, n = j % a.c.N;
    o[m * a.out.stride_r + n * a.out.stride_c] = (T)(a.c.scale * x[i * cells + (d.turned ? n * d.c + m : j)]);
  }
}

template <class E>
void launch_typed(const OrthoArgs& a, hipStream_t st) {
  const OrthoDims d = dims_of(a.c);
  double* part = static_cast<double*>(a.work);
  float* x = reinterpret_cast<float*>(part + d.n * kNormParts);
  float* x2 = x + d.n * d.r * d.c;
  float* A = x2 + d.n * d.r * d.c;
  float* B = A + d.n * d.r * d.r;
  const unsigned n = (unsigned)d.n;
  const unsigned flat = (unsigned)std::min<int64_t>((d.r * d.c + 255) / 256, 4096);
  const int64_t tr = (d.r + 15) / 16, tc = (d.c + 15) / 16;
  hipLaunchKernelGGL(ortho_norm_k<E>, dim3(kNormParts, n), dim3(kNorm), 0, st, a, part);
  hipLaunchKernelGGL(ortho_load_k<E>, dim3(flat, n), dim3(256), 0, st, a, d, part, x);
  for (int i = 0; i < a.c.steps; ++i) {
    hipLaunchKernelGGL(ortho_mul_k<true>, dim3((unsigned)std::min<int64_t>(tr * tr, 1 << 20), n), dim3(256), 0, st, x, x, nullptr, A, d.r, d.r, d.c,
                       1.0f, 0.0f, d.r * d.c, d.r * d.c);
    hipLaunchKernelGGL(ortho_mul_k<true>, dim3((unsigned)std::min<int64_t>(tr * tr, 1 << 20), n), dim3(256), 0, st, A, A, A, B, d.r, d.r, d.r,
                       a.c.c, a.c.b, d.r * d.r, d.r * d.r);
    hipLaunchKernelGGL(ortho_mul_k<false>, dim3((unsigned)std::min<int64_t>(tr * tc, 1 << 20), n), dim3(256), 0, st, B, x, x, x2, d.r, d.c, d.r,
                       1.0f, a.c.a, d.r * d.r, d.r * d.c);
    std::swap(x, x2);
  }
  hipLaunchKernelGGL(ortho_store_k<E>, dim3(flat, n), dim3(256), 0, st, a, d, x);
}

}  // namespace

size_t ortho_bytes(const sim_ortho& c) {
  const OrthoDims d = dims_of(c);
  return (size_t)d.n * (kNormParts * sizeof(double) + 2 * (d.r * d.c + d.r * d.r) * sizeof(float));
}

hipError_t launch_ortho(const OrthoArgs& a, hipStream_t st) {
  if (a.c.dtype == SIM_DT_F32) launch_typed<F32>(a, st);
  else if (a.c.dtype == SIM_DT_BF16) launch_typed<BF16>(a, st);
  else launch_typed<F16>(a, st);
  return hipGetLastError();
}

}  // namespace bsim
