// ortho_kernels.hip -- updates orthogonalised by Newton-Schulz products.
//
// X = U / (|U|_F + eps) with its shorter side as rows (U^T for more rows than columns: the polynomial is odd,
// so it commutes with transposing), then A = X X^T, B = b A + c A A, X = a X + B X: three products a step, of which the first
// two are symmetric, so only the tiles on and below the diagonal are formed and written twice.
//
// Operands are fp16 parts of the value times 2^10: one part (11 bits) where the result is bf16 and rounded to 8 bits
// anyway, two (22 bits) otherwise, of which the product of the two second ones, below 2^-22 of the term, is left out. Every
// singular value of X stays below about 1.2 with the usual coefficients, so elements lie within fp16's range with room for 60,
// and the elements of a 65536 x 65536 update, 2^-16 of its norm, are still normal numbers. Sums are fp32.
#include <algorithm>

#include "ops_dev.hpp"

namespace bsim {
namespace {

typedef _Float16 H8 __attribute__((ext_vector_type(8)));
typedef _Float16 H4 __attribute__((ext_vector_type(4)));
typedef float F16x __attribute__((ext_vector_type(16)));

constexpr float kUp = 1024.0f, kDown = 1.0f / 1024.0f;   // of what is held

// Matrices in the work memory: X of r x c, A and B of r x r, all padded with zeros to R and C, multiples of a tile.
struct OrthoDims {
  int n, r, c, R, C;
  bool turned;   // U's columns are X's rows
};
struct Layout {
  OrthoDims d;
  int tile, parts;
  size_t x, a;                 // elements of a part of one matrix
  size_t sums, x0, x1, A, B, bytes;   // offsets in bytes
};
constexpr int kNorm = 256, kNormParts = 64, kFill = 256;
int round_up(int v, int to) { return (v + to - 1) / to * to; }
Layout layout_of(const sim_ortho& o) {
  Layout l;
  const bool t = o.M > o.N;
  l.d = OrthoDims{(int)o.n, (int)(t ? o.N : o.M), (int)(t ? o.M : o.N), 0, 0, t};
  const int64_t wide = (int64_t)l.d.n * ((l.d.r + 127) / 128) * ((l.d.c + 127) / 128);
  l.tile = wide >= kFill ? 128 : 64;
  l.parts = o.dtype == SIM_DT_BF16 ? 1 : 2;
  l.d.R = round_up(l.d.r, l.tile);
  l.d.C = round_up(l.d.c, l.tile);
  l.x = (size_t)l.d.R * l.d.C;
  l.a = (size_t)l.d.R * l.d.R;
  const size_t n = l.d.n, e = sizeof(_Float16) * l.parts;
  l.sums = 0;
  l.x0 = n * kNormParts * sizeof(double);
  l.x1 = l.x0 + n * l.x * e;
  l.A = l.x1 + n * l.x * e;
  l.B = l.A + n * l.a * e;
  l.bytes = l.B + n * l.a * e;
  return l;
}

// U as rows of its faster axis
struct View {
  int64_t si, slow, fast;
  int rows, cols;     // along them
  bool by_rows;       // the slow axis is U's rows
};
View view_of(const sim_mats& m, const sim_ortho& c) {
  const bool by_rows = m.stride_c <= m.stride_r;
  return by_rows ? View{m.stride_i, m.stride_r, m.stride_c, (int)c.M, (int)c.N, true}
                 : View{m.stride_i, m.stride_c, m.stride_r, (int)c.N, (int)c.M, false};
}

template <class E>
__global__ __launch_bounds__(kNorm) void ortho_norm_k(const void* u0, View v, double* part) {
  typedef typename E::T T;
  __shared__ double lds[kNorm / 64];
  const T* u = static_cast<const T*>(u0) + blockIdx.y * v.si;
  double s = 0.0;
  for (int i = blockIdx.x; i < v.rows; i += kNormParts) {
    const T* row = u + i * v.slow;
#pragma unroll 4
    for (int j = threadIdx.x; j < v.cols; j += kNorm) {
      const double x = (double)(float)row[j * v.fast];
      s = fma(x, x, s);
    }
  }
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.y * kNormParts + blockIdx.x] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__device__ __forceinline__ void split(float x, _Float16 (&p)[2]) {
  p[0] = (_Float16)x;
  p[1] = (_Float16)(x - (float)p[0]);
}
__device__ __forceinline__ void split(float x, _Float16 (&p)[1]) { p[0] = (_Float16)x; }

// X's parts, padding included: tiles of 64 x 64, read along U's faster axis and written along X's rows.
template <class E, int NP>
__global__ __launch_bounds__(256) void ortho_load_k(const void* u0, View v, OrthoDims d, const double* part, double eps,
                                                    _Float16* x) {
  typedef typename E::T T;
  __shared__ float t[64][65];
  const int tiles = d.C / 64, r0 = blockIdx.x / tiles * 64, c0 = blockIdx.x % tiles * 64;
  double s = 0.0;
  for (int p = 0; p < kNormParts; ++p) s += part[blockIdx.y * kNormParts + p];
  // an infinity or NaN makes NaN of the whole; of no update nothing is left, whatever eps
  const double f = s == 0.0 ? 0.0 : (s - s == 0.0 ? (double)kUp / (sqrt(s) + eps) : __longlong_as_double(0x7FF8000000000000ll));
  const T* u = static_cast<const T*>(u0) + blockIdx.y * v.si;
  const bool rows = v.by_rows != d.turned;   // X's rows lie along the slow axis
  for (int i = threadIdx.x; i < 64 * 64; i += 256) {
    const int a = i >> 6, b = i & 63, r = r0 + (rows ? a : b), c = c0 + (rows ? b : a);
    float w = 0.0f;
    if (r < d.r && c < d.c) w = (float)((double)(float)u[(rows ? r : c) * v.slow + (rows ? c : r) * v.fast] * f);
    t[rows ? a : b][rows ? b : a] = w;
  }
  __syncthreads();
  const size_t cells = (size_t)d.R * d.C;
  for (int i = threadIdx.x; i < 64 * 64; i += 256) {
    _Float16 p[NP];
    split(t[i >> 6][i & 63], p);
#pragma unroll
    for (int q = 0; q < NP; ++q)
      x[((size_t)blockIdx.y * NP + q) * cells + (size_t)(r0 + (i >> 6)) * d.C + c0 + (i & 63)] = p[q];
  }
}

// The result, in any strides.
struct Out {
  void* data;
  int64_t si, sr, sc;   // of X's rows and columns
  int dtype;
  float scale;
  __device__ __forceinline__ void put(int i, int r, int c, float held) const {
    const int64_t at = i * si + r * sr + c * sc;
    const float v = held * scale;
    if (dtype == SIM_DT_F32) static_cast<float*>(data)[at] = v;
    else if (dtype == SIM_DT_BF16) static_cast<__bf16*>(data)[at] = (__bf16)v;
    else static_cast<_Float16*>(data)[at] = (_Float16)v;
  }
};
template <int NP>
__global__ __launch_bounds__(256) void ortho_store_k(const _Float16* x, OrthoDims d, Out o) {   // no steps
  const int i = blockIdx.y, r = blockIdx.x;
  const size_t cells = (size_t)d.R * d.C;
  for (int c = threadIdx.x; c < d.c; c += 256) {
    float v = 0.0f;
#pragma unroll
    for (int q = NP - 1; q >= 0; --q) v += (float)x[((size_t)i * NP + q) * cells + (size_t)r * d.C + c];
    o.put(i, r, c, v);
  }
}

__device__ __forceinline__ H4 read_turned(const _Float16* p) {
  typedef short S4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) S4 L4;
  return __builtin_bit_cast(H4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((L4*)(p)));
}

// The three products, tiles of TM x TM by four waves, each TM/2 x TM/2 in tiles of 32:
//   kGram   out = P P^T             P = X, K = C
//   kPoly   out = b P + c P P^T     P = A (symmetric), K = R
//   kStep   out = a Q + P Q         P = B, Q = X [K][.], read turned from LDS
// K goes by BK; its next part is loaded into registers while the present one is multiplied, and goes to the other half of LDS.
// In LDS a row's chunks of 16 bytes are exchanged so that 16 rows at one place of K lie in different banks.
enum { kGram = 0, kPoly = 1, kStep = 2 };
struct Mul {
  const _Float16 *P, *Q;
  _Float16* out;
  size_t p, q, o;     // elements of a part
  int K, rows, cols;  // tiles of the result
  int ld;             // of out and Q
  float own, mul;     // the result is own * (P or Q) + mul * product, as it is held
  Out last;           // kStep: where the last step goes
  int r, c;
  bool end;
};
template <int NP, int TM, int KIND>
__global__ __launch_bounds__(256, 2) void ortho_mul_k(Mul m) {
  constexpr int BK = NP == 1 ? 64 : 32, CH = BK / 8, W = TM / 64, U = TM * BK / 8 / 256;
  constexpr int QC = TM / 8;   // chunks of a row of Q, turned
  __shared__ __align__(16) _Float16 ps[2][NP][TM * BK], qs[2][NP][TM * BK];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = (wave >> 1) * (TM / 2), wc = (wave & 1) * (TM / 2), l32 = lane & 31, half = lane >> 5;
  // neighbours of a run of tiles per XCD share their operands in its L2; runs go down bands of eight rows of tiles
  const int all = gridDim.x, xcd = blockIdx.x & 7, each = all >> 3, more = all & 7;
  int id = xcd * each + (xcd < more ? xcd : more) + (blockIdx.x >> 3);
  int ti, tj;
  if (KIND == kStep) {
    const int band = id / (8 * m.cols), in = id - band * 8 * m.cols, high = m.rows - band * 8 < 8 ? m.rows - band * 8 : 8;
    tj = in / high;
    ti = band * 8 + in % high;
  } else {
    ti = (int)((sqrtf(8.0f * id + 1.0f) - 1.0f) * 0.5f);
    while ((ti + 1) * (ti + 2) / 2 <= id) ++ti;
    while (ti * (ti + 1) / 2 > id) --ti;
    tj = id - ti * (ti + 1) / 2;
  }
  const int i = blockIdx.y, r0 = ti * TM, c0 = tj * TM, K = m.K;
  const _Float16* P = m.P + (size_t)i * NP * m.p + (size_t)r0 * K;
  const _Float16* Q = KIND == kStep ? m.Q + (size_t)i * NP * m.q + c0 : m.P + (size_t)i * NP * m.p + (size_t)c0 * K;
  H8 pr[NP][U], qr[NP][U];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int unit = threadIdx.x + u * 256, row = unit / CH, ch = unit % CH;
#pragma unroll
      for (int q = 0; q < NP; ++q) {
        pr[q][u] = *reinterpret_cast<const H8*>(P + q * m.p + (size_t)row * K + k0 + ch * 8);
        if (KIND == kStep) qr[q][u] = *reinterpret_cast<const H8*>(Q + q * m.q + (size_t)(k0 + unit / QC) * m.ld + unit % QC * 8);
        else qr[q][u] = *reinterpret_cast<const H8*>(Q + q * m.p + (size_t)row * K + k0 + ch * 8);
      }
    }
  };
  auto swap_p = [](int row, int ch) { return row * BK + ((ch ^ ((row / (16 / CH)) & (CH - 1))) * 8); };
  auto swap_q = [](int row, int ch) { return row * TM + ((ch ^ ((row & 3) << 2 & (QC - 1))) * 8); };
  auto store = [&](int to) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int unit = threadIdx.x + u * 256, at = swap_p(unit / CH, unit % CH);
#pragma unroll
      for (int q = 0; q < NP; ++q) {
        *reinterpret_cast<H8*>(&ps[to][q][at]) = pr[q][u];
        *reinterpret_cast<H8*>(&qs[to][q][KIND == kStep ? swap_q(unit / QC, unit % QC) : at]) = qr[q][u];
      }
    }
  };
  F16x acc[W][W];
#pragma unroll
  for (int x = 0; x < W; ++x) {
#pragma unroll
    for (int y = 0; y < W; ++y) acc[x][y] = F16x{};
  }
  auto multiply = [&](int from) {
#pragma unroll
    for (int kk = 0; kk < BK / 16; ++kk) {
      H8 a[W][NP], b[W][NP];
#pragma unroll
      for (int x = 0; x < W; ++x) {
#pragma unroll
        for (int q = 0; q < NP; ++q) {
          a[x][q] = *reinterpret_cast<const H8*>(&ps[from][q][swap_p(wr + 32 * x + l32, 2 * kk + half)]);
          if (KIND == kStep) {
            const int k = 16 * kk + 8 * half + ((lane & 15) >> 2), c = wc + 32 * x + (lane & 16) + 4 * (lane & 3);
            const H4 lo = read_turned(&qs[from][q][swap_q(k, c / 8) + (c & 7)]);
            const H4 hi = read_turned(&qs[from][q][swap_q(k + 4, c / 8) + (c & 7)]);
            b[x][q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          } else {
            b[x][q] = *reinterpret_cast<const H8*>(&qs[from][q][swap_p(wc + 32 * x + l32, 2 * kk + half)]);
          }
        }
      }
#pragma unroll
      for (int p = 0; p < NP; ++p) {
#pragma unroll
        for (int q = 0; q + p < NP; ++q) {
#pragma unroll
          for (int x = 0; x < W; ++x) {
#pragma unroll
            for (int y = 0; y < W; ++y)
              acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[x][p], b[y][q], acc[x][y], 0, 0, 0);
          }
        }
      }
    }
  };
  fetch(0);
  store(0);
  __syncthreads();
  int use = 0;
  for (int k0 = 0; k0 < K; k0 += BK) {
    if (k0 + BK < K) fetch(k0 + BK);
    multiply(use);
    if (k0 + BK < K) store(use ^ 1);
    __syncthreads();
    use ^= 1;
  }
  // lane: column l32 of a tile, rows 8 (e / 4) + 4 half + e % 4
  const _Float16* own = KIND == kStep ? m.Q + (size_t)i * NP * m.q : m.P + (size_t)i * NP * m.p;
  const size_t own_part = KIND == kStep ? m.q : m.p;
  _Float16* out = m.out + (size_t)i * NP * m.o;
#pragma unroll
  for (int x = 0; x < W; ++x) {
#pragma unroll
    for (int y = 0; y < W; ++y) {
      const int c = c0 + wc + 32 * y + l32;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int r = r0 + wr + 32 * x + 8 * g + 4 * half;
        H4 keep[NP];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const size_t at = (size_t)(r + e) * m.ld + c;
          float v = acc[x][y][4 * g + e] * m.mul;
          if (KIND != kGram) {
            float w = 0.0f;
#pragma unroll
            for (int q = NP - 1; q >= 0; --q) w += (float)own[q * own_part + at];
            v = fmaf(m.own, w, v);
          }
          if (KIND == kStep && m.end) {
            if (r + e < m.r && c < m.c) m.last.put(i, r + e, c, v);
            continue;
          }
          _Float16 p[NP];
          split(v, p);
#pragma unroll
          for (int q = 0; q < NP; ++q) {
            out[q * m.o + at] = p[q];
            keep[q][e] = p[q];
          }
        }
        if (KIND != kStep && ti != tj) {
#pragma unroll
          for (int q = 0; q < NP; ++q) *reinterpret_cast<H4*>(&out[q * m.o + (size_t)c * m.ld + r]) = keep[q];
        }
      }
    }
  }
}

template <int NP, int TM>
void steps_of(const OrthoArgs& a, const Layout& l, const Out& last, hipStream_t st) {
  char* w = static_cast<char*>(a.work);
  _Float16 *x = reinterpret_cast<_Float16*>(w + l.x0), *y = reinterpret_cast<_Float16*>(w + l.x1);
  _Float16 *A = reinterpret_cast<_Float16*>(w + l.A), *B = reinterpret_cast<_Float16*>(w + l.B);
  const int tr = l.d.R / TM, tc = l.d.C / TM;
  const unsigned n = (unsigned)l.d.n;
  const dim3 half((unsigned)((int64_t)tr * (tr + 1) / 2), n), whole((unsigned)((int64_t)tr * tc), n), block(256);
  for (int i = 0; i < a.c.steps; ++i) {
    Mul m{};
    m.P = x; m.p = l.x; m.out = A; m.o = l.a; m.K = l.d.C; m.ld = l.d.R; m.mul = kDown;
    hipLaunchKernelGGL((ortho_mul_k<NP, TM, kGram>), half, block, 0, st, m);
    m.P = A; m.p = l.a; m.out = B; m.K = l.d.R; m.own = a.c.b; m.mul = a.c.c * kDown;
    hipLaunchKernelGGL((ortho_mul_k<NP, TM, kPoly>), half, block, 0, st, m);
    m.P = B; m.Q = x; m.q = l.x; m.out = y; m.o = l.x; m.ld = l.d.C; m.own = a.c.a; m.mul = kDown;
    m.rows = tr; m.cols = tc; m.r = l.d.r; m.c = l.d.c; m.last = last; m.end = i + 1 == a.c.steps;
    hipLaunchKernelGGL((ortho_mul_k<NP, TM, kStep>), whole, block, 0, st, m);
    std::swap(x, y);
  }
}

template <class E, int NP>
void launch_typed(const OrthoArgs& a, hipStream_t st) {
  const Layout l = layout_of(a.c);
  char* w = static_cast<char*>(a.work);
  double* sums = reinterpret_cast<double*>(w + l.sums);
  _Float16* x = reinterpret_cast<_Float16*>(w + l.x0);
  const unsigned n = (unsigned)l.d.n;
  const View v = view_of(a.u, a.c);
  const Out out{a.out.data, a.out.stride_i, l.d.turned ? a.out.stride_c : a.out.stride_r,
                l.d.turned ? a.out.stride_r : a.out.stride_c, a.c.dtype, a.c.scale * kDown};
  hipLaunchKernelGGL(ortho_norm_k<E>, dim3(kNormParts, n), dim3(kNorm), 0, st, a.u.data, v, sums);
  hipLaunchKernelGGL((ortho_load_k<E, NP>), dim3((unsigned)((int64_t)(l.d.R / 64) * (l.d.C / 64)), n), dim3(256), 0, st, a.u.data, v,
                     l.d, sums, (double)a.c.eps, x);
  if (a.c.steps == 0) hipLaunchKernelGGL(ortho_store_k<NP>, dim3(l.d.r, n), dim3(256), 0, st, x, l.d, out);
  else if (l.tile == 128) steps_of<NP, 128>(a, l, out, st);
  else steps_of<NP, 64>(a, l, out, st);
}

}  // namespace

size_t ortho_bytes(const sim_ortho& c) { return c.n && c.M && c.N ? layout_of(c).bytes : 0; }

hipError_t launch_ortho(const OrthoArgs& a, hipStream_t st) {
  if (a.c.dtype == SIM_DT_F32) launch_typed<F32, 2>(a, st);
  else if (a.c.dtype == SIM_DT_BF16) launch_typed<BF16, 1>(a, st);
  else launch_typed<F16, 2>(a, st);
  return hipGetLastError();
}

}  // namespace bsim
