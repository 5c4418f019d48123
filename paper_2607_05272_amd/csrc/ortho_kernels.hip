// ortho_kernels.hip -- updates orthogonalised by Newton-Schulz products.
//
// X = U / (|U|_F + eps) with its shorter side as rows (U^T for more rows than columns: the polynomial is odd,
// so it commutes with transposing), then A = X X^T, B = b A + c A A, X = a X + B X: three products a step, of which the first
// two are symmetric, so only the tiles on and below the diagonal are formed and written twice.
//
// Operands are two fp16 parts (22 bits) of the value times 2^10; the product of two second parts, below 2^-22 of the term,
// is left out. One part (11 bits) would not do for bf16 either: the steps multiply what lies outside of the directions of an
// update of low rank by up to 3.4445^5 = 485, the rounding of X too (512 x 1365 bf16, error of the result before its own
// rounding of 1.7e-3: rank 1 9.7e-2 with one part, 2.4e-5 with two; rank 32 2.8e-2, 6.7e-6; random 1.4e-3, 3.4e-7). Every
// singular value of X stays below about 1.2 with the usual coefficients, so elements lie within fp16's range with room for 60,
// and the elements of a 65536 x 65536 update, 2^-16 of its norm, are still normal numbers. Sums are fp32.
#include <algorithm>
#include <atomic>

#include "ops_dev.hpp"

namespace bsim {
namespace {

typedef _Float16 H8 __attribute__((ext_vector_type(8)));
typedef _Float16 H4 __attribute__((ext_vector_type(4)));
typedef float Fl4 __attribute__((ext_vector_type(4)));
typedef float F16x __attribute__((ext_vector_type(16)));

constexpr float kUp = 1024.0f, kDown = 1.0f / 1024.0f;   // of what is held
constexpr int kParts = 2;

// Matrices in the work memory: X of r x c, A and B of r x r, all padded with zeros to R and C, multiples of a tile.
struct OrthoDims {
  int n, r, c, R, C;
  bool turned;   // U's columns are X's rows
};
struct Layout {
  OrthoDims d;
  int half, whole;             // tiles of the symmetric products and of X
  int sums_n;                  // workgroups that add up squares of a matrix
  size_t x, a;                 // elements of a part of one matrix
  size_t sums, x0, x1, A, B, parts_at, bytes;   // offsets in bytes
  int split;                   // parts of X X^T's sum over K, each by workgroups of its own
};
constexpr int kNorm = 256, kFillTiles = 512, kShare = 512;
int round_up(int v, int to) { return (v + to - 1) / to * to; }
// Tiles of X: of 256 where there are enough for the CUs (one takes a CU) and K is long, of 128 where they fill half of the chip's
// places, and padding adds little; of the symmetric products larger than 64 where the rows are many and the products long. The
// numbers lie between the sizes that were measured (us, tiles of the symmetric products / of X; * the rule's, up to 8% behind
// the best; any type, held and multiplied alike):
//                     64/64   64/128  128/128  64/256  128/256  256/256
//   4096 x 8192       10829     9367     8592    8789     8025    7108*
//   2048 x 8192        2676     2352     2057    2219     1924*   2539
//   1536 x 6144        1214     1230     1212    1169*    1141    1522
//   8 x 1024 x 4096    2648     2263     2255    2159     2175*   2368
//   3000 x 3000        2645     2701     2544    2544     2382*   2807
//   3 x 1500 x 1500    1260     1093     1063*   1296     1268    1649
//   2 x 2048 x 2048    1627     1436     1452*   1610     1625    2046
//   2048 x 3000        1197     1151     1091*   1394     1333    1795
//   8 x 1024 x 1024     865      766*     807     874      913    1144
//   4 x 1024 x 1024     504      500*     556     720      776    1122
//   6 x 768 x 2048      762      743*     832     715      803    1079
//   8 x 700 x 1500      636*     689      719     674      702     974
//   100 x 512 x 512    1891     1741*    1688    1690     1615    1988
//   12 x 1365 x 512     527      533*     610     536      655     915
//   4 x 256 x 256       102*     139      209     241      308     444
void pick_tiles(int64_t n, int64_t r, int64_t c, int* half, int* whole) {
  auto up = [](int64_t v, int64_t t) { return (v + t - 1) / t; };
  auto tiles = [&](int64_t t) { return n * up(r, t) * up(c, t); };
  auto below = [&](int64_t t) { return n * up(r, t) * (up(r, t) + 1) / 2; };   // on and below the diagonal
  auto close = [&](int64_t t) { return 16 * tiles(t) * t * t <= 17 * tiles(64) * 64 * 64; };
  *whole = r >= 1024 && tiles(256) >= 140 && close(256) ? 256 : (tiles(128) >= 256 && close(128) ? 128 : 64);
  *half = *whole == 256 && r >= 2048 && below(256) >= 128              ? 256
          : *whole >= 128 && r >= 1024 && below(128) * (r + c) >= 640000 ? 128 : 64;
}
Layout layout_of(const sim_ortho& o) {
  Layout l;
  const bool t = o.M > o.N;
  l.d = OrthoDims{(int)o.n, (int)(t ? o.N : o.M), (int)(t ? o.M : o.N), 0, 0, t};
  const int64_t r = l.d.r, c = l.d.c, n = l.d.n;
  pick_tiles(n, r, c, &l.half, &l.whole);
  l.d.R = round_up(l.d.r, std::max(l.half, l.whole));
  l.d.C = round_up(l.d.c, l.whole);
  l.x = (size_t)l.d.R * l.d.C;
  l.a = (size_t)l.d.R * l.d.R;
  const size_t e = sizeof(_Float16) * kParts;
  l.sums = 0;
  l.sums_n = (int)std::max<int64_t>(1, std::min<int64_t>({std::max(o.M, o.N), 1024, (2048 + n - 1) / n}));
  l.x0 = (n * l.sums_n * sizeof(double) + 15) / 16 * 16;
  l.x1 = l.x0 + n * l.x * e;
  l.A = l.x1 + n * l.x * e;
  l.B = l.A + n * l.a * e;
  l.parts_at = (l.B + n * l.a * e + 15) / 16 * 16;
  // Few tiles and many columns: K in shares of at least kShare (us, whole and in shares: 64 x 16384 814, 115; 1024 x 16384
  // 1402, 1068; 768 x 2048 265, 230; 2 x 40 x 4000 255, 117; 4096 x 8192 7472, 7114)
  const int64_t k = l.d.R / l.half, tiles = n * k * (k + 1) / 2;
  l.split = (int)std::max<int64_t>(1, std::min<int64_t>(kFillTiles / tiles, l.d.C / kShare));
  l.bytes = l.parts_at + (l.split > 1 ? n * l.split * l.a * sizeof(float) : 0);
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

// Sums of squares, in fp64 and a fixed order. Bound by HBM: bf16 4096 x 8192, 67 MB, 20 us (3.4 TB/s).
template <class E>
__global__ __launch_bounds__(kNorm) void ortho_norm_k(const void* u0, View v, double* part) {
  typedef typename E::T T;
  __shared__ double lds[kNorm / 64];
  const T* u = static_cast<const T*>(u0) + blockIdx.y * v.si;
  double s = 0.0;
  for (int i = blockIdx.x; i < v.rows; i += gridDim.x) {
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
  if (threadIdx.x == 0) part[blockIdx.y * gridDim.x + blockIdx.x] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__device__ __forceinline__ void split(float x, _Float16 (&p)[kParts]) {
  p[0] = (_Float16)x;
  p[1] = (_Float16)(x - (float)p[0]);
}

// X's parts, padding included: tiles of 64 x 64, read along U's faster axis and written along X's rows, eight elements a thread at
// once (one by one where they do not lie side by side, and at the edges). bf16 4096 x 8192, 201 MB, 42 us (4.8 TB/s).
template <class E>
__global__ __launch_bounds__(256) void ortho_load_k(const void* u0, View v, OrthoDims d, const double* part, int parts,
                                                    double eps, _Float16* x) {
  typedef typename E::T T;
  __shared__ float t[64][65];
  const int tiles = d.C / 64, r0 = blockIdx.x / tiles * 64, c0 = blockIdx.x % tiles * 64;
  double s = 0.0;   // every wave adds them up in the same order
  for (int p = threadIdx.x & 63; p < parts; p += 64) s += part[(size_t)blockIdx.y * parts + p];
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o);
  // an infinity or NaN makes NaN of the whole; of no update nothing is left, whatever eps
  const double f = s == 0.0 ? 0.0 : (s - s == 0.0 ? (double)kUp / (sqrt(s) + eps) : __longlong_as_double(0x7FF8000000000000ll));
  const T* u = static_cast<const T*>(u0) + blockIdx.y * v.si;
  const bool rows = v.by_rows != d.turned;   // X's rows lie along the slow axis
  const int s0 = rows ? r0 : c0, f0 = rows ? c0 : r0;
  const bool whole = v.fast == 1 && s0 + 64 <= v.rows && f0 + 64 <= v.cols;
  for (int k = threadIdx.x; k < 64 * 8; k += 256) {
    typedef T Raw __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    typedef T Val __attribute__((ext_vector_type(8)));
    const int sl = s0 + (k >> 3), fa = f0 + (k & 7) * 8, i = k >> 3, j = (k & 7) * 8;
    float w[8];
    if (whole) {
      const Val y = __builtin_bit_cast(Val, *reinterpret_cast<const Raw*>(u + sl * v.slow + fa));
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = (float)((double)(float)y[e] * f);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = 0.0f;
        if (sl < v.rows && fa + e < v.cols) w[e] = (float)((double)(float)u[sl * v.slow + (fa + e) * v.fast] * f);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) t[rows ? i : j + e][rows ? j + e : i] = w[e];
  }
  __syncthreads();
  const size_t cells = (size_t)d.R * d.C;
  for (int k = threadIdx.x; k < 64 * 8; k += 256) {
    const int i = k >> 3, j = (k & 7) * 8;
    H8 w[kParts];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 p[kParts];
      split(t[i][j + e], p);
#pragma unroll
      for (int q = 0; q < kParts; ++q) w[q][e] = p[q];
    }
#pragma unroll
    for (int q = 0; q < kParts; ++q)
      *reinterpret_cast<H8*>(x + ((size_t)blockIdx.y * kParts + q) * cells + (size_t)(r0 + i) * d.C + c0 + j) = w[q];
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
__global__ __launch_bounds__(256) void ortho_store_k(const _Float16* x, OrthoDims d, Out o) {   // no steps
  const int i = blockIdx.y, r = blockIdx.x;
  const size_t cells = (size_t)d.R * d.C;
  for (int c = threadIdx.x; c < d.c; c += 256) {
    float v = 0.0f;
#pragma unroll
    for (int q = kParts - 1; q >= 0; --q) v += (float)x[((size_t)i * kParts + q) * cells + (size_t)r * d.C + c];
    o.put(i, r, c, v);
  }
}

__device__ __forceinline__ H4 read_turned(const _Float16* p) {
  typedef short S4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) S4 L4;
  return __builtin_bit_cast(H4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((L4*)(p)));
}

// The three products, tiles of TM x TM:
//   kGram   out = P P^T             P = X, K = C
//   kPoly   out = b P + c P P^T     P = A (symmetric), K = R
//   kStep   out = a Q + P Q         P = B, Q = X [K][.], read turned from LDS
// K goes by BK; its next parts are on their way to registers while the present one is multiplied, and go to the other half
// of LDS one after another. In LDS a row's chunks of 16 bytes are exchanged so that 16 rows at one place of K lie in
// different banks. Tiles of 256 are shared by eight waves, 128 x 64 each (of 64 x 64 LDS feeds the matrix units too slowly:
// it gives 128 bytes a cycle, and a wave needs 128 of them per 8 cycles of MFMA), smaller ones by four. Large ones are bound by
// the matrix units (4096 x 8192, of three products of parts: kStep 664 us, 1240 TFLOP/s, for 1063 that one large library product
// reaches; kGram 412, 1060 of the tiles that it forms; kPoly 273, 800: 136 tiles on 256 CUs), small ones by a tile's chain
// (4 x 256 x 256: 5.3 to 6.1 us each).
enum { kGram = 0, kPoly = 1, kStep = 2 };
struct Mul {
  const _Float16 *P, *Q;
  _Float16* out;
  size_t p, q, o;     // elements of a part
  int K, rows, cols;  // tiles of the result
  int ld;             // of out and Q
  float own, mul;     // the result is own * (P or Q) + mul * product, as it is held
  float* parts;       // kGram, shares of K: their sums
  Out last;           // kStep: where the last step goes
  int r, c;
  bool end;
};
constexpr int threads_of(int TM) { return TM == 256 ? 512 : 256; }
template <int TM>
struct Form {
  static constexpr int BK = TM == 64 ? 64 : 32;   // two stages of 128 x 64 would leave a CU one workgroup
  static constexpr int kRows = TM == 256 ? 4 : TM / 64, kCols = TM == 256 ? 2 : TM / 64;
  static constexpr int kStage = kParts * TM * BK;   // elements of P or Q in half of LDS
  static constexpr size_t kBand = 64 * (TM + 1) * sizeof(float);   // of the result
  static constexpr size_t kLds = std::max(4 * kStage * sizeof(_Float16), kBand);
};
template <int TM, int KIND>
__global__ __launch_bounds__(threads_of(TM), TM == 256 ? 1 : 2) void ortho_mul_k(Mul m) {
  typedef Form<TM> Fm;
  constexpr int BK = Fm::BK, CH = BK / 8, NT = threads_of(TM), U = TM * BK / 8 / NT, WR = Fm::kRows, WC = Fm::kCols;
  constexpr int AHEAD = TM == 256 ? 1 : 2;   // parts of K on their way
  constexpr int QC = TM / 8;   // chunks of a row of Q, turned
  extern __shared__ __align__(16) char raw[];
  _Float16* const lds = reinterpret_cast<_Float16*>(raw);   // [half][P, Q][part]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int AC = TM / (32 * WC);   // waves along the columns
  const int wr = wave / AC * 32 * WR, wc = wave % AC * 32 * WC, l32 = lane & 31, half = lane >> 5;
  // a run of (share of K, matrix, tile) per XCD, so that neighbours share their operands in its L2 and many matrices are each
  // read by few XCDs; runs go down bands of eight rows of tiles
  const unsigned lin = (blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x, xcd = lin & 7;
  const unsigned all = gridDim.x * gridDim.y * gridDim.z, each = all >> 3, more = all & 7;
  const unsigned unit0 = xcd * each + (xcd < more ? xcd : more) + (lin >> 3);
  const int id = unit0 % gridDim.x, i = unit0 / gridDim.x % gridDim.y, z = unit0 / gridDim.x / gridDim.y;
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
  const int r0 = ti * TM, c0 = tj * TM, ldk = m.K;
  const bool shares = KIND == kGram && gridDim.z > 1;
  int K = ldk, from = 0;   // the steps of BK that are this workgroup's
  if (shares) {
    const int all_k = ldk / BK;
    from = (int)((int64_t)all_k * z / gridDim.z) * BK;
    K = (int)((int64_t)all_k * (z + 1) / gridDim.z) * BK - from;
  }
  const _Float16* P = m.P + (size_t)i * kParts * m.p + (size_t)r0 * ldk + from;
  const _Float16* Q = KIND == kStep ? m.Q + (size_t)i * kParts * m.q + c0 : m.P + (size_t)i * kParts * m.p + (size_t)c0 * ldk + from;
  struct Stage { H8 p[kParts][U], q[kParts][U]; };
  Stage in[AHEAD];
  auto fetch = [&](Stage& g, int k0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int unit = threadIdx.x + u * NT, row = unit / CH, ch = unit % CH;
#pragma unroll
      for (int q = 0; q < kParts; ++q) {
        g.p[q][u] = *reinterpret_cast<const H8*>(P + q * m.p + (size_t)row * ldk + k0 + ch * 8);
        if (KIND == kStep) g.q[q][u] = *reinterpret_cast<const H8*>(Q + q * m.q + (size_t)(k0 + unit / QC) * m.ld + unit % QC * 8);
        else g.q[q][u] = *reinterpret_cast<const H8*>(Q + q * m.p + (size_t)row * ldk + k0 + ch * 8);
      }
    }
  };
  auto swap_p = [](int row, int ch) { return row * BK + ((ch ^ ((row / (16 / CH)) & (CH - 1))) * 8); };
  auto swap_q = [](int row, int ch) { return row * TM + ((ch ^ ((row & 3) << 2 & (QC - 1))) * 8); };
  auto ps = [&](int h, int q) { return lds + (2 * h) * Fm::kStage + q * (TM * BK); };
  auto qs = [&](int h, int q) { return lds + (2 * h + 1) * Fm::kStage + q * (TM * BK); };
  auto store = [&](const Stage& g, int to) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int unit = threadIdx.x + u * NT, at = swap_p(unit / CH, unit % CH);
#pragma unroll
      for (int q = 0; q < kParts; ++q) {
        *reinterpret_cast<H8*>(ps(to, q) + at) = g.p[q][u];
        *reinterpret_cast<H8*>(qs(to, q) + (KIND == kStep ? swap_q(unit / QC, unit % QC) : at)) = g.q[q][u];
      }
    }
  };
  F16x acc[WR][WC];
#pragma unroll
  for (int x = 0; x < WR; ++x) {
#pragma unroll
    for (int y = 0; y < WC; ++y) acc[x][y] = F16x{};
  }
  auto multiply = [&](int from) {
#pragma unroll
    for (int kk = 0; kk < BK / 16; ++kk) {
      H8 a[WR][kParts], b[WC][kParts];
#pragma unroll
      for (int q = 0; q < kParts; ++q) {
#pragma unroll
        for (int x = 0; x < WR; ++x)
          a[x][q] = *reinterpret_cast<const H8*>(ps(from, q) + swap_p(wr + 32 * x + l32, 2 * kk + half));
#pragma unroll
        for (int y = 0; y < WC; ++y) {
          if (KIND == kStep) {
            const int k = 16 * kk + 8 * half + ((lane & 15) >> 2), c = wc + 32 * y + (lane & 16) + 4 * (lane & 3);
            const H4 lo = read_turned(qs(from, q) + swap_q(k, c / 8) + (c & 7));
            const H4 hi = read_turned(qs(from, q) + swap_q(k + 4, c / 8) + (c & 7));
            b[y][q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          } else {
            b[y][q] = *reinterpret_cast<const H8*>(qs(from, q) + swap_p(wc + 32 * y + l32, 2 * kk + half));
          }
        }
      }
#pragma unroll
      for (int p = 0; p < kParts; ++p) {
#pragma unroll
        for (int q = 0; q + p < kParts; ++q) {
#pragma unroll
          for (int x = 0; x < WR; ++x) {
#pragma unroll
            for (int y = 0; y < WC; ++y)
              acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[x][p], b[y][q], acc[x][y], 0, 0, 0);
          }
        }
      }
    }
  };
#pragma unroll
  for (int j = 0; j < AHEAD; ++j)
    if (j * BK < K) fetch(in[j], j * BK);
  store(in[0], 0);
  if (AHEAD * BK < K) fetch(in[0], AHEAD * BK);
  __syncthreads();
  int use = 0;
  for (int k1 = 0; k1 < K; k1 += AHEAD * BK) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int k0 = k1 + j * BK;
      if (k0 < K) {
        Stage& next = in[(j + 1) % AHEAD];
        multiply(use);
        if (k0 + BK < K) store(next, use ^ 1);
        if (k0 + (AHEAD + 1) * BK < K) fetch(next, k0 + (AHEAD + 1) * BK);
        __syncthreads();
        use ^= 1;
      }
    }
  }
  // The result goes through LDS, 64 rows at once, so that memory is read and written in chunks of 16 bytes, also where a
  // tile is written a second time, turned.
  constexpr int S = TM + 1;   // eight rows apart lie in different banks
  float* const t = reinterpret_cast<float*>(raw);
  const _Float16* own = KIND == kStep ? m.Q + (size_t)i * kParts * m.q : m.P + (size_t)i * kParts * m.p;
  const size_t own_part = KIND == kStep ? m.q : m.p;
  _Float16* out = m.out + (size_t)i * kParts * m.o;
  const bool end = KIND == kStep && m.end, twice = KIND != kStep && ti != tj && !shares;
  for (int band = 0; band < TM; band += 64) {
#pragma unroll
    for (int x = 0; x < WR; ++x) {
      const int rr = wr + 32 * x - band;   // lane: column l32 of a tile, rows 8 (e / 4) + 4 half + e % 4
      if (rr < 0 || rr >= 64) continue;
#pragma unroll
      for (int y = 0; y < WC; ++y) {
#pragma unroll
        for (int e = 0; e < 16; ++e) t[(rr + 8 * (e / 4) + 4 * half + e % 4) * S + wc + 32 * y + l32] = acc[x][y][e];
      }
    }
    __syncthreads();
    for (int unit = threadIdx.x; unit < 64 * QC; unit += NT) {
      const int rr = unit / QC, c = unit % QC * 8;
      const size_t at = (size_t)(r0 + band + rr) * m.ld + c0 + c;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = t[rr * S + c + e] * m.mul;
      if (shares) {
        Fl4* to = reinterpret_cast<Fl4*>(m.parts + ((size_t)i * gridDim.z + z) * m.o + at);
        to[0] = Fl4{v[0], v[1], v[2], v[3]};
        to[1] = Fl4{v[4], v[5], v[6], v[7]};
        continue;
      }
      if (KIND != kGram) {
        H8 w[kParts];
#pragma unroll
        for (int q = 0; q < kParts; ++q) w[q] = *reinterpret_cast<const H8*>(own + q * own_part + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = fmaf(m.own, (float)w[1][e] + (float)w[0][e], v[e]);
        }
      }
      if (end || twice) {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[rr * S + c + e] = v[e];
      }
      if (!end) {
        H8 w[kParts];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          _Float16 p[kParts];
          split(v[e], p);
#pragma unroll
          for (int q = 0; q < kParts; ++q) w[q][e] = p[q];
        }
#pragma unroll
        for (int q = 0; q < kParts; ++q) *reinterpret_cast<H8*>(out + q * m.o + at) = w[q];
      }
    }
    __syncthreads();
    if (twice) {
      for (int unit = threadIdx.x; unit < 8 * TM; unit += NT) {
        const int c = unit / 8, rr = unit % 8 * 8;
        H8 w[kParts];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          _Float16 p[kParts];
          split(t[(rr + e) * S + c], p);
#pragma unroll
          for (int q = 0; q < kParts; ++q) w[q][e] = p[q];
        }
#pragma unroll
        for (int q = 0; q < kParts; ++q)
          *reinterpret_cast<H8*>(out + q * m.o + (size_t)(c0 + c) * m.ld + r0 + band + rr) = w[q];
      }
    }
    if (end) {
      const bool down = m.last.sr < m.last.sc;   // along the result's adjacent elements
      for (int cell = threadIdx.x; cell < 64 * TM; cell += NT) {
        const int rr = down ? cell & 63 : cell / TM, c = down ? cell >> 6 : cell % TM;
        if (r0 + band + rr < m.r && c0 + c < m.c) m.last.put(i, r0 + band + rr, c0 + c, t[rr * S + c]);
      }
    }
    if (end || twice) __syncthreads();
  }
}

// The shares' sums, in order, to A's parts: 16 x 64 at once, on and below the diagonal, and turned. Bound by HBM: three shares
// of 4096 x 4096, 174 MB, 36 us (4.8 TB/s).
__global__ __launch_bounds__(256) void ortho_sum_k(const float* in, int shares, _Float16* out, int R, int half) {
  __shared__ float t[16][65];
  const int tiles = R / 64, r0 = blockIdx.x / tiles * 16, c0 = blockIdx.x % tiles * 64;
  if (r0 / half < c0 / half) return;   // formed turned (by tiles of `half`, as they are there)
  const size_t cells = (size_t)R * R;
  in += (size_t)blockIdx.y * shares * cells;
  out += (size_t)blockIdx.y * kParts * cells;
  const int row = threadIdx.x >> 4, c = (threadIdx.x & 15) * 4;
  const size_t at = (size_t)(r0 + row) * R + c0 + c;
  Fl4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
  for (int z = 0; z < shares; ++z) s += *reinterpret_cast<const Fl4*>(in + z * cells + at);
  H4 w[kParts];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    _Float16 p[kParts];
    split(s[e], p);
    t[row][c + e] = s[e];
#pragma unroll
    for (int q = 0; q < kParts; ++q) w[q][e] = p[q];
  }
#pragma unroll
  for (int q = 0; q < kParts; ++q) *reinterpret_cast<H4*>(out + q * cells + at) = w[q];
  if (r0 / half == c0 / half) return;
  __syncthreads();
  const int col = threadIdx.x >> 2, rr = (threadIdx.x & 3) * 4;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    _Float16 p[kParts];
    split(t[rr + e][col], p);
#pragma unroll
    for (int q = 0; q < kParts; ++q) w[q][e] = p[q];
  }
#pragma unroll
  for (int q = 0; q < kParts; ++q) *reinterpret_cast<H4*>(out + q * cells + (size_t)(c0 + col) * R + r0 + rr) = w[q];
}

template <int TM, int KIND>
hipError_t launch_mul(const Mul& m, const Layout& l, hipStream_t st) {
  static std::atomic<uint64_t> done;
  const size_t lds = Form<TM>::kLds;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(&ortho_mul_k<TM, KIND>), lds, done);
  if (e != hipSuccess) return e;
  const int64_t tr = l.d.R / TM, tc = l.d.C / TM;
  const dim3 grid((unsigned)(KIND == kStep ? tr * tc : tr * (tr + 1) / 2), (unsigned)l.d.n,
                  KIND == kGram ? l.split : 1), block(threads_of(TM));
  hipLaunchKernelGGL((ortho_mul_k<TM, KIND>), grid, block, lds, st, m);
  return hipSuccess;
}
template <int KIND>
hipError_t launch_mul(int tile, const Mul& m, const Layout& l, hipStream_t st) {
  return tile == 256 ? launch_mul<256, KIND>(m, l, st) : tile == 128 ? launch_mul<128, KIND>(m, l, st) : launch_mul<64, KIND>(m, l, st);
}

hipError_t steps_of(const OrthoArgs& a, const Layout& l, const Out& last, hipStream_t st) {
  char* w = static_cast<char*>(a.work);
  _Float16 *x = reinterpret_cast<_Float16*>(w + l.x0), *y = reinterpret_cast<_Float16*>(w + l.x1);
  _Float16 *A = reinterpret_cast<_Float16*>(w + l.A), *B = reinterpret_cast<_Float16*>(w + l.B);
  hipError_t e = hipSuccess;
  for (int i = 0; i < a.c.steps && e == hipSuccess; ++i) {
    Mul m{};
    m.P = x; m.p = l.x; m.out = A; m.o = l.a; m.K = l.d.C; m.ld = l.d.R; m.mul = kDown;
    m.parts = reinterpret_cast<float*>(w + l.parts_at);
    if ((e = launch_mul<kGram>(l.half, m, l, st)) != hipSuccess) break;
    if (l.split > 1)
      hipLaunchKernelGGL(ortho_sum_k, dim3((unsigned)((int64_t)(l.d.R / 64) * (l.d.R / 16)), (unsigned)l.d.n), dim3(256), 0, st, m.parts,
                         l.split, A, l.d.R, l.half);
    m.P = A; m.p = l.a; m.out = B; m.K = l.d.R; m.own = a.c.b; m.mul = a.c.c * kDown;
    if ((e = launch_mul<kPoly>(l.half, m, l, st)) != hipSuccess) break;
    m.P = B; m.Q = x; m.q = l.x; m.out = y; m.o = l.x; m.ld = l.d.C; m.own = a.c.a; m.mul = kDown;
    m.rows = l.d.R / l.whole; m.cols = l.d.C / l.whole; m.r = l.d.r; m.c = l.d.c; m.last = last; m.end = i + 1 == a.c.steps;
    e = launch_mul<kStep>(l.whole, m, l, st);
    std::swap(x, y);
  }
  return e;
}

template <class E>
hipError_t launch_typed(const OrthoArgs& a, hipStream_t st) {
  const Layout l = layout_of(a.c);
  char* w = static_cast<char*>(a.work);
  double* sums = reinterpret_cast<double*>(w + l.sums);
  _Float16* x = reinterpret_cast<_Float16*>(w + l.x0);
  const unsigned n = (unsigned)l.d.n;
  const View v = view_of(a.u, a.c);
  const Out out{a.out.data, a.out.stride_i, l.d.turned ? a.out.stride_c : a.out.stride_r,
                l.d.turned ? a.out.stride_r : a.out.stride_c, a.c.dtype, a.c.scale * kDown};
  hipLaunchKernelGGL(ortho_norm_k<E>, dim3(l.sums_n, n), dim3(kNorm), 0, st, a.u.data, v, sums);
  hipLaunchKernelGGL(ortho_load_k<E>, dim3((unsigned)((int64_t)(l.d.R / 64) * (l.d.C / 64)), n), dim3(256), 0, st, a.u.data, v,
                     l.d, sums, l.sums_n, (double)a.c.eps, x);
  if (a.c.steps == 0) {
    hipLaunchKernelGGL(ortho_store_k, dim3(l.d.r, n), dim3(256), 0, st, x, l.d, out);
    return hipSuccess;
  }
  return steps_of(a, l, out, st);
}

}  // namespace

size_t ortho_bytes(const sim_ortho& c) { return c.n && c.M && c.N ? layout_of(c).bytes : 0; }

hipError_t launch_ortho(const OrthoArgs& a, hipStream_t st) {
  const hipError_t e = a.c.dtype == SIM_DT_F32 ? launch_typed<F32>(a, st)
                       : a.c.dtype == SIM_DT_BF16 ? launch_typed<BF16>(a, st) : launch_typed<F16>(a, st);
  return e == hipSuccess ? hipGetLastError() : e;
}

}  // namespace bsim
