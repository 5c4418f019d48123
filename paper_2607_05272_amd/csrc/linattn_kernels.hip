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
#include <atomic>

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
  float* parts;         // states before (after attn_join_k) or of the segments that time is split into
  int64_t pr, pc;       // strides of their rows and columns
  int64_t seg;          // steps of a segment
  int segs;
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

// One step after another: 64 columns of a state, in registers, a thread's rows 16 apart. Bound by reading and
// writing the state where there are many (64 sequences x 16 heads x 128 x 128, one step: 134 MB in 23 us, 5.8 TB/s, the
// last-level cache holding a part), by a launch's and a step's chain otherwise (8 heads x 64 x 64: 4.4 us).
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

// ---- runs of steps by matrix instructions ----------------------------------------------------------
// C steps at once:  out = so (l^(i+1-lag) Q S + (Q K^T o su l^(i-j) [j <= i]) V),  S = l^m S + K^T (su l^(m-1-j+lag) V)
// for m live ones. Values are bf16 parts that add up to them: NI of an input (bf16 1, fp16 2, fp32 3: exact), NC of
// what is multiplied again on the way to out (the weighted products, S: 2 for 16-bit types, whose outputs are rounded
// to fewer bits, 3 for fp32), and 3 of the weighted V, which S, an fp32 output held in the accumulators, is made of. A product of parts
// i and j is left out where i + j reaches the larger of the counts: it is below the last bits that are kept.
template <class E> struct PartsOf;
template <> struct PartsOf<BF16> { static constexpr int kIn = 1, kMade = 2; };
template <> struct PartsOf<F16> { static constexpr int kIn = 2, kMade = 2; };
template <> struct PartsOf<F32> { static constexpr int kIn = 3, kMade = 3; };

typedef __bf16 Bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 Bf4 __attribute__((ext_vector_type(4)));
typedef float Fl4 __attribute__((ext_vector_type(4)));

// the parts of values, an even number of them (two conversions are one instruction)
template <int N, int W>
__device__ __forceinline__ void split(const float (&x)[W], __bf16 (&p)[N][W]) {
  typedef float F2 __attribute__((ext_vector_type(2)));
  typedef __bf16 B2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int w = 0; w < W; w += 2) {
    F2 rest = {x[w], x[w + 1]};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const B2 h = __builtin_convertvector(rest, B2);
      p[i][w] = h[0];
      p[i][w + 1] = h[1];
      if (i + 1 < N) rest -= __builtin_convertvector(h, F2);
    }
  }
}
template <int W>
__device__ __forceinline__ auto packed(const __bf16 (&p)[W]) {
  typedef __bf16 B __attribute__((ext_vector_type(W)));
  B v;
#pragma unroll
  for (int w = 0; w < W; ++w) v[w] = p[w];
  return v;
}
// c += a b, as far as the parts' products count
template <int NA, int NB>
__device__ __forceinline__ void mul_parts(const Bf8 (&a)[NA], const Bf8 (&b)[NB], Fl4& c) {
  constexpr int most = NA > NB ? NA : NB;
#pragma unroll
  for (int i = 0; i < NA; ++i) {
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (i + j < most) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], c, 0, 0, 0);
  }
}
// Of a matrix in LDS, four rows by 16 columns per 16 lanes, turned: lane i gets column i. p: this lane's place, row
// i / 4 and column 4 (i % 4).
__device__ __forceinline__ Bf4 read_turned(const __bf16* p) {
  typedef short S4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) S4 L4;
  return __builtin_bit_cast(Bf4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((L4*)(p)));
}
__device__ __forceinline__ Bf8 both(Bf4 a, Bf4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// Rows of LDS start four banks apart where they are read along (q, the products), eight where they are read turned, eight
// rows by 16 columns per 32 lanes (k, which is read both ways, v): no two lanes of a step meet in a bank.
constexpr int kPad = 8, kPadTurned = 16;
template <class E, int DQ, int NW, int HV, int C>
struct RunLds {
  static constexpr int NI = PartsOf<E>::kIn, NC = PartsOf<E>::kMade, DV = 16 * NW, TT = C / 16;
  __bf16 q[NI][C][DQ + kPad], k[NI][C][DQ + kPadTurned], v[NI][C][DV + kPadTurned], p[NC][C][C + kPad];
  Fl4 half[HV > 1 ? NW : 1][HV][HV > 1 ? TT / HV : 1][HV > 1 ? 64 : 1];   // a half's sums that the other one needs
  float pow[C + 1], into[C];   // l^i; su l^(m-1-j+lag)
};

// eight elements of a row from p on
template <class T>
struct Eight {
  typedef T Raw __attribute__((ext_vector_type(8), aligned(sizeof(T))));
  typedef T Val __attribute__((ext_vector_type(8)));
  Val v;
  __device__ __forceinline__ void load(const T* p) { v = __builtin_bit_cast(Val, *reinterpret_cast<const Raw*>(p)); }
  // the elements from n on (n <= 0: all), then zeros
  __device__ __forceinline__ void skip(int n) {
    constexpr int W = sizeof(Val) / 4, each = 8 / W;   // words, elements of one
    typedef uint32_t Words __attribute__((ext_vector_type(W)));
    Words w = __builtin_bit_cast(Words, v);
    n = n < 0 ? 0 : n;
#pragma unroll
    for (int bit = 4; bit >= each; bit /= 2) {
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = n & bit ? (i + bit / each < W ? w[i + bit / each] : 0u) : w[i];
    }
    if constexpr (each == 2) {
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = n & 1 ? __builtin_amdgcn_alignbit(i + 1 < W ? w[i + 1] : 0u, w[i], 16) : w[i];
    }
    v = __builtin_bit_cast(Val, w);
  }
};

// How much of a run there is: all; some steps or columns, of those eight at least; fewer.
enum { kAll = 0, kSome = 1, kFewer = 2 };

// a run of C steps of one array, D columns, in registers between global memory and LDS: a thread's units of eight
// are kRows steps apart. What is not there is read elsewhere in the row or run, so that no load waits for a condition, and
// becomes zero on its way to LDS.
template <class E, int D, int C, int NT>
struct Tile {
  typedef typename E::T T;
  static constexpr int kUnits = C * D / 8, N = (kUnits + NT - 1) / NT, NI = PartsOf<E>::kIn, kRows = NT * 8 / D;
  static constexpr bool kPart = kUnits < NT;   // more threads than units: the last ones follow the last step
  static_assert((kPart || kUnits % NT == 0) && NT * 8 % D == 0, "whole units");
  Eight<T> u[N];
  const T* p;
  __device__ static __forceinline__ int column() { return threadIdx.x % (D / 8) * 8; }
  __device__ static __forceinline__ int row() {
    const int i = threadIdx.x / (D / 8);
    return kPart && i >= C ? C - 1 : i;
  }
  // the next run starts at step i of the processing order; the array's columns from c0 on, `width` of them
  __device__ __forceinline__ void start(const AttnRun& r, const In& x, int b, int h, int64_t i, int64_t n, int c0, int width) {
    const int64_t step = r.back ? -x.st : x.st;
    const int c = column(), from = c >= width ? 0 : (c + 8 > width && width >= 8 ? width - 8 : c);   // the last ones end with the row
    p = row_of<T>(x, b, r.back ? n - 1 - i : i, h) + c0 + from + row() * step;
  }
  // `now` steps, `step` elements from one to the next
  template <int HOW>
  __device__ __forceinline__ void fetch(int now, int64_t step, int width) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int at = row() + j * kRows;
      if (HOW == kAll) {
        u[j].load(p + j * kRows * step);
      } else {
        const T* q = p + ((at < now ? at : now - 1) - row()) * step;
        if (HOW == kSome || width >= 8) {
          u[j].load(q);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) u[j].v[i] = q[column() + i < width ? i : 0];
        }
      }
    }
    p += C * step;
  }
  template <int S>
  __device__ __forceinline__ void store(__bf16 (*lds)[C][S], bool all, int now, int width) {
    const int c = column();
    if (!all) {
      if ((width & 7) && width >= 8) {
#pragma unroll
        for (int j = 0; j < N; ++j) u[j].skip(c + 8 - width);   // the last ones end with the row
      } else if (width < 8) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
#pragma unroll
          for (int i = 0; i < 8; ++i) u[j].v[i] = c + i < width ? u[j].v[i] : (T)0.0f;
        }
      }
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (row() + j * kRows >= now || c >= width) u[j].v = typename Eight<T>::Val{};
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (kPart && threadIdx.x >= kUnits) continue;
      if constexpr (NI == 1) {
        *reinterpret_cast<typename Eight<T>::Val*>(&lds[0][row() + j * kRows][c]) = u[j].v;
      } else {
        float x[8];
        __bf16 w[NI][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)u[j].v[e];
        split(x, w);
#pragma unroll
        for (int q = 0; q < NI; ++q) *reinterpret_cast<Bf8*>(&lds[q][row() + j * kRows][c]) = packed(w[q]);
      }
    }
  }
};

// A workgroup takes a segment of a sequence and head and 16 columns of its state per wave, or per HV waves that share its
// rows, which hold them as accumulators (lane: column lane % 16, rows 4 (lane / 16) + 0..3 of each tile of 16), so that two
// tiles are an operand of the next product as they are. While a run is multiplied the next one's loads fly. Bound by the
// chains of the phases (LDS reads, conversions, products) between barriers where a SIMD has one or two waves, which is what
// the halves are for: bf16 8 x 2048 x 16 heads x 128, ragged, 113 us for 35 of HBM, one workgroup per CU. Of 7964 cycles a
// run of 64 steps there, waves spend 1935 on Q K^T, 1710 on K^T V, 1331 on Q S, 667 on (..) V, 660 at barriers, 538 on LDS
// stores, 481 on the output, 358 on issuing loads.
template <class E, int DQ, int NW, int HV, int C, bool OUT>
__global__ __launch_bounds__(64 * NW * HV, NW * HV == 4 ? 2 : 1) void attn_run_k(AttnRun r) {
  typedef typename E::T T;
  typedef RunLds<E, DQ, NW, HV, C> Lds;
  constexpr int NI = Lds::NI, NC = Lds::NC, DV = Lds::DV, KT = DQ / 16 / HV, TT = C / 16, NT = 64 * NW * HV, TO = TT / HV;
  extern __shared__ __align__(16) char raw[];
  Lds& m = *reinterpret_cast<Lds*>(raw);
  const int lane = threadIdx.x & 63, lc = lane & 15, lg = lane >> 4;
  const int any = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // the same in all of a wave's lanes
  const int wave = any % NW, hv = any / NW, k0 = hv * KT;             // its columns, and its rows' first tile
  const int cols = (r.Dv + DV - 1) / DV;
  const int seg = blockIdx.y, c0 = blockIdx.x % cols * DV, bh = blockIdx.x / cols, h = bh % r.H, b = bh / r.H;
  const float l = decay_of(r, h);
  const int64_t n = steps_of(r, b), first = seg * r.seg, last = first + r.seg < r.T ? first + r.seg : r.T;
  const int64_t live = n < last ? n : last;   // of the segment's steps in processing order: [first, live)
  const int width = r.Dv - c0 < DV ? r.Dv - c0 : DV;
  const double log2l = log2((double)l);
  auto power = [&](int i) { return i == 0 ? 1.0f : (float)exp2(i * log2l); };
  Fl4 st[KT];
  const bool split_time = r.segs > 1;
  const float* s0 = split_time ? r.parts + ((int64_t)bh * r.segs + seg) * r.Dq * r.Dv
                               : (r.s0 ? r.s0 + (int64_t)bh * r.Dq * r.Dv : nullptr);
  const int64_t sr = split_time ? r.pr : r.sr, sc = split_time ? r.pc : r.sc;
  if (!OUT && split_time) s0 = nullptr;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const int c = c0 + wave * 16 + lc;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = (k0 + kt) * 16 + 4 * lg + i;
      st[kt][i] = s0 && row < r.Dq && c < r.Dv ? s0[row * sr + c * sc] : 0.0f;
    }
  }
  if (threadIdx.x <= C) m.pow[threadIdx.x] = power(threadIdx.x);
  // the tiles beside the diagonal in a step of 32 stay zeros
  static_assert(TT % 2 == 0, "steps of 32");
  if (OUT) {
    for (int i = threadIdx.x; i < NC * TT / 2 * 256; i += NT)
      m.p[i / (TT / 2 * 256)][i / 256 % (TT / 2) * 32 + (i & 15)][i / 256 % (TT / 2) * 32 + 16 + (i >> 4 & 15)] = (__bf16)0.0f;
  }
  __syncthreads();
  float out_w[TT];   // so l^(t+1-lag) of this lane's step of each tile
#pragma unroll
  for (int t = 0; t < TT; ++t) out_w[t] = r.so * m.pow[16 * t + lc + 1 - r.lag];
  const float inner = r.so * r.su;
  Tile<E, DQ, C, NT> q, k;
  Tile<E, DV, C, NT> v;
  if (OUT) q.start(r, r.q, b, h, first, n, 0, r.Dq);
  k.start(r, r.k, b, h, first, n, 0, r.Dq);
  v.start(r, r.v, b, h, first, n, c0, width);
  const bool full = r.Dq == DQ && width == DV, eights = r.Dq >= 8 && width >= 8;
  auto fetch = [&](int64_t left) {
    const int now = left < C ? (int)left : C;
    auto go = [&](auto H) {
      constexpr int HOW = decltype(H)::value;
      if (OUT) q.template fetch<HOW>(now, r.back ? -r.q.st : r.q.st, r.Dq);
      k.template fetch<HOW>(now, r.back ? -r.k.st : r.k.st, r.Dq);
      v.template fetch<HOW>(now, r.back ? -r.v.st : r.v.st, width);
    };
    if (full && now == C) go(std::integral_constant<int, kAll>{});
    else if (eights) go(std::integral_constant<int, kSome>{});
    else go(std::integral_constant<int, kFewer>{});
  };
  const int64_t turn = r.back ? -r.ot : r.ot;   // of out, from one step to the next
  int64_t at0 = b * r.ob + (r.back ? n - 1 - first : first) * r.ot + h * r.oh + c0 + lc * turn + wave * 16 + 4 * lg;
  if (first < live) fetch(live - first);
  for (int64_t i0 = first; i0 < live; i0 += C) {
    const int now = live - i0 < C ? (int)(live - i0) : C;
    __syncthreads();
    const bool all = full && now == C;
    if (OUT) q.store(m.q, all, now, r.Dq);
    k.store(m.k, all, now, r.Dq);
    v.store(m.v, all, now, width);
    if (threadIdx.x < C) {
      const int j = threadIdx.x;
      m.into[j] = j < now ? r.su * m.pow[now - 1 - j + r.lag] : 0.0f;
    }
    __syncthreads();
    if (i0 + C < live) fetch(live - i0 - C);
    if constexpr (OUT) {
      // weighted products, turned: rows j, columns i; a wave's tiles of j <= i side by side
      constexpr int W = NW * HV, kTiles = TT * (TT + 1) / 2, kMost = (kTiles + W - 1) / W;
      auto products = [&](auto N) {
        constexpr int MINE = decltype(N)::value;
        if constexpr (MINE > 0) {
          int ti[MINE], tj[MINE];
          Fl4 w[MINE];
#pragma unroll
          for (int n = 0; n < MINE; ++n) {
            const int at = any + n * W;
            ti[n] = 0;
#pragma unroll
            for (int x = 1; x < TT; ++x) ti[n] += at >= x * (x + 1) / 2;
            tj[n] = at - ti[n] * (ti[n] + 1) / 2;
            w[n] = Fl4{0.0f, 0.0f, 0.0f, 0.0f};
          }
#pragma unroll
          for (int kk = 0; kk < DQ / 32; ++kk) {
#pragma unroll
            for (int n = 0; n < MINE; ++n) {
              Bf8 a[NI], x[NI];
#pragma unroll
              for (int p = 0; p < NI; ++p) {
                a[p] = *reinterpret_cast<const Bf8*>(&m.k[p][16 * tj[n] + lc][32 * kk + 8 * lg]);
                x[p] = *reinterpret_cast<const Bf8*>(&m.q[p][16 * ti[n] + lc][32 * kk + 8 * lg]);
              }
              mul_parts(a, x, w[n]);
            }
          }
#pragma unroll
          for (int n = 0; n < MINE; ++n) {
            float y[4];
            __bf16 o[NC][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int gap = 16 * (ti[n] - tj[n]) + lc - (4 * lg + i);
              y[i] = gap >= 0 ? w[n][i] * (inner * m.pow[gap < 0 ? 0 : gap]) : 0.0f;
            }
            split(y, o);
#pragma unroll
            for (int x = 0; x < NC; ++x)
              *reinterpret_cast<Bf4*>(&m.p[x][16 * ti[n] + lc][16 * tj[n] + 4 * lg]) = packed(o[x]);
          }
        }
      };
      if (any + (kMost - 1) * W < kTiles) products(std::integral_constant<int, kMost>{});
      else products(std::integral_constant<int, kMost - 1>{});
      // S^T Q^T, columns i
      Fl4 acc[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t) acc[t] = Fl4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kk = 0; kk < KT / 2; ++kk) {
        Bf8 s[NC];
        float w[8];
        __bf16 p[NC][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = st[2 * kk + i / 4][i % 4];
        split(w, p);
#pragma unroll
        for (int x = 0; x < NC; ++x) s[x] = packed(p[x]);
#pragma unroll
        for (int t = 0; t < TT; ++t) {
          Bf8 x[NI];
#pragma unroll
          for (int p = 0; p < NI; ++p) {
            const __bf16* row = &m.q[p][16 * t + lc][16 * k0 + 32 * kk + 4 * lg];
            x[p] = both(*reinterpret_cast<const Bf4*>(row), *reinterpret_cast<const Bf4*>(row + 16));
          }
          mul_parts(s, x, acc[t]);
        }
      }
#pragma unroll
      for (int t = 0; t < TT; ++t) acc[t] *= out_w[t];
      // of the halves' sums each goes on with every HV-th tile
      Fl4 y[TO];
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        if (HV == 1 || t % HV == hv) y[t / HV] = acc[t];
        else m.half[wave][t % HV][t / HV][lane] = acc[t];
      }
      __syncthreads();   // the weighted products are there
      if constexpr (HV > 1) {
#pragma unroll
        for (int t = 0; t < TO; ++t) y[t] += m.half[wave][hv][t][lane];
      }
      Bf8 a[C / 32][NI];
      uint32_t odd = 0;   // bits 15 and 31: all exponent bits of a value of this wave's columns
#pragma unroll
      for (int j = 0; j < C / 32; ++j) {
#pragma unroll
        for (int p = 0; p < NI; ++p) {
          const __bf16* at = &m.v[p][32 * j + 4 * lg + lc / 4][wave * 16 + 4 * (lc % 4)];
          a[j][p] = both(read_turned(at), read_turned(at + 16 * (DV + kPadTurned)));
        }
        typedef uint32_t U4 __attribute__((ext_vector_type(4)));
        const U4 w = __builtin_bit_cast(U4, a[j][0]);
#pragma unroll
        for (int i = 0; i < 4; ++i) odd |= (w[i] & 0x7F807F80u) + 0x00800080u;
      }
      if (!__any(odd & 0x80008000u)) {
#pragma unroll
        for (int j = 0; j < C / 32; ++j) {
#pragma unroll
          for (int o = 2 * j / HV; o < TO; ++o) {   // tiles below the diagonal, those that stand on it in 32 x 32 among them
            const int t = HV * o + hv;
            Bf8 x[NC];
#pragma unroll
            for (int p = 0; p < NC; ++p) {
              const __bf16* row = &m.p[p][16 * t + lc][32 * j + 4 * lg];
              x[p] = both(*reinterpret_cast<const Bf4*>(row), *reinterpret_cast<const Bf4*>(row + 16));
            }
            mul_parts(a[j], x, y[o]);
          }
        }
      } else {
        // An infinity or NaN among the values: by the zeros above the diagonal it would reach steps before its own. What
        // the look for it costs: 8 x 2048 x 16 heads x 128 111 and 115 us.
#pragma unroll
        for (int o = 0; o < TO; ++o) {
          const int i = 16 * (HV * o + hv) + lc;
#pragma unroll 1
          for (int j = 0; j <= i; ++j) {
            float w = 0.0f;
#pragma unroll
            for (int p = NC - 1; p >= 0; --p) w += (float)m.p[p][i][j];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float x = 0.0f;
#pragma unroll
              for (int p = NI - 1; p >= 0; --p) x += (float)m.v[p][j][wave * 16 + 4 * lg + e];
              y[o][e] = fmaf(w, x, y[o][e]);
            }
          }
        }
      }
      either(full && now == C && !r.wide, [&](auto W) {
        constexpr bool WHOLE = decltype(W)::value;
        typedef T Raw __attribute__((ext_vector_type(4), aligned(sizeof(T))));
        typedef T Val __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int o = 0; o < TO; ++o) {
          const int t = HV * o + hv;
          const int64_t at = at0 + 16 * t * turn;
          if (WHOLE) {
            *reinterpret_cast<Raw*>(static_cast<T*>(r.out) + at) = __builtin_bit_cast(Raw, __builtin_convertvector(y[o], Val));
          } else if (16 * t + lc < now) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (wave * 16 + 4 * lg + e >= width) continue;
              if (r.wide) static_cast<float*>(r.out)[at + e] = y[o][e];
              else static_cast<T*>(r.out)[at + e] = (T)y[o][e];
            }
          }
        }
      });
      at0 += C * turn;
    }
    // S = l^m S + K^T V weighted
    const float fade = m.pow[now];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      st[kt] *= fade;
    }
#pragma unroll
    for (int j = 0; j < C / 32; ++j) {
      Bf8 x[3];
      Bf8 a[NI];
#pragma unroll
      for (int p = 0; p < NI; ++p) {
        const __bf16* at = &m.v[p][32 * j + 4 * lg + lc / 4][wave * 16 + 4 * (lc % 4)];
        a[p] = both(read_turned(at), read_turned(at + 16 * (DV + kPadTurned)));
      }
      float w[8];
      __bf16 o[3][8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[i] = (float)a[0][i];
#pragma unroll
        for (int p = 1; p < NI; ++p) w[i] += (float)a[p][i];
        w[i] *= m.into[32 * j + 16 * (i / 4) + 4 * lg + i % 4];
      }
      split(w, o);
#pragma unroll
      for (int p = 0; p < 3; ++p) x[p] = packed(o[p]);
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        Bf8 a[NI];
#pragma unroll
        for (int p = 0; p < NI; ++p) {
          const __bf16* at = &m.k[p][32 * j + 4 * lg + lc / 4][16 * (k0 + kt) + 4 * (lc % 4)];
          a[p] = both(read_turned(at), read_turned(at + 16 * (DQ + kPadTurned)));
        }
        mul_parts(a, x, st[kt]);
      }
    }
  }
  if (OUT) {   // padding
    const int c = threadIdx.x % (DV / 8) * 8, row = threadIdx.x / (DV / 8), have = width - c;
    for (int64_t i = (live > first ? live : first) + row; i < last && have > 0; i += NT * 8 / DV) {
      const int64_t at = b * r.ob + i * r.ot + h * r.oh + c0 + c;
      if (!r.wide && have >= 8) {
        *reinterpret_cast<typename Eight<T>::Raw*>(static_cast<T*>(r.out) + at) = typename Eight<T>::Raw{};
        continue;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e >= have) continue;
        if (r.wide) static_cast<float*>(r.out)[at + e] = 0.0f;
        else static_cast<T*>(r.out)[at + e] = (T)0.0f;
      }
    }
  }
  float* to = OUT ? (split_time || !r.state ? nullptr : r.state + (int64_t)bh * r.Dq * r.Dv)
                  : (split_time ? r.parts + ((int64_t)bh * r.segs + seg) * r.Dq * r.Dv : r.state + (int64_t)bh * r.Dq * r.Dv);
  if (!to) return;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const int c = c0 + wave * 16 + lc;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = (k0 + kt) * 16 + 4 * lg + i;
      if (row < r.Dq && c < r.Dv) to[row * sr + c * sc] = st[kt][i];
    }
  }
}

// The segments' own last states become the states that they start from: an element of the state a thread. Bound by a
// chain of loads: 64 segments of 8 heads x 64 x 64 10 us (32 loads ahead: 11).
__global__ __launch_bounds__(256) void attn_join_k(AttnRun r) {
  const int h = blockIdx.y % r.H, b = blockIdx.y / r.H;
  const int cells = r.Dq * r.Dv, i = blockIdx.x * 256 + threadIdx.x;
  float l = r.decay[h];
  l = l >= 0.0f ? (l > 1.0f ? 1.0f : l) : 0.0f;
  int64_t n = r.len ? r.len[b] : r.T;
  n = n < 0 ? 0 : (n > r.T ? r.T : n);
  if (i >= cells) return;
  const int64_t at = (int64_t)blockIdx.y * cells + i / r.Dv * r.sr + i % r.Dv * r.sc;
  float s = r.s0 ? r.s0[at] : 0.0f;
  const double log2l = log2((double)l);
  const float whole = (float)exp2((double)r.seg * log2l);
  float* p = r.parts + (int64_t)blockIdx.y * r.segs * cells + i;
  constexpr int kAhead = 16;   // loads that fly together
  for (int g0 = 0; g0 < r.segs; g0 += kAhead) {
    float own[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (g0 + u < r.segs) own[u] = p[(int64_t)(g0 + u) * cells];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (g0 + u >= r.segs) continue;
      p[(int64_t)(g0 + u) * cells] = s;
      const int64_t left = n - (g0 + u) * r.seg;
      if (left > 0) s = fmaf(left >= r.seg ? whole : (float)exp2((double)left * log2l), s, own[u]);
    }
  }
  if (r.state) r.state[at] = s;
}

// Gradients of shared keys and values: the sum over the heads that share them, in order. They are kept in fp32 until
// here, so that a gradient is rounded once; bound by HBM (16 x 385 x 6 heads x 80, 17 MB, 7 us).
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

// Steps one after another up to kFew of them, by runs beyond.
constexpr int kFew = 16;
constexpr int run_steps(int dtype, int DQ) {   // of a run: as many as LDS holds of q, k, v and the products
  return (dtype == SIM_DT_F32 && DQ > 64) || (dtype == SIM_DT_F16 && DQ > 128) ? 32 : 64;
}
// What a workgroup takes: columns of a state (128 by eight waves; 64 by four, or by eight that halve its rows), and a sequence's
// steps or a segment of them, at the cost of reading k and v once more. By the sequences and heads there are and what their
// registers leave room for. Measured on either side of each border (us; bf16 but where stated; segs: in segments of all heads
// together, as many workgroups as stated; heads of B x H):
//   Dv > 64: segments of 128 columns for few heads and many steps, halves while one round of workgroups (two a head) fits
//   the CUs, 128 columns beyond
//     T 2048, 128 x 128, heads 32 / 64 / 80 / 96 / 112 / 128 / 192 / 240 / 256 / 384
//       128 in 256 segs    58    89   110   141   148   154
//       halves            113   113   113   115   114   115   223   223   224   338
//       128               158   157   157   158   159   163   168   171   171   331
//     T 512, heads 128 / 144, fp32: halves 63 / 117, 128 83 / 84; fp16 46 / 87, 62 / 63; bf16 36 / 65, 47 / 48
//     64 heads, T 300 / 512 / 768 / 1024 fp32: 128 in segs 51 / 57 / 60 / 88, halves 26 / 34 / 47 / 109; a training step
//     208 / 234 / 246, 123 / 168 / 235 (fp32 of 768 336, 378)
//   Dq > 64 >= Dv, 128 x 64: halves, in segs of 256 for few heads and many steps
//     64 heads, T 512 / 1024: in segs 39 / 41, whole 33 / 59; 112 heads, T 1024: 63, 59
//   64 x 64: segments of 64 columns for few heads and many steps, then halves for one round, then 64 columns, but not in
//   fp32, of which no second workgroup fits a CU
//     T 2048, heads 64 / 112 / 128 / 192 / 256: 64 in 512 segs 44 / 65 / 67 / 106 / 112, halves 85 / 86 / 86 / 86 / 87; fp32
//     T 1024, heads 64 / 112 / 128: 54 / 94 / 95, 75 / 76 / 76
//     T 700, heads 256 / 272, halves and 64: bf16 36 / 67, 44 / 53; fp16 47 / 89, 55 / 67; fp32 60 / 111, 75 / 142
//     fp32 T 400, 384 / 768 heads: halves 76 / 118, 64 95 / 149;  bf16 T 2048, 368 heads: 167, 130
//     64 heads, T 512 / 768: in segs 34 / 32, halves 26 / 35; training 137 / 132, 132 / 176
//   Dq > 128: halves, in segs of 256; 32 heads of 256 x 256, T 512: in segs 73, whole 48; 768 fp32: 134, 130
struct Plan { int columns, halves, segs; };
constexpr int kLeast = 256;       // steps of a segment
constexpr int kSegsFrom = 512;    // steps beyond which there are segments: two of them cost more than they give
Plan plan_of(int64_t B, int64_t T, int H, int Dq, int Dv, int dtype) {
  const int64_t heads = B * H;
  Plan p{64, 1, 1};
  if (T <= kFew || heads == 0) return p;
  int fill = 0;   // workgroups that are resident at once: segments make no more
  if (Dq > 128) { p.halves = 2; fill = 256; }
  else if (Dv > 64 && heads > 128) p.columns = 128;
  else if (Dv > 64 && heads < 96 && T > kSegsFrom) { p.columns = 128; fill = 256; }
  else if (Dv > 64) p.halves = 2;
  else if (Dq > 64) { p.halves = 2; fill = heads < 128 ? 256 : 0; }
  else if (heads < 128 && T > kSegsFrom) fill = 512;
  else if (heads <= 256 || dtype == SIM_DT_F32) p.halves = 2;
  if (T <= kSegsFrom) return p;
  const int64_t groups = heads * ((Dv + p.columns - 1) / p.columns);
  p.segs = (int)std::max<int64_t>(1, std::min<int64_t>((T + kLeast - 1) / kLeast, fill / groups));
  return p;
}
size_t parts_bytes(int64_t B, int64_t T, int H, int Dq, int Dv, int dtype) {
  const int g = plan_of(B, T, H, Dq, Dv, dtype).segs;
  return g > 1 ? (size_t)B * H * g * Dq * Dv * sizeof(float) : 0;
}

// all of a run, or of one in segments the states that they start from (and the last one), or the result from these
enum { kWhole = 0, kStates = 1, kResult = 2 };
template <class E, int DQ, int NW, int HV, int C>
hipError_t launch_runs(AttnRun r, int64_t B, int what, hipStream_t st) {
  typedef RunLds<E, DQ, NW, HV, C> Lds;
  static std::atomic<uint64_t> done[2];
  hipError_t e = allow_lds(reinterpret_cast<const void*>(&attn_run_k<E, DQ, NW, HV, C, true>), sizeof(Lds), done[0]);
  if (e == hipSuccess) e = allow_lds(reinterpret_cast<const void*>(&attn_run_k<E, DQ, NW, HV, C, false>), sizeof(Lds), done[1]);
  if (e != hipSuccess) return e;
  const int cols = (r.Dv + Lds::DV - 1) / Lds::DV;
  const dim3 grid((unsigned)(B * r.H * cols), r.segs), block(64 * NW * HV);
  if (r.segs > 1 && what != kResult) {
    hipLaunchKernelGGL((attn_run_k<E, DQ, NW, HV, C, false>), grid, block, sizeof(Lds), st, r);
    hipLaunchKernelGGL(attn_join_k, dim3((r.Dq * r.Dv + 255) / 256, (unsigned)(B * r.H)), dim3(256), 0, st, r);
    r.err = nullptr;
    if (!r.out || what == kStates) return hipSuccess;
  }
  if (r.out) hipLaunchKernelGGL((attn_run_k<E, DQ, NW, HV, C, true>), grid, block, sizeof(Lds), st, r);
  else hipLaunchKernelGGL((attn_run_k<E, DQ, NW, HV, C, false>), grid, block, sizeof(Lds), st, r);
  return hipSuccess;
}

template <class E>
hipError_t launch_run(AttnRun r, int64_t B, float* parts, int what, hipStream_t st) {
  constexpr int dt = std::is_same<E, F32>::value ? SIM_DT_F32 : (std::is_same<E, F16>::value ? SIM_DT_F16 : SIM_DT_BF16);
  if (r.T <= kFew) {
    const dim3 grid((unsigned)(B * r.H), (r.Dv + 63) / 64), block(kStep);
    if (r.Dq <= 64) hipLaunchKernelGGL((attn_step_k<E, 4>), grid, block, 0, st, r);
    else if (r.Dq <= 128) hipLaunchKernelGGL((attn_step_k<E, 8>), grid, block, 0, st, r);
    else hipLaunchKernelGGL((attn_step_k<E, 16>), grid, block, 0, st, r);
    return hipSuccess;
  }
  const Plan plan = plan_of(B, r.T, r.H, r.Dq, r.Dv, dt);
  r.segs = plan.segs;
  r.seg = r.T;
  if (r.segs > 1) {   // whole runs
    const int64_t each = (r.T + r.segs - 1) / r.segs;
    r.seg = (each + 63) / 64 * 64;
    r.segs = (int)((r.T + r.seg - 1) / r.seg);
    r.parts = parts;
    if (r.pr == 0) { r.pr = r.Dv; r.pc = 1; }
  }
  constexpr int C64 = run_steps(dt, 64), C128 = run_steps(dt, 128), C256 = run_steps(dt, 256);
  if (r.Dq > 128) return launch_runs<E, 256, 4, 2, C256>(r, B, what, st);
  if (r.Dq > 64)
    return plan.columns == 128 ? launch_runs<E, 128, 8, 1, C128>(r, B, what, st) : launch_runs<E, 128, 4, 2, C128>(r, B, what, st);
  return plan.columns == 128 ? launch_runs<E, 64, 8, 1, C64>(r, B, what, st)
         : plan.halves == 2 ? launch_runs<E, 64, 4, 2, C64>(r, B, what, st) : launch_runs<E, 64, 4, 1, C64>(r, B, what, st);
}

In in_of(const sim_heads& x, int share) { return In{x.data, x.stride_b, x.stride_t, x.stride_h, share}; }

// fp32 gradients of shared heads before they are added up
size_t share_cells(const sim_linear_attn& c, bool grad) {
  return grad && c.H > c.Hk ? ((size_t)c.B * c.T * c.H * std::max(c.Dk, c.Dv) + 3) / 4 * 4 : 0;
}

template <class E>
hipError_t launch_typed(const AttnArgs& a, bool grad, hipStream_t st) {
  const sim_linear_attn& c = a.c;
  const int g = c.H / c.Hk;
  AttnRun f{};
  f.decay = a.decay; f.len = a.len; f.err = a.err; f.T = c.T; f.H = c.H;
  f.segs = 1; f.seg = c.T;
  const In q = in_of(a.q, 1), k = in_of(a.k, g), v = in_of(a.v, g), dy = in_of(a.dy, 1);
  float* const shares = static_cast<float*>(a.work);
  float* const parts = shares + share_cells(c, grad);
  auto dims = [&](AttnRun& r, int Dq, int Dv, bool turned) {   // turned: states are [Dv][Dq] in memory
    r.Dq = Dq; r.Dv = Dv;
    r.sr = turned ? 1 : Dv; r.sc = turned ? Dq : 1;
  };
  auto out = [&](AttnRun& r, const sim_heads& o) {
    r.out = c.T ? o.data : nullptr; r.ob = o.stride_b; r.ot = o.stride_t; r.oh = o.stride_h;
  };
  if (!grad) {
    AttnRun r = f;
    r.q = q; r.k = k; r.v = v;
    dims(r, c.Dk, c.Dv, false);
    out(r, a.y);
    r.s0 = a.s0; r.state = a.state; r.so = c.scale; r.su = 1.0f;
    return launch_run<E>(r, c.B, parts, kWhole, st);
  }
  hipError_t e = hipSuccess;
  // lengths and decays are told of by the first run there is
  if (a.dq.data) {
    AttnRun r = f;
    r.q = dy; r.k = v; r.v = k;
    dims(r, c.Dv, c.Dk, true);
    out(r, a.dq);
    r.s0 = a.s0; r.so = c.scale; r.su = 1.0f;
    if ((e = launch_run<E>(r, c.B, parts, kWhole, st)) != hipSuccess) return e;
    f.err = nullptr;
  }
  f.back = true; f.lag = 1; f.so = 1.0f; f.su = c.scale;
  AttnRun rk = f, rv = f;
  rk.q = v; rk.k = dy; rk.v = q;
  rk.s0 = rv.s0 = a.ds;
  dims(rk, c.Dv, c.Dk, true);
  rv.q = k; rv.k = q; rv.v = dy;
  dims(rv, c.Dk, c.Dv, false);
  // Both go by the same states, each other's turned: in segments they are formed once, for either alone too, so that
  // a gradient is the same whichever others are wanted.
  const int segs = plan_of(c.B, c.T, c.H, c.Dv, c.Dk, c.dtype).segs;
  int what = kWhole;
  if (segs > 1 && segs == plan_of(c.B, c.T, c.H, c.Dk, c.Dv, c.dtype).segs && (a.dk.data || a.dv.data || a.state)) {
    AttnRun r = rk;
    r.state = a.state;
    if ((e = launch_run<E>(r, c.B, parts, kStates, st)) != hipSuccess) return e;
    rk.err = rv.err = nullptr;
    rv.pr = 1; rv.pc = c.Dk;
    what = kResult;
  } else {
    rv.state = a.state;
  }
  auto shared = [&](AttnRun& r, const sim_heads& o, int D) {
    out(r, o);
    if (g == 1 || !r.out) return launch_run<E>(r, c.B, parts, what, st);
    r.out = shares; r.wide = true;
    r.oh = D; r.ot = (int64_t)c.H * D; r.ob = c.T * r.ot;
    const hipError_t e = launch_run<E>(r, c.B, parts, what, st);
    if (e != hipSuccess) return e;
    const int64_t cells = c.B * c.T * c.Hk * D;
    hipLaunchKernelGGL(attn_share_k<E>, dim3((unsigned)std::min<int64_t>((cells + 255) / 256, 1 << 16)), dim3(256), 0, st,
                       shares, o, cells, c.T, c.Hk, g, D);
    return hipSuccess;
  };
  if (a.dk.data) {
    if ((e = shared(rk, a.dk, c.Dk)) != hipSuccess) return e;
    rv.err = nullptr;
  }
  if (a.dv.data || rv.state) e = shared(rv, a.dv, c.Dv);   // the last one: ds0 may be written over dstate
  return e;
}

}  // namespace

size_t attn_work_bytes(const sim_linear_attn& c, bool grad) {
  size_t parts = parts_bytes(c.B, c.T, c.H, c.Dk, c.Dv, c.dtype);
  if (grad) parts = std::max(parts, parts_bytes(c.B, c.T, c.H, c.Dv, c.Dk, c.dtype));
  return share_cells(c, grad) * sizeof(float) + parts;
}

hipError_t launch_attn(const AttnArgs& a, bool grad, hipStream_t st) {
  const hipError_t e = a.c.dtype == SIM_DT_F32 ? launch_typed<F32>(a, grad, st)
                       : a.c.dtype == SIM_DT_BF16 ? launch_typed<BF16>(a, grad, st) : launch_typed<F16>(a, grad, st);
  return e == hipSuccess ? hipGetLastError() : e;
}

}  // namespace bsim
