// scan_kernels.hip -- the gated linear recurrence and its gradient over [B][T][D].
//
//   linear   h = g_t h + x_t,        sigmoid  f = 1/(1 + exp(-g_t)), h = f h + (1 - f) x_t
//
// A run of steps maps the state h before it to A h + X, with A the product of its gates and X its
// result from 0; two runs in a row join to (A2 A1, A2 X1 + X2). So a workgroup takes a tile of
// segments, a thread each: it scans its segment from 0 in registers, the segments' (A, X) are
// scanned across the workgroup, and each thread then adds A_l times the state that its segment starts
// from. Each element is read once and written once; a multiplication and an addition per element
// (and a sigmoid): bound by HBM. The price is that the products A must stay in the type's range, which with
// |gate| <= 1 they do, or fall to 0 where what they carry no longer counts (an infinite one times a state
// of 0 is NaN).
//
// Positions p = 0..T-1 are taken in processing order, t = p, or from the end. Padding is the
// identity (A, X) = (1, 0), so the state passes through it on either side of a sequence.
#include <algorithm>

#include "ops_dev.hpp"

namespace bsim {
namespace {

constexpr int kLogThreads = 8, kThreads = 1 << kLogThreads, kWaves = kThreads / 64;

__device__ __forceinline__ float fma_w(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ double fma_w(double a, double b, double c) { return fma(a, b, c); }

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

__device__ __forceinline__ int seq_len(const ScanArgs& s, int64_t b, bool tell) {
  const int T = (int)s.c.T;
  if (!s.len) return T;
  int n = s.len[b];
  if (n < 0 || n > T) {
    if (tell) atomicOr(s.err, ERR_LENGTH);
    n = n < 0 ? 0 : T;
  }
  return n;
}

// How a launch cuts its arrays. Channels adjacent (time = 0): a thread has L steps of V channels,
// 1 << lx threads stand beside each other along the channels and the others along the steps. One
// channel whose steps are adjacent (time = 1): a thread has L adjacent steps, a sequence has
// 1 << gs threads.
struct ScanPlan {
  int time, vec;      // vec (time = 1): the steps of every array in use are adjacent
  int lx, gs;
  int64_t tiles;      // workgroups side by side
  int64_t per;        // time = 0: channel tiles of a sequence
  int chunks;         // time-wise pieces, each a workgroup that goes over `ctiles` tiles
  int ctiles;
  int runs;           // tile_of
};

// N elements, in registers and (at any alignment of the element) in memory
template <class T, int N>
struct VecOf {
  typedef T V __attribute__((ext_vector_type(N)));
  typedef T M __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <class T>
struct VecOf<T, 1> { typedef T V; typedef T M; };
template <class T, int N>
__device__ __forceinline__ typename VecOf<T, N>::V read(const T* p) {
  return __builtin_bit_cast(typename VecOf<T, N>::V, *reinterpret_cast<const typename VecOf<T, N>::M*>(p));
}
template <class T, int N>
__device__ __forceinline__ void write(T* p, typename VecOf<T, N>::V v) {
  *reinterpret_cast<typename VecOf<T, N>::M*>(p) = __builtin_bit_cast(typename VecOf<T, N>::M, v);
}

// What a thread is to its tile.
struct Place {
  int unit, segw, nsw;   // lanes from one segment to the next; its place in the wave; their number
  int wave, wv, nwv;     // its wave in the workgroup and in the scan, and their number
  int seg, nseg;         // its segment in the tile
  int col;               // its column of the scan's LDS
};
__device__ __forceinline__ Place place_of(const ScanPlan& p) {
  Place q;
  const int tid = threadIdx.x, lane = tid & 63;
  q.wave = tid >> 6;
  if (p.time) {
    const int gs = 1 << p.gs;
    q.unit = 1;
    q.nsw = gs < 64 ? gs : 64;
    q.segw = lane & (q.nsw - 1);
    q.nwv = gs < 64 ? 1 : gs >> 6;
    q.wv = q.wave & (q.nwv - 1);
    q.seg = tid & (gs - 1);
    q.nseg = gs;
    q.col = 0;
  } else {
    q.unit = 1 << p.lx;
    q.nsw = 64 >> p.lx;
    q.segw = lane >> p.lx;
    q.nwv = kWaves;
    q.wv = q.wave;
    q.seg = tid >> p.lx;
    q.nseg = kThreads >> p.lx;
    q.col = lane & (q.unit - 1);
  }
  return q;
}

// One run's (A, X) of V channels per thread, scanned over the tile's segments in order. On return
// (A, X) is the run of all segments of this wave before this one, and `carry`, the state at the
// tile's start, has become the state at the wave's start; total: the state at the tile's end.
// `lds` holds kWaves rows of 64 columns of V pairs and is free again after the next barrier.
template <class W, int V>
__device__ __forceinline__ void scan_tile(const Place& q, W (&A)[V], W (&X)[V], W (&carry)[V], W (&total)[V],
                                          W (*lds)[64][V][2]) {
  for (int d = 1; d < q.nsw; d <<= 1) {
    const bool take = q.segw >= d;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const W a = __shfl_up(A[v], d * q.unit), x = __shfl_up(X[v], d * q.unit);
      X[v] = take ? fma_w(A[v], x, X[v]) : X[v];
      A[v] = take ? A[v] * a : A[v];
    }
  }
  if (q.nwv > 1 && q.segw == q.nsw - 1) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      lds[q.wave][q.col][v][0] = A[v];
      lds[q.wave][q.col][v][1] = X[v];
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const W a = __shfl_up(A[v], q.unit), x = __shfl_up(X[v], q.unit);
    A[v] = q.segw > 0 ? a : (W)1;
    X[v] = q.segw > 0 ? x : (W)0;
  }
  if (q.nwv > 1) {
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) total[v] = carry[v];
    W run[kWaves][V][2];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const auto& row = lds[(q.wave - q.wv + w) & (kWaves - 1)][q.col];
#pragma unroll
      for (int v = 0; v < V; ++v) { run[w][v][0] = row[v][0]; run[w][v][1] = row[v][1]; }
    }
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        carry[v] = w == q.wv ? total[v] : carry[v];
        total[v] = w < q.nwv ? fma_w(run[w][v][0], total[v], run[w][v][1]) : total[v];
      }
    }
  }
}

// N values rounded to the element type, 16-bit ones in pairs
template <class E, int N>
__device__ __forceinline__ typename VecOf<typename E::T, N>::V round_to(const typename E::W (&w)[N]) {
  typedef typename E::W W;
  if constexpr (N == 1) {
    return (typename E::T)w[0];
  } else {
    typedef W Wide __attribute__((ext_vector_type(N)));
    Wide v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = w[i];
    typedef typename E::T Narrow __attribute__((ext_vector_type(N)));
    return __builtin_bit_cast(typename VecOf<typename E::T, N>::V, __builtin_convertvector(v, Narrow));
  }
}

// The L steps by V channels (or L adjacent steps) that a thread reads of one array.
template <class E, int V, int L, bool TV>
struct Block {
  typedef typename E::T T;
  typedef typename E::W W;
  typedef typename VecOf<T, TV ? L : V>::V Vec;
  Vec r[TV ? 1 : L];
  __device__ __forceinline__ W get(int l, int v) const {
    if constexpr (TV) return (W)r[0][l];
    else if constexpr (V == 1) return (W)r[l];
    else return (W)r[l][v];
  }
  // keeps one pass's widened values and gates from being held for the next
  __device__ __forceinline__ void forget() {
#pragma unroll
    for (Vec& v : r) hide(v);
  }
  __device__ __forceinline__ void set(int l, const W (&o)[V]) {
    if constexpr (TV) r[0][l] = (T)o[0];
    else r[l] = round_to<E, V>(o);
  }
};

// Where a thread's block lies: steps t0 + l (or t0 + L - 1 - l, back) of its channels.
struct Where {
  int t0;        // the first step in memory
  int n, T;      // steps of the sequence, of the arrays
  int d, skip;   // first channel, and how many from it are another thread's
  bool back, vec;
  __device__ __forceinline__ int t(int l, int L) const { return back ? t0 + L - 1 - l : t0 + l; }
};

// Whether a thread's steps, and those `shift` from them, all lie in the sequence, for every lane of the wave.
template <int L>
__device__ __forceinline__ bool whole(const Where& w, int shift = 0) {
  const int lo = w.t0 + (shift < 0 ? shift : 0), hi = w.t0 + L + (shift > 0 ? shift : 0);
  return __all(lo >= 0 && hi <= w.n);
}

// Reads steps t + shift; those outside the sequence (unless it is `whole` there) read some other step of
// it (or, where it has none, nothing): the caller does not use them.
template <class E, int V, int L, bool TV>
__device__ __forceinline__ void load(Block<E, V, L, TV>& blk, const sim_seq& q, int64_t b, const Where& w,
                                     bool whole, int shift = 0) {
  typedef typename E::T T;
  typedef typename Block<E, V, L, TV>::Vec Vec;
  const T* p = static_cast<const T*>(q.data) + b * q.stride_b;
  if constexpr (TV) {
    if (w.vec && shift == 0 && w.t0 >= 0 && w.t0 + L <= w.T) {
      blk.r[0] = read<T, L>(p + w.t0);
    } else if (w.n > 0) {
#pragma unroll
      for (int l = 0; l < L; ++l) {
        int t = w.t0 + l + shift;
        t = t < 0 ? 0 : (t >= w.n ? w.n - 1 : t);
        blk.r[0][l] = p[(int64_t)t * q.stride_t];
      }
    }
    if (w.back) {
      Vec o = blk.r[0];
#pragma unroll
      for (int l = 0; l < L; ++l) blk.r[0][l] = o[L - 1 - l];
    }
  } else if (whole) {
    const int64_t step = w.back ? -q.stride_t : q.stride_t;
    p += (int64_t)(w.t(0, L) + shift) * q.stride_t + w.d;
#pragma unroll
    for (int l = 0; l < L; ++l) blk.r[l] = read<T, V>(p + l * step);
  } else if (w.n > 0) {
#pragma unroll
    for (int l = 0; l < L; ++l) {
      int t = w.t(l, L) + shift;
      t = t < 0 ? 0 : (t >= w.n ? w.n - 1 : t);
      blk.r[l] = read<T, V>(p + (int64_t)t * q.stride_t + w.d);
    }
  }
}

template <class E, int V, int L, bool TV>
__device__ __forceinline__ void store(const Block<E, V, L, TV>& blk, const sim_seq& q, int64_t b, const Where& w,
                                      bool whole) {
  typedef typename E::T T;
  typedef typename Block<E, V, L, TV>::Vec Vec;
  T* p = static_cast<T*>(q.data) + b * q.stride_b;
  if constexpr (TV) {
    Vec o = blk.r[0];
    if (w.back) {
#pragma unroll
      for (int l = 0; l < L; ++l) o[l] = blk.r[0][L - 1 - l];
    }
    if (w.vec && w.t0 >= 0 && w.t0 + L <= w.T) {
      write<T, L>(p + w.t0, o);
    } else {
#pragma unroll
      for (int l = 0; l < L; ++l)
        if (w.t0 + l >= 0 && w.t0 + l < w.T) p[(int64_t)(w.t0 + l) * q.stride_t] = o[l];
    }
  } else {
#pragma unroll
    for (int l = 0; l < L; ++l) {
      const int t = w.t(l, L);
      if (!whole && (t < 0 || t >= w.T)) continue;
      T* at = p + (int64_t)t * q.stride_t + w.d;
      if (w.skip == 0) {
        write<T, V>(at, blk.r[l]);
      } else if constexpr (V > 1) {
#pragma unroll
        for (int v = 1; v < V; ++v)
          if (v >= w.skip) at[v] = blk.r[l][v];
      }
    }
  }
}

// The block of position p: for one channel whose steps are adjacent, blocks start at multiples
// of L in memory in either direction (the first one back is cut off by T instead).
template <int L, bool TV>
__device__ __forceinline__ int first_step(int p, int T, bool back) {
  const int end = TV ? (T + L - 1) / L * L : T;
  int t = back ? end - L - p : p;
  fresh(t);
  return t;
}

// LDS rows of the scan, two so that one barrier per tile is enough
template <class W, int V>
struct ScanLds { W v[2][kWaves][64][V][2]; };

// Workgroups are dealt out to the eight XCDs in turn. Where rows do not start on cache lines, neighbours
// share lines, so each XCD gets a run of tiles: the one that workgroup i of n takes (fp64 1365 x 26762
// 284 -> 223 us; rows on lines the other way: fp32 1025 x 16 x 1536 153 in turn, 162 in runs).
__device__ __forceinline__ int64_t tile_of(const ScanPlan& p, int64_t i) {
  if (!p.runs) return i;
  const int64_t each = p.tiles >> 3, rest = p.tiles & 7, x = i & 7;
  return x * each + (x < rest ? x : rest) + (i >> 3);
}

// The chunks are taken from the last one on, whose inputs the launch before this one read last and left in
// the caches (bf16 1 x 65536 x 512 training step 236 -> 230 us, fp16 4 x 5995 x 381 71 -> 69).
__device__ __forceinline__ int chunk_of(const ScanPlan& p) { return p.chunks - 1 - (int)blockIdx.y; }

// What a workgroup's thread is in the whole launch. The last thread of a row takes the last V channels,
// the first `skip` of which its neighbour writes; threads past the row (skip = V) write none.
struct Job {
  int64_t b;
  int d, skip;
  bool live;
};
template <int V, bool TV>
__device__ __forceinline__ Job job_of(const ScanPlan& p, const Place& q, const sim_scan& c, int64_t blk) {
  Job j;
  if (TV) {
    j.b = (blk << (kLogThreads - p.gs)) + (threadIdx.x >> p.gs);
    j.d = j.skip = 0;
    j.live = j.b < c.B;
    if (!j.live) j.b = c.B - 1;
  } else {
    j.b = blk / p.per;
    const int64_t d = (((blk % p.per) << p.lx) + q.col) * V;
    j.live = d < c.D;
    j.d = (int)(d < c.D - V ? d : c.D - V);
    j.skip = (int)(d - j.d < V ? d - j.d : V);
  }
  return j;
}

// The states before each chunk are found from the chunks' runs, which a launch before this one left
// in the work memory: slot 0 holds the state before the first, slot i + 1 the run of chunk i.
template <class W>
__device__ __forceinline__ W* slot(const ScanArgs& s, int64_t i) {
  return static_cast<W*>(s.work) + i * 2 * s.c.B * s.c.D;
}

template <class W, int V>
__device__ __forceinline__ void state_before(const ScanArgs& s, const ScanPlan& p, const Place& q, const Job& j,
                                             int chunk, const void* first, W (&h)[V], ScanLds<W, V>& lds) {
  const int64_t at = j.b * s.c.D + j.d, n = s.c.B * s.c.D;
  const W* h0 = p.chunks > 1 ? slot<W>(s, 0) : static_cast<const W*>(first);
#pragma unroll
  for (int v = 0; v < V; ++v) h[v] = h0 ? h0[at + v] : (W)0;
  for (int base = 0; base < chunk; base += q.nseg) {
    const int i = base + q.seg;
    W A[V], X[V], end[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const bool has = i < chunk;
      A[v] = has ? slot<W>(s, i + 1)[at + v] : (W)1;
      X[v] = has ? slot<W>(s, i + 1)[n + at + v] : (W)0;
    }
    __syncthreads();
    scan_tile<W, V>(q, A, X, h, end, lds.v[0]);
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = end[v];
  }
  __syncthreads();
}

// A chunk's run: each thread takes a contiguous part of it, then one scan. Its inputs are read again by the
// launch after it, the price of splitting a sequence: 13 passes over an array in a training step instead of
// 9, which fills a chip that 8 workgroups would leave empty (bf16 1 x 65536 x 512: 38 us, 3.5 TB/s; gradient
// 29 us, 4.6 TB/s).
template <class E, bool SIG, int V, int L, bool TV, bool GRAD>
__global__ __launch_bounds__(kThreads) void scan_runs_k(ScanArgs s, ScanPlan p) {
  typedef typename E::W W;
  __shared__ ScanLds<W, V> lds;
  const Place q = place_of(p);
  const bool back = GRAD ? !s.c.reverse : s.c.reverse != 0;
  const Job j = job_of<V, TV>(p, q, s.c, tile_of(p, blockIdx.x));
  const int n = seq_len(s, j.b, false), T = (int)s.c.T;
  const int64_t at = j.b * s.c.D + j.d, bd = s.c.B * s.c.D;
  W A[V], X[V];
#pragma unroll
  for (int v = 0; v < V; ++v) { A[v] = (W)1; X[v] = (W)0; }
  const int p0 = ((int)blockIdx.y * q.nseg + q.seg) * p.ctiles * L;
  for (int i = 0; i < p.ctiles; ++i) {
    Where w{first_step<L, TV>(p0 + i * L, T, back), n, T, j.d, j.skip, back, p.vec != 0};
    const bool all = whole<L>(w);
    Block<E, V, L, TV> g{}, x{};
    load(g, s.g, j.b, w, all);
    load(x, GRAD ? s.dy : s.x, j.b, w, all);
    either(all, [&](auto ALL) {
#pragma unroll
      for (int l = 0; l < L; ++l) {
        const int t = w.t(l, L);
        const bool on = ALL || (t >= 0 && t < n);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          W a, r;
          gate_of<W, SIG>(g.get(l, v), a, r);
          // gradient: C = a (dy + C)
          const W nx = GRAD ? a * (x.get(l, v) + X[v]) : fma_w(a, X[v], r * x.get(l, v));
          X[v] = on ? nx : X[v];
          A[v] = on ? A[v] * a : A[v];
        }
      }
    });
  }
  W carry[V], end[V], run[V];
#pragma unroll
  for (int v = 0; v < V; ++v) { carry[v] = (W)0; run[v] = A[v]; }
  // the product of all gates: the same scan with the inputs left out, from 1
  W A2[V], Z[V], one[V];
#pragma unroll
  for (int v = 0; v < V; ++v) { A2[v] = run[v]; Z[v] = (W)0; one[v] = (W)1; }
  scan_tile<W, V>(q, A, X, carry, end, lds.v[0]);
  W prod[V];
  scan_tile<W, V>(q, A2, Z, one, prod, lds.v[1]);
  if (q.seg == 0 && j.live) {
    const void* first = GRAD ? s.ds : s.h0;
    W* o = slot<W>(s, blockIdx.y + 1);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (v < j.skip) continue;
      o[at + v] = prod[v];
      o[bd + at + v] = end[v];
      if (blockIdx.y == 0) slot<W>(s, 0)[at + v] = first ? static_cast<const W*>(first)[at + v] : (W)0;
    }
  }
}

// The recurrence: a segment's products and states stay in registers (64 of them) between the pass from 0 and
// the one that adds the state before it; the next tile's loads fly under the scan. Bound by HBM with many
// workgroups (fp32 16 x 1025 x 1536 72 us, 4.2 TB/s; fp64 1 x 4000 x 8192 157 us, 5.0; one channel, fp32
// 4096 x 4096 38 us, 5.3; with half of the steps padding, which is not read but goes through the scan, the first
// 63 us, 3.3 TB/s), by the latency of a tile (loads, scan, barrier) with the one a CU that 2048 bf16
// channels of 8 sequences make: 61 us, 3.3 TB/s. Splitting those over time instead reads twice (88 us for
// as many elements); two tiles ahead, 512 threads or wider pieces of a row are slower (62, 58, 75).
template <class E, bool SIG, int V, int L, bool TV>
__global__ __launch_bounds__(kThreads) void scan_tile_k(ScanArgs s, ScanPlan p) {
  typedef typename E::W W;
  __shared__ ScanLds<W, V> lds;
  const Place q = place_of(p);
  const int chunk = chunk_of(p);
  const bool back = s.c.reverse != 0;
  for (int64_t blk = blockIdx.x; blk < p.tiles; blk += gridDim.x) {
    const Job j = job_of<V, TV>(p, q, s.c, tile_of(p, blk));
    const int n = seq_len(s, j.b, q.seg == 0 && chunk == 0), T = (int)s.c.T;
    const int64_t at = j.b * s.c.D + j.d;
    W h[V];
    state_before<W, V>(s, p, q, j, chunk, s.h0, h, lds);
    const int span = q.nseg * L;
    const int p0 = chunk * p.ctiles * span + q.seg * L;
    Where w{first_step<L, TV>(p0, T, back), n, T, j.d, j.skip, back, p.vec != 0};
    Block<E, V, L, TV> g{}, x{};
    bool all = whole<L>(w);
    load(g, s.g, j.b, w, all);
    load(x, s.x, j.b, w, all);
    for (int i = 0; i < p.ctiles; ++i) {
      // the segment from a state of 0, and its gates' products
      W A[L][V], X[L][V];
      either(all, [&](auto ALL) {
#pragma unroll
        for (int l = 0; l < L; ++l) {
          const int t = w.t(l, L);
          const bool on = ALL || (t >= 0 && t < n);
#pragma unroll
          for (int v = 0; v < V; ++v) {
            W a, r;
            gate_of<W, SIG>(g.get(l, v), a, r);
            W u = r * x.get(l, v);
            a = on ? a : (W)1;
            u = on ? u : (W)0;
            A[l][v] = l ? A[l - (l > 0)][v] * a : a;
            X[l][v] = l ? fma_w(a, X[l - (l > 0)][v], u) : u;
          }
        }
      });
      const Where now = w;
      const bool now_all = all;
      if (i + 1 < p.ctiles) {   // the next tile's loads fly during the scan
        w.t0 = first_step<L, TV>(p0 + (i + 1) * span, T, back);
        all = whole<L>(w);
        load(g, s.g, j.b, w, all);
        load(x, s.x, j.b, w, all);
      }
      W a[V], u[V], end[V];
#pragma unroll
      for (int v = 0; v < V; ++v) { a[v] = A[L - 1][v]; u[v] = X[L - 1][v]; }
      scan_tile<W, V>(q, a, u, h, end, lds.v[i & 1]);
      Block<E, V, L, TV> y;
      W in[V];
#pragma unroll
      for (int v = 0; v < V; ++v) in[v] = fma_w(a[v], h[v], u[v]);
      either(now_all, [&](auto ALL) {
#pragma unroll
        for (int l = 0; l < L; ++l) {
          const int t = now.t(l, L);
          const bool on = ALL || (t >= 0 && t < n);
          W o[V];
#pragma unroll
          for (int v = 0; v < V; ++v) o[v] = on ? fma_w(A[l][v], in[v], X[l][v]) : (W)0;
          y.set(l, o);
        }
      });
      if (s.y.data && j.live) store(y, s.y, j.b, now, now_all);
      // where the sequence's last step is, the state after it, as y has it
      const int tl = back ? 0 : n - 1;
      const bool none = n == 0 && i == 0 && chunk == 0 && q.seg == 0;
      if (s.state && j.live && (none || (n > 0 && now.t0 <= tl && tl < now.t0 + L))) {
        W last[V];
#pragma unroll
        for (int v = 0; v < V; ++v) last[v] = in[v];
#pragma unroll
        for (int l = 0; l < L; ++l) {
#pragma unroll
          for (int v = 0; v < V; ++v)
            last[v] = !none && now.t(l, L) == tl ? fma_w(A[l][v], in[v], X[l][v]) : last[v];
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (v >= j.skip) static_cast<W*>(s.state)[at + v] = last[v];
      }
      if (q.nwv > 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = end[v];
      }
    }
    __syncthreads();
  }
}

// The gradient, against the order of the states: C, what later steps ask of a state, goes through the same
// scan (C = a (dy + C)), and a second pass over the raw elements, kept in registers, makes dg and dx. It
// computes the gates twice: keeping them takes 30 registers and a third of the waves (bf16 16 x 1024 x 4096
// step 317 us, 305 so). Bound by HBM: fp32 16 x 1025 x 1536 119 us for five arrays, 4.2 TB/s (half of
// the steps padding 96 us, 3.7); bf16 1 x 65536 x 512 111 us for six, 3.6 TB/s in chunks. The next tile's loads under the
// scan help unaligned rows by 5% and cost aligned ones as much (187 against 181 us): not done.
template <class E, bool SIG, int V, int L, bool TV>
__global__ __launch_bounds__(kThreads) void scan_grad_k(ScanArgs s, ScanPlan p) {
  typedef typename E::W W;
  __shared__ ScanLds<W, V> lds;
  const Place q = place_of(p);
  const int chunk = chunk_of(p);
  const bool back = !s.c.reverse;
  for (int64_t blk = blockIdx.x; blk < p.tiles; blk += gridDim.x) {
    const Job j = job_of<V, TV>(p, q, s.c, tile_of(p, blk));
    const int n = seq_len(s, j.b, q.seg == 0 && chunk == 0), T = (int)s.c.T;
    const int64_t at = j.b * s.c.D + j.d;
    W C[V], h0[V];
    state_before<W, V>(s, p, q, j, chunk, s.ds, C, lds);
#pragma unroll
    for (int v = 0; v < V; ++v) h0[v] = s.h0 && s.dg.data ? static_cast<const W*>(s.h0)[at + v] : (W)0;
    const int span = q.nseg * L;
    const int p0 = chunk * p.ctiles * span + q.seg * L;
    for (int i = 0; i < p.ctiles; ++i) {
      const Where w{first_step<L, TV>(p0 + i * span, T, back), n, T, j.d, j.skip, back, p.vec != 0};
      Block<E, V, L, TV> g{}, dy{}, y{}, x{};
      const int before = s.c.reverse ? 1 : -1;   // from a step to the one whose state it starts from
      const bool all = whole<L>(w, before);
      load(g, s.g, j.b, w, all);
      load(dy, s.dy, j.b, w, all);
      if (s.dg.data) {
        load(y, s.y, j.b, w, all, before);
        if (SIG) load(x, s.x, j.b, w, all);
      }
      W a[V], u[V], end[V];
#pragma unroll
      for (int v = 0; v < V; ++v) { a[v] = (W)1; u[v] = (W)0; }
      either(all, [&](auto ALL) {
#pragma unroll
        for (int l = 0; l < L; ++l) {
          const int t = w.t(l, L);
          const bool on = ALL || (t >= 0 && t < n);
#pragma unroll
          for (int v = 0; v < V; ++v) {
            W f, r;
            gate_of<W, SIG>(g.get(l, v), f, r);
            const W nu = f * (dy.get(l, v) + u[v]);
            u[v] = on ? nu : u[v];
            a[v] = on ? a[v] * f : a[v];
          }
        }
      });
      scan_tile<W, V>(q, a, u, C, end, lds.v[i & 1]);
      Block<E, V, L, TV> og, ox;
      g.forget();
      dy.forget();
      W c[V];
#pragma unroll
      for (int v = 0; v < V; ++v) c[v] = fma_w(a[v], C[v], u[v]);
      either(all, [&](auto ALL) {
#pragma unroll
        for (int l = 0; l < L; ++l) {
          const int t = w.t(l, L), tp = t + before;
          const bool on = ALL || (t >= 0 && t < n), has = ALL || (tp >= 0 && tp < n);
          W wg[V], wx[V];
#pragma unroll
          for (int v = 0; v < V; ++v) {
            W f, r;
            gate_of<W, SIG>(g.get(l, v), f, r);
            const W G = dy.get(l, v) + c[v];
            const W hp = has ? y.get(l, v) : h0[v];
            wx[v] = on ? r * G : (W)0;
            wg[v] = on ? (SIG ? G * (hp - x.get(l, v)) * (f * r) : G * hp) : (W)0;
            c[v] = on ? f * G : c[v];
          }
          ox.set(l, wx);
          og.set(l, wg);
        }
      });
      if (j.live) {
        if (s.dg.data) store(og, s.dg, j.b, w, all);
        if (s.dx.data) store(ox, s.dx, j.b, w, all);
        if (i + 1 == p.ctiles && chunk + 1 == p.chunks && s.state && q.seg == q.nseg - 1) {
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (v >= j.skip) static_cast<W*>(s.state)[at + v] = c[v];
        }
      }
      if (q.nwv > 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) C[v] = end[v];
      }
    }
    __syncthreads();
  }
}

// A few steps (serving: one): a thread has V channels and takes them in turn; bound by the launch (bf16
// 64 x 1 x 2048 2.3 us), and from about 1000 workgroups on by HBM (512 x 1 x 8192 11.7 us, 5.0 TB/s).
template <class E, bool SIG, int V>
__global__ __launch_bounds__(kThreads) void scan_step_k(ScanArgs s) {
  typedef typename E::T T;
  typedef typename E::W W;
  typedef typename VecOf<T, V>::V Vec;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, per = s.c.D / V;
  if (i >= s.c.B * per) return;
  const int64_t b = i / per, d = i % per * V, at = b * s.c.D + d;
  const int n = seq_len(s, b, d == 0);
  const T* g = static_cast<const T*>(s.g.data) + b * s.g.stride_b + d;
  const T* x = static_cast<const T*>(s.x.data) + b * s.x.stride_b + d;
  T* y = static_cast<T*>(s.y.data) + b * s.y.stride_b + d;
  W h[V];
#pragma unroll
  for (int v = 0; v < V; ++v) h[v] = s.h0 ? static_cast<const W*>(s.h0)[at + v] : (W)0;
  for (int64_t p = 0; p < s.c.T; ++p) {
    const int64_t t = s.c.reverse ? s.c.T - 1 - p : p;
    Vec out{};
    if (t < n) {
      const Vec gv = read<T, V>(g + t * s.g.stride_t), xv = read<T, V>(x + t * s.x.stride_t);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        W a, r;
        if constexpr (V == 1) {
          gate_of<W, SIG>((W)gv, a, r);
          h[v] = fma_w(a, h[v], r * (W)xv);
          out = (T)h[v];
        } else {
          gate_of<W, SIG>((W)gv[v], a, r);
          h[v] = fma_w(a, h[v], r * (W)xv[v]);
          out[v] = (T)h[v];
        }
      }
    }
    if (s.y.data) write<T, V>(y + t * s.y.stride_t, out);
  }
  if (s.state) {
#pragma unroll
    for (int v = 0; v < V; ++v) static_cast<W*>(s.state)[at + v] = h[v];
  }
}

// ---- plans ------------------------------------------------------------------------------------
constexpr int kStepT = 4;             // up to this many steps, step after step
constexpr int kChans = 4;             // channels of an access, at most 16 bytes
constexpr int kHold = 64;             // bytes of an array that a thread holds so: L steps
constexpr int kHoldG = 16;            // at most so many elements in the gradient, which holds four arrays
constexpr int kSteps1 = 16, kStepsG1 = 8;   // L of single elements along the channels
constexpr int kStepsT = 8;            // L along time
constexpr int kRow = 128;             // a cache line
constexpr int kEnough = 200;          // workgroups that keep HBM busy
constexpr int kWant = 512;            // of a sequence split over time
constexpr int64_t kMaxGrid = 1 << 22;

int ceil_log2(int64_t x) {
  int r = 0;
  while (((int64_t)1 << r) < x) ++r;
  return r;
}

int elem_bytes(const sim_scan& c) { return c.dtype == SIM_DT_F64 ? 8 : (c.dtype == SIM_DT_F32 ? 4 : 2); }
constexpr int vec_channels(int eb) { return kChans * eb < 16 ? kChans : 16 / eb; }
constexpr int vec_steps(int eb, bool grad) {
  return (grad && kHold / eb > kHoldG ? kHoldG : kHold / eb) / vec_channels(eb);
}

// workgroups side by side if 1 << lx threads share a row
int64_t tiles_of(const sim_scan& c, int V, int lx) {
  const int64_t chans = (int64_t)V << lx;
  return c.B * ((c.D + chans - 1) / chans);
}
// How much of a row a workgroup takes: a cache line if that leaves enough workgroups (the gradient, which
// loads nothing ahead, needs more). With fewer channels narrower pieces, down to 16 bytes, as long as
// that is enough or the sequence is short; otherwise lines again, and time is split. With many channels
// wider pieces, whose scans have fewer segments, for the larger types. Us at pieces of 16, 32, 64, 128,
// 256, 512, 1024 bytes (forward or, t, with the gradient):
//   fp64 1 x 1000 x 256   6.1   6.8   9.7   9.4   9.7  13   27     fp64 1 x 990 x 1218   14.5 13.5 17.4 17.3 19  19  24
//   fp64 1 x 2000 x 4000  78    55    42    39    58   60   63     fp64 1 x 1365 x 26752 -    508  283  209  -   182 164
//   bf16 4 x 500 x 512    6.8   6.7   9.4   12.9  14   19   30     bf16 11 x 3232 x 153  23.8 29.7 26.6 26.6 36  47  47
//   t fp32 2 x 2000 x 1024  45  38    47    44    46   62  109     t bf16 1 x 8000 x 1024  86 71   66   67   94  188 430
//   fp32 1 x 1365 x 26752  184 135   114   101    92   94  145     t bf16 8 x 2048 x 2048  249 217 181  221  220 222 211
int row_threads(const sim_scan& c, bool grad, int V, int L) {
  const int piece = V * elem_bytes(c), line = ceil_log2(kRow / piece);
  int lx = line;
  if (tiles_of(c, V, lx) >= (grad ? 2 * kEnough : kEnough)) {
    const int widest = grad ? lx : (piece / V == 8 ? lx + 3 : (piece / V == 4 ? lx + 1 : lx));
    const int64_t enough = piece / V == 8 ? kEnough : 2 * kEnough;
    while (lx < std::min(widest, 6) && tiles_of(c, V, lx + 1) >= enough) ++lx;
    return lx;
  }
  const int narrowest = ceil_log2(std::max(1, 16 / piece));
  while (lx > narrowest) {
    --lx;
    if (tiles_of(c, V, lx) >= kEnough) return lx;
  }
  return (int64_t)(kThreads >> lx) * L * 2 >= c.T ? lx : line;
}

ScanPlan plan_of(const sim_scan& c, bool grad, bool time, bool vec) {
  const int eb = elem_bytes(c), V = time || c.D < vec_channels(eb) ? 1 : vec_channels(eb);
  ScanPlan p{};
  p.time = time;
  p.vec = vec;
  int64_t total;   // tiles of a sequence, in time
  if (time) {
    p.gs = std::min(kLogThreads, ceil_log2((c.T + kStepsT - 1) / kStepsT));
    const int rows = kThreads >> p.gs;
    p.tiles = (c.B + rows - 1) / rows;
    p.per = 1;
    total = ((c.T + kStepsT - 1) / kStepsT + (1 << p.gs) - 1) >> p.gs;
  } else {
    const int L = V > 1 ? vec_steps(eb, grad) : (grad ? kStepsG1 : kSteps1);
    const int64_t wide = (c.D + V - 1) / V;   // threads that the channels need
    p.lx = std::min(ceil_log2(wide), row_threads(c, grad, V, L));
    // shorter sequences: more channels and fewer segments
    while (p.lx < 6 && ((int64_t)1 << p.lx) < wide && (int64_t)(kThreads >> p.lx) * L >= 2 * c.T &&
           tiles_of(c, V, p.lx) >= 2 * kEnough) ++p.lx;
    const int64_t chans = (int64_t)V << p.lx, span = (int64_t)(kThreads >> p.lx) * L;
    p.per = (c.D + chans - 1) / chans;
    p.tiles = c.B * p.per;
    total = (c.T + span - 1) / span;
  }
  if (total < 1) total = 1;
  int64_t want = p.tiles ? kWant / p.tiles : 1;
  if (p.tiles >= kEnough || total < 4) want = 1;
  if (want > total) want = total;
  p.ctiles = (int)((total + want - 1) / want);
  p.chunks = (int)((total + p.ctiles - 1) / p.ctiles);
  return p;
}

size_t plan_bytes(const sim_scan& c, const ScanPlan& p) {
  if (p.chunks <= 1) return 0;
  return (size_t)(p.chunks + 1) * 2 * c.B * c.D * (c.dtype == SIM_DT_F64 ? 8 : 4);
}

// whether every row of every array in use starts on a cache line
bool on_lines(const ScanArgs& a) {
  const int eb = elem_bytes(a.c);
  for (const sim_seq* q : {&a.g, &a.x, &a.y, &a.dy, &a.dg, &a.dx})
    if (q->data && (reinterpret_cast<uintptr_t>(q->data) % 128 || (a.c.B > 1 && q->stride_b * eb % 128) ||
                    (a.c.T > 1 && q->stride_t * eb % 128)))
      return false;
  return true;
}

template <class E, bool SIG, int V, int L, int LG, bool TV>
void run(const ScanArgs& a, bool grad, bool vec, hipStream_t st) {
  ScanPlan p = plan_of(a.c, grad, TV, vec);
  p.runs = !TV && (!on_lines(a) || (V * elem_bytes(a.c) << p.lx) < kRow);
  const dim3 grid((unsigned)std::min<int64_t>(p.tiles, kMaxGrid), (unsigned)p.chunks), block(kThreads);
  if (p.chunks > 1) {
    const dim3 runs((unsigned)p.tiles, (unsigned)p.chunks - 1);
    if (grad) hipLaunchKernelGGL((scan_runs_k<E, SIG, V, LG, TV, true>), runs, block, 0, st, a, p);
    else hipLaunchKernelGGL((scan_runs_k<E, SIG, V, L, TV, false>), runs, block, 0, st, a, p);
  }
  if (grad) hipLaunchKernelGGL((scan_grad_k<E, SIG, V, LG, TV>), grid, block, 0, st, a, p);
  else hipLaunchKernelGGL((scan_tile_k<E, SIG, V, L, TV>), grid, block, 0, st, a, p);
}

template <class E, bool SIG>
hipError_t go(ScanArgs a, bool grad, hipStream_t st) {
  constexpr int eb = sizeof(typename E::T), V = vec_channels(eb);
  // sequences side by side in every array are channels (lengths apart)
  bool flat = a.c.B > 1 && !a.len;
  for (const sim_seq* q : {&a.g, &a.x, &a.y, &a.dy, &a.dg, &a.dx})
    if (q->data && q->stride_b != a.c.D) flat = false;
  if (flat) {
    a.c.D *= a.c.B;
    a.c.B = 1;
  }
  bool time = a.c.D == 1 && a.c.T > 1, adjacent = true;
  for (const sim_seq* q : {&a.g, &a.x, &a.y, &a.dy, &a.dg, &a.dx}) {
    if (!q->data) continue;
    if (q->stride_t > 1) time = false;
    if (q->stride_t != 1) adjacent = false;
  }
  if (!grad && a.c.T <= kStepT) {
    const bool v = a.c.D % V == 0;
    const int64_t n = a.c.B * (v ? a.c.D / V : a.c.D);
    const dim3 grid((unsigned)((n + kThreads - 1) / kThreads)), block(kThreads);
    if (v) hipLaunchKernelGGL((scan_step_k<E, SIG, V>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((scan_step_k<E, SIG, 1>), grid, block, 0, st, a);
  } else if (time) {
    run<E, SIG, 1, kStepsT, kStepsT, true>(a, grad, adjacent, st);
  } else if (a.c.D >= V) {
    run<E, SIG, V, vec_steps(eb, false), vec_steps(eb, true), false>(a, grad, true, st);
  } else {
    run<E, SIG, 1, kSteps1, kStepsG1, false>(a, grad, false, st);
  }
  return hipGetLastError();
}
template <class E>
hipError_t go(const ScanArgs& a, bool grad, hipStream_t st) {
  return a.c.kind == SIM_GATE_SIGMOID ? go<E, true>(a, grad, st) : go<E, false>(a, grad, st);
}

}  // namespace

size_t scan_work_bytes(const sim_scan& c, bool grad) {
  if (!grad && c.T <= kStepT) return 0;
  size_t need = 0;
  sim_scan flat = c;   // as one sequence of all channels, if the strides allow it
  flat.D *= c.B;
  flat.B = 1;
  for (const sim_scan& s : {c, flat}) {
    need = std::max(need, plan_bytes(s, plan_of(s, grad, false, true)));
    if (s.D == 1) need = std::max(need, plan_bytes(s, plan_of(s, grad, true, true)));
  }
  return need;
}

hipError_t launch_scan(const ScanArgs& a, bool grad, hipStream_t st) {
  switch (a.c.dtype) {
    case SIM_DT_F64: return go<F64>(a, grad, st);
    case SIM_DT_F32: return go<F32>(a, grad, st);
    case SIM_DT_BF16: return go<BF16>(a, grad, st);
    default: return go<F16>(a, grad, st);
  }
}

}  // namespace bsim
