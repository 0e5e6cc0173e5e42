// Linear recurrence h_t = a_t k_t h_{t-1} + u_t over a trajectory, and its
// gradient.
//
// A step is an affine map of the carried state (h -> a h + u; backwards, with
// f the gradient that arrives from later steps, f -> a (dh + f)), and maps
// compose: (A1, B1) then (A2, B2) is (A2 A1, A2 B1 + B2).  Both passes touch
// each value once per direction, 2 to 4 floating operations against 4 to 12
// bytes, so HBM bounds them and what matters is bytes in flight:
//   * lanes of a wave hold neighbouring channels (one dword per lane and step:
//     a float, or two bfloat16 of one row), so each access is 256 contiguous
//     bytes;
//   * a wave walks SCAN_K steps at a time whose inputs were loaded while the
//     SCAN_K steps before them were computed;
//   * with few channels the steps are split: S waves of a workgroup take
//     SCAN_K consecutive steps each, fold them to one map, exchange the maps
//     through LDS and replay their steps from the state that reaches them
//     (inputs stay in registers, so they are read once); and with very few
//     channels the trajectory is cut into segments, one workgroup each, whose
//     waves (which then take steps in a row, and never wait for one another)
//     are folded to maps in the workspace by a first launch and replayed by a
//     second (inputs are read twice).
// Episode ends cut the state: a map that contains one does not read its input.
// It is marked by SCAN_CUT in place of A, so that 0 * NaN never arises.
// A map's A is a product of factors, which may leave float32's range and come
// back, or grow while the states are 0, where every state fits: it is float64,
// held within 2^500 (a larger one meets a state of 0, or makes an infinity of
// any other float32 anyway; and four factors below 2^128 may follow before the
// next check).
#include <initializer_list>

#include "rl_internal.h"

namespace rl {
namespace {

constexpr int SCAN_K = 8;           // steps a wave holds in registers
constexpr int SCAN_CUT = 0x7ff8dead;  // upper half of a NaN that stands for "the state before is cut off"
constexpr double SCAN_MOST = 0x1p500;

// A channel's value: one float, or a complex number.
template <bool DIAG>
struct Val;
template <>
struct Val<false> {
  float x;
  __device__ static Val zero() { return {0.f}; }
  __device__ static Val add(Val a, Val b) { return {a.x + b.x}; }
  __device__ static Val mul(Val a, Val b) { return {a.x * b.x}; }
  __device__ static Val fma(Val a, Val h, Val u) { return {fmaf(a.x, h.x, u.x)}; }
  __device__ Val conj() const { return *this; }
};
template <>
struct Val<true> {
  float x, y;
  __device__ static Val zero() { return {0.f, 0.f}; }
  __device__ static Val add(Val a, Val b) { return {a.x + b.x, a.y + b.y}; }
  __device__ static Val mul(Val a, Val b) { return {fmaf(a.x, b.x, -a.y * b.y), fmaf(a.x, b.y, a.y * b.x)}; }
  __device__ static Val fma(Val a, Val h, Val u) {
    return {fmaf(a.x, h.x, fmaf(-a.y, h.y, u.x)), fmaf(a.x, h.y, fmaf(a.y, h.x, u.y))};
  }
  __device__ Val conj() const { return {x, -y}; }
};

__device__ __forceinline__ double bounded(double x) { return fabs(x) > SCAN_MOST ? copysign(SCAN_MOST, x) : x; }

// The same in float64: products of factors, and a state on its way through maps.
template <bool DIAG>
struct Wide;
template <>
struct Wide<false> {
  double x;
  __device__ static Wide one() { return {1.}; }
  __device__ static Wide of(Val<false> v) { return {(double)v.x}; }
  __device__ static Wide mul(Wide a, Wide b) { return {a.x * b.x}; }
  __device__ static Wide fma(Wide a, Wide h, Val<false> u) { return {::fma(a.x, h.x, (double)u.x)}; }
  __device__ Wide held() const { return {bounded(x)}; }
  __device__ Val<false> val() const { return {(float)x}; }
};
template <>
struct Wide<true> {
  double x, y;
  __device__ static Wide one() { return {1., 0.}; }
  __device__ static Wide of(Val<true> v) { return {(double)v.x, (double)v.y}; }
  __device__ static Wide mul(Wide a, Wide b) { return {::fma(a.x, b.x, -a.y * b.y), ::fma(a.x, b.y, a.y * b.x)}; }
  __device__ static Wide fma(Wide a, Wide h, Val<true> u) {
    return {::fma(a.x, h.x, ::fma(-a.y, h.y, (double)u.x)), ::fma(a.x, h.y, ::fma(a.y, h.x, (double)u.y))};
  }
  __device__ Wide held() const { return {bounded(x), bounded(y)}; }
  __device__ Val<true> val() const { return {(float)x, (float)y}; }
};

// An affine map of the carried state, or (a cut one) a constant.
template <bool DIAG>
struct Map {
  using V = Val<DIAG>;
  using W = Wide<DIAG>;
  W a;
  V b;
  __device__ static Map constant(V b) {
    W a = W::one();
    a.x = __hiloint2double(SCAN_CUT, 0);
    return {a, b};
  }
  __device__ bool cut() const { return __double2hiint(a.x) == SCAN_CUT; }
  __device__ W operator()(W h) const { return cut() ? W::of(b) : W::fma(a, h, b); }
  // this map after m
  __device__ Map after(const Map& m) const {
    if (cut()) return *this;
    const V end = W::fma(a, W::of(m.b), b).val();
    if (m.cut()) return constant(end);
    return {W::mul(a, m.a).held(), end};
  }
};

// The map folded from steps with product a and end value b, of which one was
// cut (or not): a product that happens to be the marker becomes another NaN.
template <bool DIAG>
__device__ __forceinline__ Map<DIAG> folded(Wide<DIAG> a, Val<DIAG> b, bool cut) {
  if (cut) return Map<DIAG>::constant(b);
  Map<DIAG> m{a.held(), b};
  if (m.cut()) m.a.x = __hiloint2double(0x7ff80000, 0);
  return m;
}

// The product of a block's factors: gate after gate (k: its place in the
// block), or the n-th power of one factor (p: the SCAN_K-th).
__device__ __forceinline__ void take_gate(Wide<false>& a, Val<false> gate, int k) {
  a = Wide<false>::mul(a, Wide<false>::of(gate));
  if (k % 4 == 3) a = a.held();
}
__device__ __forceinline__ Wide<true> power(Val<true> lam) {
  Wide<true> p = Wide<true>::of(lam);
#pragma unroll
  for (int k = 1; k < SCAN_K; k *= 2) p = Wide<true>::mul(p, p).held();
  return p;
}
__device__ __forceinline__ Wide<true> power(Val<true> lam, Wide<true> p, int n) {
  if (n >= SCAN_K) return p;
  Wide<true> a = Wide<true>::one();
  for (int k = 0; k < n; ++k) a = Wide<true>::mul(a, Wide<true>::of(lam)).held();
  return a;
}

// The V neighbouring channels of a lane (of one row) at a step, as loaded:
// one dword, or two for complex values (real and imaginary parts).
template <int DT, bool DIAG, int V>
struct Raw {
  uint32_t w[DIAG ? 2 : 1];
  __device__ Val<DIAG> get(int v) const {
    auto f = [&](uint32_t x) {
      if constexpr (DT == DT_F32) return __uint_as_float(x);
      else return __uint_as_float(v == 0 ? x << 16 : x & 0xffff0000u);
    };
    if constexpr (DIAG) return {f(w[0]), f(w[1])};
    else return {f(w[0])};
  }
};

template <int DT>
constexpr int elem_bytes() { return DT == DT_F32 ? 4 : 2; }

// Workgroups of a 1-D grid go to the 8 XCDs in turn, each with an L2 cache of
// its own.  This gives each XCD a run of neighbouring channels instead, so that
// cache lines that two workgroups share (rows that are not aligned to lines)
// are read and written once: gradients of 1001 steps x 14541 float32 channels
// 73 us instead of 87.  One-wave workgroups gain from it where a step has 8 MB
// and more (64 x 2.1 M complex float32: 428 us, 467 in turn); below that they
// are better off in turn (128 x 262144 complex float32: 109 us, 115 in runs).
template <int S>
__device__ __forceinline__ int scan_block(size_t step_bytes) {
  const int id = blockIdx.x, n = gridDim.x, x = id % 8;
  if (gridDim.y > 1 || (S == 1 && step_bytes < (8u << 20))) return id;
  return x * (n / 8) + (x < n % 8 ? x : n % 8) + id / 8;
}

// Where a lane's channels lie.  Steps are M elements apart; off0 is the
// element offset (in a step) of the workgroup's first lane, uniform, so that
// addresses are a scalar base plus a 32-bit lane offset.
template <bool DIAG, int V>
struct Lane {
  int c, p;          // first channel, its place in the row
  int env;
  size_t off0, M;
  uint32_t rel;      // elements from off0
  bool live;         // lanes past the last channel repeat the last one and store nothing
  __device__ Lane(const ScanArgs& a, int lane, int block) {
    const int N = a.E * a.A * a.W;
    const int64_t ci = ((int64_t)block * 64 + lane) * V;
    live = ci < N;
    c = live ? (int)ci : N - V;
    const int row = c / a.W;
    p = c - row * a.W;
    env = row / a.A;
    M = (size_t)N * (DIAG ? 2 : 1);
    const int64_t c0 = (int64_t)block * 64 * V;  // the first lane's channel: always < N
    const int row0 = (int)(c0 / a.W);
    off0 = (size_t)c0 + (DIAG ? (size_t)row0 * a.W : 0);
    rel = (uint32_t)((size_t)c + (DIAG ? (size_t)row * a.W : 0) - off0);
  }
};

template <int DT, bool DIAG, int V>
__device__ __forceinline__ Raw<DT, DIAG, V> load_raw(const void* base, const Lane<DIAG, V>& l, int t, int W) {
  constexpr int ES = elem_bytes<DT>();
  const char* s = static_cast<const char*>(base) + ((size_t)t * l.M + l.off0) * ES;
  Raw<DT, DIAG, V> r;
#pragma unroll
  for (int i = 0; i < (DIAG ? 2 : 1); ++i) {
    const char* q = s + (size_t)i * W * ES + l.rel * (uint32_t)ES;
    if constexpr (ES * V == 4) r.w[i] = *reinterpret_cast<const uint32_t*>(q);
    else r.w[i] = *reinterpret_cast<const uint16_t*>(q);
  }
  return r;
}

template <int DT, bool DIAG, int V>
__device__ __forceinline__ void store_vals(void* base, const Lane<DIAG, V>& l, int t, int W, const Val<DIAG> (&v)[V]) {
  constexpr int ES = elem_bytes<DT>();
  char* s = static_cast<char*>(base) + ((size_t)t * l.M + l.off0) * ES;
  auto put = [&](char* q, float a, float b) {
    if constexpr (DT == DT_F32) *reinterpret_cast<float*>(q) = a;
    else if constexpr (V == 2) *reinterpret_cast<uint32_t*>(q) = pack_bf16x2(a, b);
    else *reinterpret_cast<uint16_t*>(q) = f32_to_bf16(a);
  };
  put(s + l.rel * (uint32_t)ES, v[0].x, v[V - 1].x);
  if constexpr (DIAG) put(s + (size_t)W * ES + l.rel * (uint32_t)ES, v[0].y, v[V - 1].y);
}

// A lane's float32 states.
template <bool DIAG, int V>
__device__ __forceinline__ void load_state(const float* base, const Lane<DIAG, V>& l, int W, Val<DIAG> (&v)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    v[i] = Val<DIAG>::zero();
    if (base) {
      v[i].x = base[l.off0 + l.rel + i];
      if constexpr (DIAG) v[i].y = base[l.off0 + l.rel + i + W];
    }
  }
}
template <bool DIAG, int V>
__device__ __forceinline__ void store_state(float* base, const Lane<DIAG, V>& l, int W, const Val<DIAG> (&v)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    base[l.off0 + l.rel + i] = v[i].x;
    if constexpr (DIAG) base[l.off0 + l.rel + i + W] = v[i].y;
  }
}

// The maps of a workgroup's waves, exchanged through LDS.  `into` is the state
// that reaches wave w when `carry` enters the first one, and carry becomes the
// state that leaves the last one.  Two buffers, so one barrier per exchange:
// a wave that writes buffer b again has passed the barrier of the exchange in
// between, which every wave reaches after reading b.
template <bool DIAG, int V, int S>
struct Exchange {
  // Maps read at a time: more of them hold registers that the gradients of complex channels do not have (128 steps x
  // 65536 of them: 73 us with 4, 58 with 1), and gates have (2000 x 32768: 99 and 105 us).
  static constexpr int TOGETHER = DIAG ? 1 : 4;
  Wide<DIAG> a[2][S][V][64];
  Val<DIAG> b[2][S][V][64];
  __device__ Map<DIAG> map(int buf, int w, int v, int lane) const { return {a[buf][w][v][lane], b[buf][w][v][lane]}; }
  __device__ void share(int buf, int w, int lane, const Map<DIAG> (&mine)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      a[buf][w][v][lane] = mine[v].a;
      b[buf][w][v][lane] = mine[v].b;
    }
    __syncthreads();
  }
  __device__ void operator()(int buf, int w, int lane, const Map<DIAG> (&mine)[V], Val<DIAG> (&carry)[V],
                             Val<DIAG> (&into)[V]) {
    share(buf, w, lane, mine);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      Wide<DIAG> c = Wide<DIAG>::of(carry[v]), at = c;
#pragma unroll TOGETHER
      for (int j = 0; j < S; ++j) {
        if (j == w) at = c;
        c = map(buf, j, v, lane)(c);
      }
      into[v] = at.val();
      carry[v] = c.val();
    }
  }
};

// Before the carried state is written: it may lie where the first one was
// read from, by waves that may have had no use for it so far.
template <int S>
__device__ __forceinline__ void states_read() {
  if constexpr (S > 1) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
}

// Workspace of a run cut into segments: slot 0 holds the constant map to the
// state that enters the first segment, slot g + 1 the map of segment g; behind
// the slots of all `segments` lie the maps of their waves, S to a segment (a
// wave has seg / S steps in a row, so that no wave waits for another inside).
template <bool DIAG>
__device__ __forceinline__ Map<DIAG>* slot(void* ws, size_t N, int g) { return static_cast<Map<DIAG>*>(ws) + N * g; }

// The state that enters segment g (the maps of slots 0..g applied in turn):
// each wave composes a part of the slots, then the waves' maps are exchanged.
template <bool DIAG, int V, int S>
__device__ __forceinline__ void enter_segment(void* ws, size_t N, int g, int w, int lane, const Lane<DIAG, V>& l,
                                              Exchange<DIAG, V, S>& ex, Val<DIAG> (&carry)[V]) {
  const int per = (g + S) / S, lo = w * per, hi = lo + per < g + 1 ? lo + per : g + 1;
  Map<DIAG> mine[V];
#pragma unroll
  for (int v = 0; v < V; ++v) mine[v] = {Wide<DIAG>::one(), Val<DIAG>::zero()};
  for (int i = lo; i < hi; ++i)
#pragma unroll
    for (int v = 0; v < V; ++v) mine[v] = slot<DIAG>(ws, N, i)[l.c + v].after(mine[v]);
  Val<DIAG> into[V];
#pragma unroll
  for (int v = 0; v < V; ++v) carry[v] = Val<DIAG>::zero();
  ex(0, w, lane, mine, carry, into);
}

template <bool DIAG, int S>
__device__ __forceinline__ Map<DIAG>* wave_slot(void* ws, size_t N, int segments, int g, int w) {
  return slot<DIAG>(ws, N, segments + 1 + g * S + w);
}

// The state that enters wave w's part of segment g.
template <bool DIAG, int V, int S>
__device__ __forceinline__ void enter_part(void* ws, size_t N, int segments, int g, int w, int lane,
                                           const Lane<DIAG, V>& l, Exchange<DIAG, V, S>& ex, Val<DIAG> (&carry)[V]) {
  enter_segment<DIAG, V, S>(ws, N, g, w, lane, l, ex, carry);
  Wide<DIAG> c[V];
#pragma unroll
  for (int v = 0; v < V; ++v) c[v] = Wide<DIAG>::of(carry[v]);
  for (int j = 0; j < w; ++j)
#pragma unroll
    for (int v = 0; v < V; ++v) c[v] = wave_slot<DIAG, S>(ws, N, segments, g, j)[l.c + v](c[v]);
#pragma unroll
  for (int v = 0; v < V; ++v) carry[v] = c[v].val();
}

// After a wave folded its part to `mine`: its map and the segment's.
template <bool DIAG, int V, int S>
__device__ __forceinline__ void leave_part(void* ws, size_t N, int segments, int g, int w, int lane,
                                           const Lane<DIAG, V>& l, Exchange<DIAG, V, S>& ex,
                                           const Map<DIAG> (&mine)[V]) {
  ex.share(0, w, lane, mine);
  if (!l.live) return;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    wave_slot<DIAG, S>(ws, N, segments, g, w)[l.c + v] = mine[v];
    if (w == 0) {
      Map<DIAG> all = mine[v];
#pragma unroll
      for (int j = 1; j < S; ++j) all = ex.map(0, j, v, lane).after(all);
      slot<DIAG>(ws, N, g + 1)[l.c + v] = all;
    }
  }
}

// What a launch does: the whole run; or, where it is cut into segments, first
// every wave's part folded to a map, then the parts replayed from the states
// that enter them.
enum { SCAN_WHOLE = 0, SCAN_FOLD = 1, SCAN_PARTS = 2 };

// Inputs of SCAN_K steps of a wave, [first, end) of them real.
template <int DT, bool DIAG, int V>
struct Block {
  Raw<DT, DIAG, V> u[SCAN_K], g[DIAG ? 1 : SCAN_K];
  uint8_t done[SCAN_K];  // of the step before
  __device__ void load(const ScanArgs& a, const Lane<DIAG, V>& l, const void* up, const void* gate,
                       const uint8_t* dn, int t0, int end) {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) {
      const int t = t0 + k;
      if (t < end) {
        u[k] = load_raw<DT, DIAG, V>(up, l, t, a.W);
        if constexpr (!DIAG) g[k] = load_raw<DT, DIAG, V>(gate, l, t, a.W);
        done[k] = 0;
        if (dn && t > 0) done[k] = dn[(size_t)(t - 1) * a.E + l.env];
      }
    }
  }
};

template <int DT, bool DIAG, int V>
__device__ __forceinline__ void load_lambda(const void* gate, const Lane<DIAG, V>& l, int W, Val<DIAG> (&lam)[V]) {
  if constexpr (DIAG) {
    const float* f = static_cast<const float*>(gate);
#pragma unroll
    for (int v = 0; v < V; ++v) lam[v] = {f[l.p + v], f[W + l.p + v]};
  }
}

// Forward.  seg: steps of a segment.
template <int DT, bool DIAG, int V, int S, int MODE>
__global__ __launch_bounds__(64 * S) void scan_kernel(ScanArgs a, const void* u, const void* gate,
                                                      const uint8_t* done, const float* h0, void* h, float* h_last,
                                                      void* ws, int seg) {
  using VT = Val<DIAG>;
  __shared__ Exchange<DIAG, V, S> ex;
  const int lane = threadIdx.x & 63, w = S == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const size_t N = (size_t)a.E * a.A * a.W;
  const Lane<DIAG, V> l(a, lane, scan_block<S>(N * (DIAG ? 2 : 1) * elem_bytes<DT>()));
  const int g = blockIdx.y;
  constexpr bool PARTS = MODE != SCAN_WHOLE;  // this wave's steps lie in a row
  const int first = PARTS ? g * seg + w * (seg / S) : 0;
  const int end = PARTS && a.T - first > seg / S ? first + seg / S : a.T;
  constexpr int STEP = PARTS ? SCAN_K : S * SCAN_K;
  VT lam[V], carry[V], into[V];
  load_lambda<DT, DIAG, V>(gate, l, a.W, lam);
  if constexpr (MODE == SCAN_PARTS) {
    enter_part<DIAG, V, S>(ws, N, gridDim.y, g, w, lane, l, ex, carry);
  } else {
    load_state<DIAG, V>(h0, l, a.W, carry);
    if (MODE == SCAN_FOLD && g == 0 && w == 0 && l.live)
#pragma unroll
      for (int v = 0; v < V; ++v) slot<DIAG>(ws, N, 0)[l.c + v] = Map<DIAG>::constant(carry[v]);
  }
  Wide<DIAG> A[V];  // the steps so far (SCAN_FOLD) or of this block
  VT B[V];
  bool cut = false;
  auto restart = [&]() {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = Wide<DIAG>::one();
      B[v] = VT::zero();
    }
    cut = false;
  };
  restart();
  Wide<DIAG> block[V];  // the factor of SCAN_K steps
  if constexpr (DIAG)
#pragma unroll
    for (int v = 0; v < V; ++v) block[v] = power(lam[v]);
  int buf = 0;
  Block<DT, DIAG, V> cur, nxt;
  const int ahead = PARTS ? 0 : w * SCAN_K;
  cur.load(a, l, u, gate, done, first + ahead, end);
  for (int t0 = first; t0 < end; t0 += STEP) {
    const int tw = t0 + ahead;
    if (t0 + STEP < end) nxt.load(a, l, u, gate, done, tw + STEP, end);
    if constexpr (MODE == SCAN_FOLD || (!PARTS && S > 1)) {
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k)
        if (tw + k < end) {
          const bool c = cur.done[k] != 0;
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const VT ak = [&] { if constexpr (DIAG) return lam[v]; else return cur.g[k].get(v); }();
            const VT uk = cur.u[k].get(v);
            B[v] = c ? uk : VT::fma(ak, B[v], uk);
            if constexpr (!DIAG) take_gate(A[v], ak, k);
          }
          cut |= c;
        }
      if constexpr (DIAG)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const Wide<DIAG> steps = power(lam[v], block[v], end - tw);
          A[v] = MODE == SCAN_FOLD ? Wide<DIAG>::mul(A[v], steps).held() : steps;
        }
    }
    if constexpr (MODE != SCAN_FOLD) {
      if constexpr (!PARTS && S > 1) {
        Map<DIAG> mine[V];
#pragma unroll
        for (int v = 0; v < V; ++v) mine[v] = folded<DIAG>(A[v], B[v], cut);
        ex(buf, w, lane, mine, carry, into);
        buf ^= 1;
        restart();
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) into[v] = carry[v];
      }
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k)
        if (tw + k < end) {
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const VT ak = [&] { if constexpr (DIAG) return lam[v]; else return cur.g[k].get(v); }();
            const VT uk = cur.u[k].get(v);
            into[v] = cur.done[k] != 0 ? uk : VT::fma(ak, into[v], uk);
          }
          if (h && l.live) store_vals<DT, DIAG, V>(h, l, tw + k, a.W, into);
        }
      if constexpr (PARTS || S == 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) carry[v] = into[v];
      }
    }
    cur = nxt;
  }
  if constexpr (MODE == SCAN_FOLD) {
    Map<DIAG> mine[V];
#pragma unroll
    for (int v = 0; v < V; ++v) mine[v] = folded<DIAG>(A[v], B[v], cut);
    leave_part<DIAG, V, S>(ws, N, gridDim.y, g, w, lane, l, ex, mine);
  } else if (h_last && end == a.T) {
    if constexpr (!PARTS) states_read<S>();
    if (!l.live || (PARTS ? first >= end : w != 0)) return;  // (the wave with the last step; any knows the state)
    if (done && done[(size_t)(a.T - 1) * a.E + l.env] != 0)
#pragma unroll
      for (int v = 0; v < V; ++v) carry[v] = VT::zero();
    store_state<DIAG, V>(h_last, l, a.W, carry);
  }
}

// Backward: steps in falling order (step r of the walk is T - 1 - r), the
// carried value the gradient that arrives at a step from later ones.  GRAD:
// the gate's gradient is wanted (h is read).
template <int DT, bool DIAG, int V, bool GRAD>
struct BackBlock {
  Raw<DT, DIAG, V> dh[SCAN_K], g[DIAG ? 1 : SCAN_K], h[GRAD ? SCAN_K : 1];
  uint8_t done[SCAN_K];  // of the step before (in time)
  __device__ void load(const ScanArgs& a, const Lane<DIAG, V>& l, const void* dhp, const void* gate, const void* hp,
                       const uint8_t* dn, int r0, int end) {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) {
      if (r0 + k < end) {
        const int t = a.T - 1 - r0 - k;
        dh[k] = load_raw<DT, DIAG, V>(dhp, l, t, a.W);
        if constexpr (!DIAG) g[k] = load_raw<DT, DIAG, V>(gate, l, t, a.W);
        done[k] = 0;
        if (t > 0) {
          if constexpr (GRAD) h[k] = load_raw<DT, DIAG, V>(hp, l, t - 1, a.W);
          if (dn) done[k] = dn[(size_t)(t - 1) * a.E + l.env];
        }
      }
    }
  }
};

template <int DT, bool DIAG, int V, int S, int MODE, bool GRAD>
__global__ __launch_bounds__(64 * S, 4) void scan_bwd_kernel(ScanArgs a, const void* gate, const uint8_t* done,
                                                          const float* h0, const void* h, const void* dh,
                                                          const float* dh_last, void* du, void* dgate, float* dh0,
                                                          void* ws, double* dlam_part, int seg) {
  using VT = Val<DIAG>;
  __shared__ Exchange<DIAG, V, S> ex;
  const int lane = threadIdx.x & 63, w = S == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const size_t N = (size_t)a.E * a.A * a.W;
  const Lane<DIAG, V> l(a, lane, scan_block<S>(N * (DIAG ? 2 : 1) * elem_bytes<DT>()));
  const int g = blockIdx.y;
  constexpr bool PARTS = MODE != SCAN_WHOLE;
  const int first = PARTS ? g * seg + w * (seg / S) : 0;
  const int end = PARTS && a.T - first > seg / S ? first + seg / S : a.T;
  constexpr int STEP = PARTS ? SCAN_K : S * SCAN_K;
  VT lam[V], carry[V], into[V], start[V];
  load_lambda<DT, DIAG, V>(gate, l, a.W, lam);
  if constexpr (GRAD) load_state<DIAG, V>(h0, l, a.W, start);
  if constexpr (MODE == SCAN_PARTS) {
    enter_part<DIAG, V, S>(ws, N, gridDim.y, g, w, lane, l, ex, carry);
  } else {
    const bool ended = done && done[(size_t)(a.T - 1) * a.E + l.env] != 0;
    load_state<DIAG, V>(ended ? nullptr : dh_last, l, a.W, carry);
    if (MODE == SCAN_FOLD && g == 0 && w == 0 && l.live)
#pragma unroll
      for (int v = 0; v < V; ++v) slot<DIAG>(ws, N, 0)[l.c + v] = Map<DIAG>::constant(carry[v]);
  }
  Wide<DIAG> A[V];
  VT B[V];
  bool cut = false;
  auto restart = [&]() {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = Wide<DIAG>::one();
      B[v] = VT::zero();
    }
    cut = false;
  };
  restart();
  double sx[V], sy[V];
#pragma unroll
  for (int v = 0; v < V; ++v) sx[v] = sy[v] = 0.;
  Wide<DIAG> block[V];  // the factor of SCAN_K steps
  if constexpr (DIAG)
#pragma unroll
    for (int v = 0; v < V; ++v) block[v] = power(lam[v].conj());
  int buf = 0;
  BackBlock<DT, DIAG, V, GRAD> cur, nxt;
  const int ahead = PARTS ? 0 : w * SCAN_K;
  cur.load(a, l, dh, gate, h, done, first + ahead, end);
  for (int r0 = first; r0 < end; r0 += STEP) {
    const int rw = r0 + ahead;
    if (r0 + STEP < end) nxt.load(a, l, dh, gate, h, done, rw + STEP, end);
    if constexpr (MODE == SCAN_FOLD || (!PARTS && S > 1)) {
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k)
        if (rw + k < end) {
          const bool c = cur.done[k] != 0;
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const VT ak = [&] { if constexpr (DIAG) return lam[v].conj(); else return cur.g[k].get(v); }();
            B[v] = c ? VT::zero() : VT::mul(ak, VT::add(cur.dh[k].get(v), B[v]));
            if constexpr (!DIAG) take_gate(A[v], ak, k);
          }
          cut |= c;
        }
      if constexpr (DIAG)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const Wide<DIAG> steps = power(lam[v].conj(), block[v], end - rw);
          A[v] = MODE == SCAN_FOLD ? Wide<DIAG>::mul(A[v], steps).held() : steps;
        }
    }
    if constexpr (MODE != SCAN_FOLD) {
      if constexpr (!PARTS && S > 1) {
        Map<DIAG> mine[V];
#pragma unroll
        for (int v = 0; v < V; ++v) mine[v] = folded<DIAG>(A[v], B[v], cut);
        ex(buf, w, lane, mine, carry, into);
        buf ^= 1;
        restart();
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) into[v] = carry[v];
      }
      float fx[V], fy[V];  // this block's part of the sums over steps: SCAN_K terms in float32 (at most 8 u of their
                           // magnitudes, as the terms' own roundings), float64 from there on
#pragma unroll
      for (int v = 0; v < V; ++v) fx[v] = fy[v] = 0.f;
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k)
        if (rw + k < end) {
          const int t = a.T - 1 - rw - k;
          const bool c = cur.done[k] != 0;
          VT gt[V], dg[V];
#pragma unroll
          for (int v = 0; v < V; ++v) {
            gt[v] = VT::add(cur.dh[k].get(v), into[v]);
            const VT ak = [&] { if constexpr (DIAG) return lam[v].conj(); else return cur.g[k].get(v); }();
            into[v] = c ? VT::zero() : VT::mul(ak, gt[v]);
            if constexpr (GRAD) {
              const bool has = !c && (t > 0 || h0);
              const VT prev = t > 0 ? cur.h[k].get(v) : start[v];
              dg[v] = has ? VT::mul(gt[v], prev.conj()) : VT::zero();
              if constexpr (DIAG) {
                fx[v] += dg[v].x;
                fy[v] += dg[v].y;
              }
            }
          }
          if (l.live) {
            store_vals<DT, DIAG, V>(du, l, t, a.W, gt);
            if constexpr (GRAD && !DIAG) store_vals<DT, DIAG, V>(dgate, l, t, a.W, dg);
          }
        }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if constexpr (PARTS || S == 1) carry[v] = into[v];
        if constexpr (GRAD && DIAG) {
          sx[v] += (double)fx[v];
          sy[v] += (double)fy[v];
        }
      }
    }
    cur = nxt;
  }
  if constexpr (MODE == SCAN_FOLD) {
    Map<DIAG> mine[V];
#pragma unroll
    for (int v = 0; v < V; ++v) mine[v] = folded<DIAG>(A[v], B[v], cut);
    leave_part<DIAG, V, S>(ws, N, gridDim.y, g, w, lane, l, ex, mine);
  } else {
    if (dh0 && end == a.T) {
      if constexpr (!PARTS) states_read<S>();
      if (l.live && (PARTS ? first < end : w == 0)) store_state<DIAG, V>(dh0, l, a.W, carry);
    }
    if constexpr (GRAD && DIAG) {
      // the waves' sums in order, then one partial sum per channel and segment
      if constexpr (S > 1) {
        __shared__ double part[S][2][V][64];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          part[w][0][v][lane] = sx[v];
          part[w][1][v][lane] = sy[v];
        }
        __syncthreads();
        if (w == 0)
#pragma unroll
          for (int v = 0; v < V; ++v)
            for (int j = 1; j < S; ++j) {
              sx[v] += part[j][0][v][lane];
              sy[v] += part[j][1][v][lane];
            }
      }
      if (w == 0 && l.live)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          dlam_part[(size_t)g * N + l.c + v] = sx[v];
          dlam_part[(size_t)(gridDim.y + g) * N + l.c + v] = sy[v];
        }
    }
  }
}

// dlam [2, P]: the partial sums [2, rows, P] added up over the rows.  A
// workgroup takes RED_P neighbouring channels (64 bytes of a row) and
// RED_NT / RED_P rows at a time.
constexpr int RED_NT = 1024, RED_P = 8;
__global__ __launch_bounds__(RED_NT) void scan_dlam_kernel(const double* part, int64_t rows, int P, float* dlam) {
  __shared__ double s[RED_NT];
  const int tid = threadIdx.x, p = blockIdx.x * RED_P + tid % RED_P, c = blockIdx.y;
  double v = 0.;
  if (p < P)
    for (int64_t r = tid / RED_P; r < rows; r += RED_NT / RED_P) v += part[(c * rows + r) * P + p];
  s[tid] = v;
  __syncthreads();
  for (int d = RED_NT / 2; d >= RED_P; d >>= 1) {
    if (tid < d) s[tid] += s[tid + d];
    __syncthreads();
  }
  if (tid < RED_P && p < P) dlam[(size_t)c * P + p] = (float)s[tid];
}

// How a call is split: S waves of a workgroup over the steps, G segments.
// Measured (one MI355X, us; float32 gates unless said otherwise):
//   * one wave per 64 channels alone has enough bytes in flight from 2048
//     waves on (250 steps x 131072 channels: 76 with S = 1, 89 with S = 8; at
//     65536 channels 53 and 46);
//   * up to 256 workgroups each has a CU to itself, where 16 waves load more
//     than 8 (2000 x 16384: 95 against 104; complex channels, whose maps cost
//     more to exchange, 250 x 16384: 19 against 20, gradients 32 against 33);
//     with more of them 8 waves leave room for a second workgroup (250 x 32768:
//     22 against 28);
//   * segments read the inputs twice, and pay where workgroups leave most CUs
//     idle (2000 x 4096: 33 in 8 segments, 67 in one; 2000 x 8192: 71 in 4, 74;
//     2000 x 16384: 143 in 2, 90; 500 x 4096: 16 in 3, 18).
struct ScanPlan {
  int S, G, seg;
};
ScanPlan scan_plan(const ScanArgs& p) {
  const int64_t lanes = (int64_t)p.E * p.A * p.W / (!p.diag && p.dt == DT_BF16 && p.W % 2 == 0 ? 2 : 1);
  const int64_t waves = (lanes + 63) / 64;
  ScanPlan s{1, 1, p.T};
  if (waves >= 2048 || p.T <= 2 * SCAN_K) return s;
  if (p.T <= 4 * SCAN_K) {
    s.S = 4;
    return s;
  }
  const int block = 8 * SCAN_K;
  const int64_t want = (512 + waves - 1) / waves, most = p.T / (2 * block), g = want < most ? want : most;
  if (waves <= 128 && g >= 2) {
    s.S = 8;
    s.seg = (int)(((p.T + g - 1) / g + block - 1) / block * block);
    s.G = (p.T + s.seg - 1) / s.seg;
  } else {
    s.S = waves > 256 || p.T <= block ? 8 : 16;
  }
  return s;
}
size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t slot_bytes(const ScanArgs& p, const ScanPlan& s) {
  if (s.G == 1) return 0;
  return round256((size_t)(s.G + 1 + s.G * s.S) * p.E * p.A * p.W * (p.diag ? sizeof(Map<true>) : sizeof(Map<false>)));
}

// Two bfloat16 channels to a lane where rows have an even number of them and
// every array starts at a dword.  Not for complex values: two dwords a step
// and the wider maps leave room for too few waves (250 steps x 16384 channels:
// 34 us with pairs, 19 without; the gradients 75 and 26).
bool pairs(const ScanArgs& p, std::initializer_list<const void*> values) {
  if (p.diag || p.dt != DT_BF16 || p.W % 2) return false;
  for (const void* v : values)
    if (reinterpret_cast<uintptr_t>(v) & 3) return false;
  return true;
}

dim3 scan_grid(const ScanArgs& p, int V, int G) {
  return dim3((unsigned)(((int64_t)p.E * p.A * p.W / V + 63) / 64), (unsigned)G);
}

template <int DT, bool DIAG, int V, int S>
void run_scan(const ScanArgs& p, const ScanPlan& pl, const void* u, const void* gate, const uint8_t* done,
              const float* h0, void* h, float* h_last, void* ws, hipStream_t s) {
  if constexpr (S == 8)  // (segments are taken with 8 waves)
    if (pl.G > 1) {
      const dim3 grid = scan_grid(p, V, pl.G);
      scan_kernel<DT, DIAG, V, S, SCAN_FOLD><<<grid, 64 * S, 0, s>>>(p, u, gate, done, h0, h, h_last, ws, pl.seg);
      scan_kernel<DT, DIAG, V, S, SCAN_PARTS><<<grid, 64 * S, 0, s>>>(p, u, gate, done, h0, h, h_last, ws, pl.seg);
      return;
    }
  scan_kernel<DT, DIAG, V, S, SCAN_WHOLE><<<scan_grid(p, V, 1), 64 * S, 0, s>>>(p, u, gate, done, h0, h, h_last, ws,
                                                                                pl.seg);
}

template <int DT, bool DIAG, int V, int S, bool GRAD>
void run_scan_bwd(const ScanArgs& p, const ScanPlan& pl, const void* gate, const uint8_t* done, const float* h0,
                  const void* h, const void* dh, const float* dh_last, void* du, void* dgate, float* dh0, void* ws,
                  hipStream_t s) {
  double* part = reinterpret_cast<double*>(static_cast<char*>(ws) + slot_bytes(p, pl));
  const dim3 grid = scan_grid(p, V, pl.G);
  bool parts = false;
  if constexpr (S == 8)
    if (pl.G > 1) {
      parts = true;
      scan_bwd_kernel<DT, DIAG, V, S, SCAN_FOLD, false><<<grid, 64 * S, 0, s>>>(p, gate, done, h0, h, dh, dh_last, du,
                                                                               dgate, dh0, ws, part, pl.seg);
      scan_bwd_kernel<DT, DIAG, V, S, SCAN_PARTS, GRAD><<<grid, 64 * S, 0, s>>>(p, gate, done, h0, h, dh, dh_last, du,
                                                                               dgate, dh0, ws, part, pl.seg);
    }
  if (!parts)
    scan_bwd_kernel<DT, DIAG, V, S, SCAN_WHOLE, GRAD><<<grid, 64 * S, 0, s>>>(p, gate, done, h0, h, dh, dh_last, du,
                                                                             dgate, dh0, ws, part, pl.seg);
  if (DIAG && GRAD)
    scan_dlam_kernel<<<dim3((unsigned)((p.W + RED_P - 1) / RED_P), 2), RED_NT, 0, s>>>(
        part, (int64_t)pl.G * p.E * p.A, p.W, static_cast<float*>(dgate));
}

// One of the compiled S.
#define RL_SCAN(DT, DIAG, V)             \
  switch (pl.S) {                        \
    case 1: RL_SCAN_S(DT, DIAG, V, 1); break;   \
    case 4: RL_SCAN_S(DT, DIAG, V, 4); break;   \
    case 8: RL_SCAN_S(DT, DIAG, V, 8); break;   \
    default: RL_SCAN_S(DT, DIAG, V, 16); break; \
  }

}  // namespace

size_t scan_workspace_bytes(const ScanArgs& p, bool backward) {
  const ScanPlan s = scan_plan(p);
  return slot_bytes(p, s) + (backward && p.diag ? sizeof(double) * 2 * (size_t)s.G * p.E * p.A * p.W : 0);
}

hipError_t launch_scan(const ScanArgs& p, const void* u, const void* gate, const uint8_t* done, const float* h0,
                       void* h, float* h_last, void* ws, hipStream_t s) {
  const ScanPlan pl = scan_plan(p);
  const bool two = pairs(p, {u, gate, h});
#define RL_SCAN_S(DT, DIAG, V, S) run_scan<DT, DIAG, V, S>(p, pl, u, gate, done, h0, h, h_last, ws, s)
  if (p.dt == DT_F32) {
    if (p.diag) RL_SCAN(DT_F32, true, 1) else RL_SCAN(DT_F32, false, 1)
  } else if (two) {
    RL_SCAN(DT_BF16, false, 2)
  } else {
    if (p.diag) RL_SCAN(DT_BF16, true, 1) else RL_SCAN(DT_BF16, false, 1)
  }
#undef RL_SCAN_S
  return hipGetLastError();
}

hipError_t launch_scan_backward(const ScanArgs& p, const void* gate, const uint8_t* done, const float* h0,
                                const void* h, const void* dh, const float* dh_last, void* du, void* dgate,
                                float* dh0, void* ws, hipStream_t s) {
  const ScanPlan pl = scan_plan(p);
  const bool two = pairs(p, {h, dh, du, gate, dgate});
#define RL_SCAN_S(DT, DIAG, V, S)                                                                               \
  (dgate ? run_scan_bwd<DT, DIAG, V, S, true>(p, pl, gate, done, h0, h, dh, dh_last, du, dgate, dh0, ws, s)     \
         : run_scan_bwd<DT, DIAG, V, S, false>(p, pl, gate, done, h0, h, dh, dh_last, du, dgate, dh0, ws, s))
  if (p.dt == DT_F32) {
    if (p.diag) RL_SCAN(DT_F32, true, 1) else RL_SCAN(DT_F32, false, 1)
  } else if (two) {
    RL_SCAN(DT_BF16, false, 2)
  } else {
    if (p.diag) RL_SCAN(DT_BF16, true, 1) else RL_SCAN(DT_BF16, false, 1)
  }
#undef RL_SCAN_S
  return hipGetLastError();
}

}  // namespace rl
