// Linear recurrence h_t = a_t k_t h_{t-1} + u_t over a trajectory, and its
// gradient: one thread per channel (a pair of values when the factors are
// complex), walking over the steps.
#include "rl_internal.h"

namespace rl {
namespace {

constexpr int SCAN_NT = 64;  // one wave per workgroup: channels spread over as many CUs as possible
constexpr int SCAN_U = 8;    // steps whose inputs are loaded ahead of the dependent recurrence

// A channel's value: one float, or a complex number.
template <bool DIAG>
struct Val;
template <>
struct Val<false> {
  float x;
  __device__ static Val zero() { return {0.f}; }
  __device__ static Val add(Val a, Val b) { return {a.x + b.x}; }
  // a * h + u
  __device__ static Val fma(Val a, Val h, Val u) { return {fmaf(a.x, h.x, u.x)}; }
  // conj(a) * h + u
  __device__ static Val fmac(Val a, Val h, Val u) { return {fmaf(a.x, h.x, u.x)}; }
};
template <>
struct Val<true> {
  float x, y;
  __device__ static Val zero() { return {0.f, 0.f}; }
  __device__ static Val add(Val a, Val b) { return {a.x + b.x, a.y + b.y}; }
  __device__ static Val fma(Val a, Val h, Val u) {
    return {fmaf(a.x, h.x, fmaf(-a.y, h.y, u.x)), fmaf(a.x, h.y, fmaf(a.y, h.x, u.y))};
  }
  __device__ static Val fmac(Val a, Val h, Val u) {
    return {fmaf(a.x, h.x, fmaf(a.y, h.y, u.x)), fmaf(a.x, h.y, fmaf(-a.y, h.x, u.y))};
  }
};

template <int DT, bool DIAG>
__device__ __forceinline__ Val<DIAG> load_val(const void* base, size_t i, int W) {
  using E = typename DType<DT>::T;
  const E* p = static_cast<const E*>(base) + i;
  if constexpr (DIAG) return {DType<DT>::to_f32(p[0]), DType<DT>::to_f32(p[W])};
  else return {DType<DT>::to_f32(p[0])};
}
template <int DT, bool DIAG>
__device__ __forceinline__ void store_val(void* base, size_t i, int W, Val<DIAG> v) {
  using E = typename DType<DT>::T;
  E* p = static_cast<E*>(base) + i;
  p[0] = DType<DT>::from_f32(v.x);
  if constexpr (DIAG) p[W] = DType<DT>::from_f32(v.y);
}

// Where channel c of a step lies: its offset in the step's values, its env.
template <bool DIAG>
struct Chan {
  int off, p, env;
  __device__ Chan(const ScanArgs& a, int c) {
    const int row = c / a.W;
    p = c - row * a.W;
    off = DIAG ? row * 2 * a.W + p : c;
    env = row / a.A;
  }
};

template <int DT, bool DIAG>
__global__ __launch_bounds__(SCAN_NT) void scan_kernel(ScanArgs a, const void* u, const void* gate,
                                                       const uint8_t* done, const float* h0, void* h,
                                                       float* h_last) {
  const int N = a.E * a.A * a.W;
  const int64_t ci = (int64_t)blockIdx.x * SCAN_NT + threadIdx.x;
  if (ci >= N) return;
  const Chan<DIAG> ch(a, (int)ci);
  const size_t M = (size_t)N * (DIAG ? 2 : 1);
  using V = Val<DIAG>;
  V st = h0 ? load_val<DT_F32, DIAG>(h0, ch.off, a.W) : V::zero();
  V g = V::zero();
  if constexpr (DIAG) g = load_val<DT_F32, true>(gate, ch.p, a.W);
  bool keep = true;
  for (int t0 = 0; t0 < a.T; t0 += SCAN_U) {
    V in[SCAN_U], ga[SCAN_U];
    bool go[SCAN_U];
#pragma unroll
    for (int k = 0; k < SCAN_U; ++k) {
      const int t = t0 + k;
      if (t < a.T) {
        in[k] = load_val<DT, DIAG>(u, (size_t)t * M + ch.off, a.W);
        if constexpr (DIAG) ga[k] = g;
        else ga[k] = load_val<DT, false>(gate, (size_t)t * M + ch.off, a.W);
        go[k] = !done || done[(size_t)t * a.E + ch.env] == 0;
      }
    }
#pragma unroll
    for (int k = 0; k < SCAN_U; ++k) {
      const int t = t0 + k;
      if (t < a.T) {
        st = keep ? V::fma(ga[k], st, in[k]) : in[k];
        keep = go[k];
        if (h) store_val<DT, DIAG>(h, (size_t)t * M + ch.off, a.W, st);
      }
    }
  }
  if (h_last) store_val<DT_F32, DIAG>(h_last, ch.off, a.W, keep ? st : V::zero());
}

// dlam_part (diagonal kind): the channel's sum of g conj(k h) over the steps.
template <int DT, bool DIAG>
__global__ __launch_bounds__(SCAN_NT) void scan_bwd_kernel(ScanArgs a, const void* gate, const uint8_t* done,
                                                           const float* h0, const void* h, const void* dh,
                                                           const float* dh_last, void* du, void* dgate, float* dh0,
                                                           double* dlam_part) {
  const int N = a.E * a.A * a.W;
  const int64_t ci = (int64_t)blockIdx.x * SCAN_NT + threadIdx.x;
  if (ci >= N) return;
  const Chan<DIAG> ch(a, (int)ci);
  const size_t M = (size_t)N * (DIAG ? 2 : 1);
  using V = Val<DIAG>;
  V lam = V::zero();
  if constexpr (DIAG) lam = load_val<DT_F32, true>(gate, ch.p, a.W);
  double sx = 0., sy = 0.;
  // gradient that reaches h_t from the steps after it
  V flow = dh_last && !(done && done[(size_t)(a.T - 1) * a.E + ch.env]) ? load_val<DT_F32, DIAG>(dh_last, ch.off, a.W)
                                                                          : V::zero();
  for (int t1 = a.T; t1 > 0; t1 -= SCAN_U) {
    V in[SCAN_U], ga[SCAN_U], prev[SCAN_U];
    bool go[SCAN_U];
#pragma unroll
    for (int k = 0; k < SCAN_U; ++k) {
      const int t = t1 - 1 - k;
      if (t >= 0) {
        in[k] = load_val<DT, DIAG>(dh, (size_t)t * M + ch.off, a.W);
        if constexpr (DIAG) ga[k] = lam;
        else ga[k] = load_val<DT, false>(gate, (size_t)t * M + ch.off, a.W);
        go[k] = t == 0 || !done || done[(size_t)(t - 1) * a.E + ch.env] == 0;
        prev[k] = V::zero();
        if (dgate) {
          if (t > 0) prev[k] = load_val<DT, DIAG>(h, (size_t)(t - 1) * M + ch.off, a.W);
          else if (h0) prev[k] = load_val<DT_F32, DIAG>(h0, ch.off, a.W);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < SCAN_U; ++k) {
      const int t = t1 - 1 - k;
      if (t >= 0) {
        const V g = V::add(in[k], flow);
        const bool has = go[k] && (t > 0 || h0);
        store_val<DT, DIAG>(du, (size_t)t * M + ch.off, a.W, g);
        if constexpr (DIAG) {
          if (has) {
            sx += (double)fmaf(g.x, prev[k].x, g.y * prev[k].y);
            sy += (double)fmaf(g.y, prev[k].x, -g.x * prev[k].y);
          }
        } else if (dgate) {
          store_val<DT, false>(dgate, (size_t)t * M + ch.off, a.W, has ? V{g.x * prev[k].x} : V::zero());
        }
        flow = go[k] ? V::fmac(ga[k], g, V::zero()) : V::zero();
      }
    }
  }
  if (dh0) store_val<DT_F32, DIAG>(dh0, ch.off, a.W, flow);
  if constexpr (DIAG) {
    if (dgate) {
      dlam_part[ci] = sx;
      dlam_part[(size_t)N + ci] = sy;
    }
  }
}

// dlam [2, P]: the partial sums [2, rows, P] added up over the rows, one
// workgroup per state channel and part.
constexpr int RED_NT = 256;
__global__ __launch_bounds__(RED_NT) void scan_dlam_kernel(const double* part, int rows, int P, float* dlam) {
  __shared__ double s[RED_NT];
  const int p = blockIdx.x, c = blockIdx.y;
  double v = 0.;
  for (int r = threadIdx.x; r < rows; r += RED_NT) v += part[((size_t)c * rows + r) * P + p];
  s[threadIdx.x] = v;
  __syncthreads();
  for (int d = RED_NT / 2; d > 0; d >>= 1) {
    if (threadIdx.x < d) s[threadIdx.x] += s[threadIdx.x + d];
    __syncthreads();
  }
  if (threadIdx.x == 0) dlam[(size_t)c * P + p] = (float)s[0];
}

}  // namespace

size_t scan_workspace_bytes(const ScanArgs& p, bool backward) {
  return backward && p.diag ? sizeof(double) * 2 * (size_t)p.E * p.A * p.W : 0;
}

hipError_t launch_scan(const ScanArgs& p, const void* u, const void* gate, const uint8_t* done, const float* h0,
                       void* h, float* h_last, void*, hipStream_t s) {
  const unsigned grid = (unsigned)(((int64_t)p.E * p.A * p.W + SCAN_NT - 1) / SCAN_NT);
#define RL_SCAN(DT, DIAG) scan_kernel<DT, DIAG><<<grid, SCAN_NT, 0, s>>>(p, u, gate, done, h0, h, h_last)
  if (p.dt == DT_F32) {
    if (p.diag) RL_SCAN(DT_F32, true);
    else RL_SCAN(DT_F32, false);
  } else {
    if (p.diag) RL_SCAN(DT_BF16, true);
    else RL_SCAN(DT_BF16, false);
  }
#undef RL_SCAN
  return hipGetLastError();
}

hipError_t launch_scan_backward(const ScanArgs& p, const void* gate, const uint8_t* done, const float* h0,
                                const void* h, const void* dh, const float* dh_last, void* du, void* dgate,
                                float* dh0, void* workspace, hipStream_t s) {
  const unsigned grid = (unsigned)(((int64_t)p.E * p.A * p.W + SCAN_NT - 1) / SCAN_NT);
  double* part = static_cast<double*>(workspace);
#define RL_SCAN(DT, DIAG) \
  scan_bwd_kernel<DT, DIAG><<<grid, SCAN_NT, 0, s>>>(p, gate, done, h0, h, dh, dh_last, du, dgate, dh0, part)
  if (p.dt == DT_F32) {
    if (p.diag) RL_SCAN(DT_F32, true);
    else RL_SCAN(DT_F32, false);
  } else {
    if (p.diag) RL_SCAN(DT_BF16, true);
    else RL_SCAN(DT_BF16, false);
  }
#undef RL_SCAN
  if (p.diag && dgate)
    scan_dlam_kernel<<<dim3((unsigned)p.W, 2), RED_NT, 0, s>>>(part, p.E * p.A, p.W, static_cast<float*>(dgate));
  return hipGetLastError();
}

}  // namespace rl
