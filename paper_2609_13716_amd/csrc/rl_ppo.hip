// Proximal policy optimisation's loss over stored rows and its gradients.
//
// A row's work is its softmax; what bounds it is HBM (8 bytes an action and 28
// a row, both directions).  A wave takes 64 consecutive rows: their 64 nA
// logits are read as nA coalesced dwords per lane and turned into one row per
// lane through LDS (row stride odd, so that lanes hit different banks; illegal
// actions become -inf on the way), and the gradients go back the same way.
// Sums over rows are float64, taken in an order that depends on the sizes only:
// per lane, wave, workgroup, then over workgroups by the launch that follows.
//   R <= PPO_SMALL   one workgroup does everything in one launch (500 rows of
//                    6: 7 us of GPU time; 15 in three launches);
//   otherwise        the advantages' sums (when they are normalised or rows
//                    masked out), the rows, the six means.
#include "rl_internal.h"

namespace rl {
namespace {

constexpr int PPO_NT = 512;         // threads of a workgroup that does rows
constexpr int PPO_SUM_NT = 1024;    // of one that adds up advantages
constexpr int64_t PPO_SMALL = 2048;
constexpr int PPO_ADV_B = 64, PPO_ROW_B = 512;  // workgroups, at most (their partial sums go to the workspace)
constexpr int PPO_STATS = 6;
constexpr int PPO_CHUNK = 8;        // dwords of a row tile that a lane has in flight

struct PpoPart {  // workspace
  double adv[PPO_ADV_B][3];  // rows counted, sum and sum of squares of their advantages
  double stat[PPO_ROW_B][PPO_STATS];
};

// The sums of v over a wave, for every lane.
template <int N>
__device__ __forceinline__ void wave_sum(double (&v)[N]) {
#pragma unroll 1
  for (int d = 32; d > 0; d >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], d, 64);
}

// The same over a workgroup of at most 16 waves, for every thread.
template <int N>
__device__ __forceinline__ void block_sum(double (&v)[N], double (*s)[N]) {
  wave_sum<N>(v);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
  if (lane == 0)
    for (int i = 0; i < N; ++i) s[w][i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (lane & 15) < nw ? s[lane & 15][i] : 0.;
#pragma unroll 1
  for (int d = 8; d > 0; d >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], d, 64);
}

// Sums of the statistics over a workgroup: v[i] into thread i < PPO_STATS's
// result.  Each wave turns its lanes' values round in LDS (`mine`, a part of
// it that nobody else uses) so that 8 lanes add up one of them together: a
// sixth of the lane exchanges that all of them in every lane take.
constexpr int TURN_LD = PPO_STATS + 1, TURN_BYTES = 64 * TURN_LD * 8;
__device__ __forceinline__ double stats_sum(const double (&v)[PPO_STATS], double* mine, double (*s)[PPO_STATS]) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
#pragma unroll
  for (int i = 0; i < PPO_STATS; ++i) mine[lane * TURN_LD + i] = v[i];
  wave_lds_sync();
  const int i = lane >> 3;
  double t = 0.;
  if (i < PPO_STATS)
    for (int q = 0; q < 8; ++q) t += mine[((lane & 7) + 8 * q) * TURN_LD + i];
  for (int d = 4; d > 0; d >>= 1) t += __shfl_xor(t, d, 64);
  if (i < PPO_STATS && (lane & 7) == 0) s[w][i] = t;
  __syncthreads();
  t = 0.;
  if (threadIdx.x < PPO_STATS)
    for (int q = 0; q < nw; ++q) t += s[q][threadIdx.x];
  return t;
}

__device__ __forceinline__ void adv_sums(const PpoArgs& p, int64_t first, int64_t step, double (&v)[3]) {
#pragma unroll 8
  for (int64_t r = first; r < p.R; r += step) {
    const uint8_t in = p.mask ? p.mask[r] : 1;
    const float read = p.adv[r];  // (before the mask is known; a padded row's value is dropped)
    const double a = in ? (double)read : 0.;
    v[0] += in ? 1. : 0.;
    v[1] += a;
    v[2] += a * a;
  }
}

struct PpoNorm {
  double inv_n, mean, rstd;
};
// From the counted rows' number, sum and sum of squares.
__device__ __forceinline__ PpoNorm ppo_norm(const PpoArgs& p, const double (&v)[3]) {
  PpoNorm r{1. / (v[0] > 0. ? v[0] : 1.), 0., 1.};
  if (p.normalize) {
    const double var = v[2] * r.inv_n - v[1] * r.inv_n * (v[1] * r.inv_n);
    r.mean = v[1] * r.inv_n;
    r.rstd = 1. / (sqrt(var < 0. ? 0. : var) + 1e-8);  // (a NaN stays one)
  }
  return r;
}

// A value that every lane has, in scalar registers.
__device__ __forceinline__ double uniform(double v) {
  const uint64_t b = __double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b), hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
  return __longlong_as_double((uint64_t)hi << 32 | lo);
}

// exp(x) for x <= 0: the hardware's 2^t with t = x log2(e) rounded, times
// 1 + ln(2) (x log2(e) - t); within 3 float32 steps (results below 2^-126 are 0).
__device__ __forceinline__ float exp_neg(float x) {
  constexpr float L2E = 1.4426950408889634f, L2E_LO = (float)(1.4426950408889634 - (double)L2E);
  const float t = x * L2E, r = fmaf(x, L2E_LO, fmaf(x, L2E, -t));
  return __builtin_amdgcn_exp2f(t) * fmaf(r, 0.6931471805599453f, 1.f);
}

// exp(x) in float64, to 1e-13: 2^k times the Taylor sum of exp(r) to r^12 / 12!
// for |r| <= ln(2) / 2 (the next term is below 2e-16).  Few registers: the
// rows that need it are rare, and what it holds all of them pay for.
__device__ __forceinline__ double exp64(double x) {
  const double k = rint(x * 1.4426950408889634);
  const double r = fma(-k, 0.6931471805599453, x);
  double s = 1. / 479001600.;
  s = fma(s, r, 1. / 39916800.);
  s = fma(s, r, 1. / 3628800.);
  s = fma(s, r, 1. / 362880.);
  s = fma(s, r, 1. / 40320.);
  s = fma(s, r, 1. / 5040.);
  s = fma(s, r, 1. / 720.);
  s = fma(s, r, 1. / 120.);
  s = fma(s, r, 1. / 24.);
  s = fma(s, r, 1. / 6.);
  s = fma(s, r, 0.5);
  s = fma(s, r, 1.);
  s = fma(s, r, 1.);
  return ldexp(s, (int)fmax(fmin(k, 2000.), -2000.));
}

// LDS floats of a row: odd, so that lanes of neighbouring rows hit different banks.
__host__ __device__ inline int ppo_ld(int na) { return na | 1; }

// A logit less the row's largest; far below zero for an illegal action (so
// that its probability is 0 and a product with it is, too).
__device__ __forceinline__ float below_top(float x, float top) { return x == -INFINITY ? -1e30f : x - top; }

// A wave's walk over the values of its 64 rows, 64 neighbouring ones at a
// time: where value 64 j + lane lies in LDS, for j = 0, 1, ..
struct Walk {
  int at, col, na, skip, dq, dr;
  __device__ Walk(int lane, int na) : na(na) {
    const int ld = ppo_ld(na), row = lane / na;
    dq = 64 / na * ld;
    dr = 64 % na;
    col = lane - row * na;
    at = row * ld + col;
    skip = ld - na;  // from the end of a row to the next
  }
  __device__ void next() {
    at += dq + dr;
    col += dr;
    if (col >= na) {
      col -= na;
      at += skip;
    }
  }
};

// The 64 rows from r0 on, by one wave: gradients written, st added to.
__device__ __forceinline__ void ppo_rows(const PpoArgs& p, const PpoNorm& nm, int64_t r0, float* s,
                                         double (&st)[PPO_STATS]) {
  const int lane = threadIdx.x & 63, na = p.NA;
  const int live = p.R - r0 < 64 ? (int)(p.R - r0) : 64, vals = live * na;
  const int64_t r = r0 + lane;
  const bool counted = lane < live && (!p.mask || p.mask[r]);
  int act = -1;
  float old = 0.f, adv_in = 0.f, value = 0.f, value_old = 0.f, ret = 0.f;
  if (counted) {
    act = p.actions[r];
    old = p.logp_old[r];
    adv_in = p.adv[r];
    value = p.value[r];
    ret = p.ret[r];
    if (p.value_clip > 0.f) value_old = p.value_old[r];
  }
  const float* x_in = p.logits + r0 * na;
  const uint8_t* l_in = p.legal ? p.legal + r0 * na : nullptr;
  Walk to(lane, na);
  for (int j0 = 0; j0 < na; j0 += PPO_CHUNK) {
    float in[PPO_CHUNK];
    uint8_t ok[PPO_CHUNK];
#pragma unroll
    for (int j = 0; j < PPO_CHUNK; ++j) {
      const int e = (j0 + j) * 64 + lane;
      in[j] = -INFINITY;
      ok[j] = 1;
      if (e < vals) {
        in[j] = x_in[e];
        if (l_in) ok[j] = l_in[e];
      }
    }
#pragma unroll
    for (int j = 0; j < PPO_CHUNK; ++j)
      if (j0 + j < na) {  // (rows past the last one: -inf)
        s[to.at] = ok[j] ? in[j] : -INFINITY;
        to.next();
      }
  }
  wave_lds_sync();
  float* x = s + lane * ppo_ld(na);
  float top = -INFINITY;
#pragma unroll 4
  for (int i = 0; i < na; ++i) top = x[i] > top ? x[i] : top;  // (a NaN is met in the sum)
  float sum = 0.f, zsum = 0.f;
#pragma unroll 4
  for (int i = 0; i < na; ++i) {
    const float z = below_top(x[i], top), e = exp_neg(z);
    sum += e;
    zsum += e * z;
  }
  const bool some = !(sum == 0.f);  // a legal action's term is 1, or NaN
  const float logs = some ? logf(sum) : 0.f, inv = some ? 1.f / sum : 0.f;
  const float ent = logs - zsum * inv;  // -sum p log p, log p = z - logs
  float slope = 0.f;                    // d policy / d log p_a
  const float xa = act >= 0 && act < na ? x[act] : -INFINITY;
  if (!(xa == -INFINITY)) {
    const float adv = (float)(((double)adv_in - nm.mean) * nm.rstd);
    const double lo = 1. - (double)p.clip, hi = 1. + (double)p.clip;
    const float diff = xa - top - logs - old, ratio = expf(diff);
    bool below = (double)ratio < lo, above = (double)ratio > hi;
    // near a border the float32 ratio does not say on which side it lies
    const float tol = 1e-6f * (16.f + fabsf(xa) + fabsf(top) + fabsf(old)) * ratio;
    if (fabs((double)ratio - lo) <= tol || fabs((double)ratio - hi) <= tol) {
      // (xa less the log of the sum, less old) against log(1 -+ clip), without logarithms
      double s64 = 0.;
#pragma unroll 1
      for (int i = 0; i < na; ++i) s64 += x[i] == -INFINITY ? 0. : exp64((double)x[i] - (double)top);
      const double e64 = exp64((double)xa - (double)top - (double)old);
      below = e64 < lo * s64;
      above = e64 > hi * s64;
    }
    const float clipped = above ? (float)hi : below ? (float)lo : ratio;
    // the smaller surrogate is the plain one unless the ratio has left the range on the advantage's side
    const bool plain = adv > 0.f ? !above : adv < 0.f ? !below : true;
    st[1] -= (double)((plain ? ratio : clipped) * adv);
    slope = plain ? -adv * ratio : 0.f;
    st[4] += (double)(ratio - 1.f - diff);
    st[5] += below || above ? 1. : 0.;
  }
  if (counted && some) st[3] += (double)ent;
  if (lane < live) {
    double dv = 0.;
    if (counted) {
      const double err = (double)value - ret, off = (double)value - value_old, vc = p.value_clip;
      double loss = 0.5 * err * err;
      dv = err;
      if (vc > 0. && fabs(off) > vc) {
        const double ec = value_old + (off > 0. ? vc : -vc) - ret;
        if (0.5 * ec * ec > loss) {
          loss = 0.5 * ec * ec;
          dv = 0.;
        }
      }
      st[2] += loss;
    }
    p.dvalue[r] = (float)((double)p.value_coef * dv * nm.inv_n);
  }
  const float inv_n = (float)nm.inv_n, c = p.entropy_coef, shift = ent - logs;
  const bool any = counted && some;
#pragma unroll 4
  for (int i = 0; i < na; ++i) {
    const float z = below_top(x[i], top), pi = exp_neg(z) * inv;
    const float d = (slope * ((i == act ? 1.f : 0.f) - pi) + c * pi * (z + shift)) * inv_n;
    x[i] = any && !(x[i] == -INFINITY) ? d : 0.f;
  }
  wave_lds_sync();
  Walk from(lane, na);
#pragma unroll 4
  for (int j = 0; j < na; ++j) {
    const int e = j * 64 + lane;
    if (e < vals) p.dlogits[r0 * na + e] = s[from.at];
    from.next();
  }
  wave_lds_sync();  // (the next rows overwrite s)
}

__device__ __forceinline__ void ppo_means(const PpoArgs& p, const double (&v)[PPO_STATS], double inv_n) {
  if (threadIdx.x != 0) return;
  for (int i = 1; i < PPO_STATS; ++i) p.stats[i] = (float)(v[i] * inv_n);
  p.stats[0] = (float)((v[1] + (double)p.value_coef * v[2] - (double)p.entropy_coef * v[3]) * inv_n);
}

__global__ __launch_bounds__(PPO_SUM_NT) void ppo_adv_kernel(PpoArgs p, PpoPart* part) {
  __shared__ double s[16][3];
  double v[3] = {0., 0., 0.};
  adv_sums(p, (int64_t)blockIdx.x * PPO_SUM_NT + threadIdx.x, (int64_t)gridDim.x * PPO_SUM_NT, v);
  block_sum<3>(v, s);
  if (threadIdx.x == 0)
    for (int i = 0; i < 3; ++i) part->adv[blockIdx.x][i] = v[i];
}

// LDS bytes of a wave: its rows, or its statistics at the end.
__host__ __device__ inline int ppo_wave_bytes(int na) {
  const int rows = 4 * 64 * ppo_ld(na);
  return rows > TURN_BYTES ? rows : TURN_BYTES;
}

__global__ __launch_bounds__(PPO_NT) void ppo_rows_kernel(PpoArgs p, PpoPart* part, int adv_blocks) {
  extern __shared__ double s_dyn[];
  __shared__ double s_stat[16][PPO_STATS];
  PpoNorm nm{1. / (double)p.R, 0., 1.};
  if (adv_blocks) {  // every wave for itself: one partial sum per lane
    double v[3] = {0., 0., 0.};
    const int b = threadIdx.x & 63;  // (PPO_ADV_B <= 64)
    if (b < adv_blocks)
      for (int i = 0; i < 3; ++i) v[i] = part->adv[b][i];
    wave_sum<3>(v);
    nm = ppo_norm(p, v);
    nm = {uniform(nm.inv_n), uniform(nm.mean), uniform(nm.rstd)};
  }
  double st[PPO_STATS] = {0., 0., 0., 0., 0., 0.};
  char* mine = reinterpret_cast<char*>(s_dyn) + (threadIdx.x >> 6) * ppo_wave_bytes(p.NA);
  for (int64_t r0 = (int64_t)blockIdx.x * PPO_NT + (threadIdx.x & ~63); r0 < p.R; r0 += (int64_t)gridDim.x * PPO_NT)
    ppo_rows(p, nm, r0, reinterpret_cast<float*>(mine), st);
  const double t = stats_sum(st, reinterpret_cast<double*>(mine), s_stat);
  if (threadIdx.x < PPO_STATS) part->stat[blockIdx.x][threadIdx.x] = t;
}

// The six means: wave i adds up value i of all workgroups (wave 0 of the six
// the rows' number; short code counts here, the launch is cold each time).
constexpr int STATS_NT = 64 * PPO_STATS;
__global__ __launch_bounds__(STATS_NT) void ppo_stats_kernel(PpoArgs p, const PpoPart* part, int adv_blocks,
                                                             int blocks) {
  __shared__ double s[PPO_STATS];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  double v = 0.;
  if (w == 0)
    for (int b = lane; b < adv_blocks; b += 64) v += part->adv[b][0];
  else
    for (int b = lane; b < blocks; b += 64) v += part->stat[b][w];
#pragma unroll 1
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  if (lane == 0) s[w] = v;
  __syncthreads();
  if (threadIdx.x != 0) return;
  const double n = adv_blocks ? (s[0] > 0. ? s[0] : 1.) : (double)p.R;
  double all[PPO_STATS];
  for (int i = 0; i < PPO_STATS; ++i) all[i] = s[i];
  ppo_means(p, all, 1. / n);
}

// Everything in one workgroup.
__global__ __launch_bounds__(1024) void ppo_small_kernel(PpoArgs p) {
  extern __shared__ double s_dyn[];
  __shared__ double s_adv[16][3], s_stat[16][PPO_STATS], s_all[PPO_STATS];
  double v[3] = {0., 0., 0.};
  adv_sums(p, threadIdx.x, blockDim.x, v);
  block_sum<3>(v, s_adv);
  const PpoNorm nm = ppo_norm(p, v);
  double st[PPO_STATS] = {0., 0., 0., 0., 0., 0.};
  char* mine = reinterpret_cast<char*>(s_dyn) + (threadIdx.x >> 6) * ppo_wave_bytes(p.NA);
  for (int64_t r0 = threadIdx.x & ~63; r0 < p.R; r0 += blockDim.x)
    ppo_rows(p, nm, r0, reinterpret_cast<float*>(mine), st);
  const double t = stats_sum(st, reinterpret_cast<double*>(mine), s_stat);
  if (threadIdx.x < PPO_STATS) s_all[threadIdx.x] = t;
  wave_lds_sync();
  for (int i = 0; i < PPO_STATS; ++i) st[i] = s_all[i];
  ppo_means(p, st, nm.inv_n);
}

}  // namespace

size_t ppo_workspace_bytes(int64_t R) { return R <= PPO_SMALL ? 0 : sizeof(PpoPart); }

hipError_t launch_ppo(const PpoArgs& p, void* workspace, hipStream_t s) {
  const size_t wave = ppo_wave_bytes(p.NA);
  if (p.R <= PPO_SMALL) {
    const int most = (int)((60u << 10) / wave), rows = (int)((p.R + 63) / 64);  // waves that fit in LDS; row tiles
    const int waves = rows < most ? rows : most;
    const int n = waves < 16 ? waves : 16;
    ppo_small_kernel<<<1, 64 * n, wave * n, s>>>(p);
    return hipGetLastError();
  }
  PpoPart* part = static_cast<PpoPart*>(workspace);
  const int64_t tiles = (p.R + PPO_NT - 1) / PPO_NT, sums = (p.R + PPO_SUM_NT - 1) / PPO_SUM_NT;
  const int blocks = (int)(tiles < PPO_ROW_B ? tiles : PPO_ROW_B);
  const int adv_blocks = p.normalize || p.mask ? (int)(sums < PPO_ADV_B ? sums : PPO_ADV_B) : 0;
  if (adv_blocks) ppo_adv_kernel<<<adv_blocks, PPO_SUM_NT, 0, s>>>(p, part);
  ppo_rows_kernel<<<blocks, PPO_NT, wave * (PPO_NT / 64), s>>>(p, part, adv_blocks);
  ppo_stats_kernel<<<1, STATS_NT, 0, s>>>(p, part, adv_blocks, blocks);
  return hipGetLastError();
}

}  // namespace rl
