// Proximal policy optimisation's loss over stored rows and its gradients.
//
// A row's work is its softmax: 8 bytes an action and 28 a row against some 40
// instructions an action and 250 a row, so that HBM and the vector units are
// busy for about as long.  A wave takes 64 consecutive rows: their 64 nA logits
// are read as 16 nA pieces of 16 bytes and turned into one row per lane through
// LDS (illegal actions become -inf on the way), the row stays in registers, and
// the gradients go back the same way.  1048576 rows of 6 take 30 us, 20 of them
// for the rows (3.9 TB/s), the rest for the two other launches.
// A row is float32, as its inputs and outputs are: the softmax, the ratio and the
// gradients are a few float32 steps from float64's.  Log ratio, value loss and
// sums over rows are float64, the sums taken in an order that depends on the
// sizes only: per lane, wave, workgroup, then over workgroups by the launch that
// follows.  Rows for which that is not enough (a ratio at a border, or beyond
// float32) are done again by the whole wave: of usual rows one in 10000.
//   few rows         one workgroup does everything in one launch (500 rows of
//                    6: 7 us of GPU time; 15 in three launches);
//   otherwise        the advantages' sums (when they are normalised or rows
//                    masked out), the rows, the six means.
#include <utility>

#include "rl_internal.h"

namespace rl {
namespace {

constexpr int PPO_NT = 512;         // threads of a workgroup that does rows
constexpr int PPO_SUM_NT = 512;     // of one that adds up advantages
// Whether one workgroup does everything.  Its time grows with rows and actions;
// three launches take 12 to 13 us in a graph, 14 to 16 called one by one,
// whatever there is to do (one workgroup: rows of 6: 2000 12.5 us, 2900 16.5;
// of 9: 1500 12.6, 2000 14.6; of 20: 800 11.9, 1200 14.5; of 32: 1024 15.3).
inline bool ppo_small(int64_t R, int na) { return R * (na + 8) <= 28 * 1024; }
constexpr int PPO_ADV_B = 64, PPO_ROW_B = 512;  // workgroups, at most (their partial sums go to the workspace)
constexpr int PPO_STATS = 6;

// Counted rows, and the sum and sum of squares of their advantages less `from`,
// one of them: so a mean far from 0 costs no digits of the variance.
struct AdvSum {
  double n, sum, sq, from;
  __device__ void add(bool in, float adv) {
    if (in && n == 0.) from = (double)adv;
    const double a = in ? (double)adv - from : 0.;  // (a padded row's value is dropped)
    n += in ? 1. : 0.;
    sum += a;
    sq += a * a;
  }
};

struct PpoPart {  // workspace
  AdvSum adv[PPO_ADV_B];
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

// The lanes' sums put together, for every lane: all taken from the value of the
// first lane that has one.
__device__ __forceinline__ AdvSum wave_sum(const AdvSum& mine) {
  const uint64_t some = __ballot(mine.n > 0.);
  AdvSum r{};
  if (some) r.from = __shfl(mine.from, __ffsll((unsigned long long)some) - 1, 64);
  const double d = mine.n > 0. ? mine.from - r.from : 0.;
  double v[3] = {mine.n, mine.sum + mine.n * d, mine.sq + d * (2. * mine.sum + mine.n * d)};
  wave_sum<3>(v);
  r.n = v[0];
  r.sum = v[1];
  r.sq = v[2];
  return r;
}

// The same over a workgroup (s: one for each wave), for every thread.
__device__ __forceinline__ AdvSum block_sum(const AdvSum& mine, AdvSum* s) {
  const AdvSum v = wave_sum(mine);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
  if (lane == 0) s[w] = v;
  __syncthreads();
  return wave_sum(lane < nw ? s[lane] : AdvSum{});
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

// A thread's part of the rows.
__device__ __forceinline__ AdvSum adv_sums(const PpoArgs& p, int64_t first, int64_t step) {
  AdvSum v{};
#pragma unroll 8
  for (int64_t r = first; r < p.R; r += step) {
    const uint8_t in = p.mask ? p.mask[r] : 1;
    const float read = p.adv[r];  // (before the mask is known)
    v.add(in, read);
  }
  return v;
}

// The same, four neighbouring rows at a time, ADV_U times that in flight; the
// same rows in the same order where they are not aligned to that.
constexpr int ADV_U = 4;
__device__ __forceinline__ AdvSum adv_sums4(const PpoArgs& p, int64_t first, int64_t step) {
  const bool whole = ((reinterpret_cast<uintptr_t>(p.adv) & 15) | (reinterpret_cast<uintptr_t>(p.mask) & 3)) == 0;
  const int64_t fours = p.R / 4;
  AdvSum v{};
  for (int64_t r = first; r < fours; r += ADV_U * step) {
    f32x4 a[ADV_U];
    uint32_t in[ADV_U];
#pragma unroll
    for (int q = 0; q < ADV_U; ++q) {
      const int64_t at = r + q * step < fours ? r + q * step : r;  // (past the last ones: read again, not counted)
      if (whole) {
        a[q] = reinterpret_cast<const f32x4*>(p.adv)[at];
        in[q] = p.mask ? reinterpret_cast<const uint32_t*>(p.mask)[at] : 0x01010101u;
      } else {
        in[q] = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          a[q][k] = p.adv[4 * at + k];
          in[q] |= (p.mask ? (uint32_t)p.mask[4 * at + k] : 1u) << 8 * k;
        }
      }
    }
#pragma unroll
    for (int q = 0; q < ADV_U; ++q) {
      if (r + q * step >= fours) in[q] = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) v.add(in[q] >> 8 * k & 255, a[q][k]);
    }
  }
  const int64_t rest = 4 * fours + first;
  if (rest < p.R) v.add(!p.mask || p.mask[rest], p.adv[rest]);
  return v;
}

struct PpoNorm {
  double inv_n, mean, rstd;
};
__device__ __forceinline__ PpoNorm ppo_norm(const PpoArgs& p, const AdvSum& v) {
  PpoNorm r{1. / (v.n > 0. ? v.n : 1.), 0., 1.};
  if (p.normalize) {
    const double off = v.sum * r.inv_n, var = v.sq * r.inv_n - off * off;
    r.mean = v.from + off;
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

__device__ __forceinline__ float uniform(float v) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}

// Lane w's value, for every lane.
__device__ __forceinline__ float of_lane(float v, int w) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), w));
}

// exp(x): the hardware's 2^t with t = x log2(e) rounded, times
// 1 + ln(2) (x log2(e) - t); within 3 float32 steps for |x| < 2^100 (results
// below 2^-126 are 0).
__device__ __forceinline__ float exp32(float x) {
  constexpr float L2E = 1.4426950408889634f, L2E_LO = (float)(1.4426950408889634 - (double)L2E);
  const float t = x * L2E, r = fmaf(x, L2E_LO, fmaf(x, L2E, -t));
  return __builtin_amdgcn_exp2f(t) * fmaf(r, 0.6931471805599453f, 1.f);
}
// log(x) for x >= 1: the hardware's logarithm to base 2 times ln(2) in two parts.
__device__ __forceinline__ float log32(float x) {
  constexpr float LN2 = 0.6931471805599453f, LN2_LO = (float)(0.6931471805599453 - (double)LN2);
  const float t = __builtin_amdgcn_logf(x);
  return fmaf(t, LN2, t * LN2_LO);
}
// 1 / x for x >= 1: the hardware's, and one Newton step.
__device__ __forceinline__ float rcp32(float x) {
  const float r = __builtin_amdgcn_rcpf(x);
  return fmaf(fmaf(-x, r, 1.f), r, r);
}

// r - 1 - d for r = exp(d), whose rounding it would be near d = 0: there the sum
// of d^k / k! from 2 to 7 (for |d| < 1/4 the next term is 2e-8 of it).
__device__ __forceinline__ double kl_term(double r, double d) {
  const float x = (float)d;
  const float s3 = fmaf(x, fmaf(x, fmaf(x, 1.f / 5040.f, 1.f / 720.f), 1.f / 120.f), 1.f / 24.f);
  const float s = fmaf(x, fmaf(x, s3, 1.f / 6.f), 0.5f);
  return fabsf(x) < 0.25f ? (double)(x * x * s) : r - 1. - d;
}

// exp(x) in float64, to 1e-13: 2^k times the Taylor sum of exp(r) to r^12 / 12!
// for |r| <= ln(2) / 2 (the next term is below 2e-16).  The rows that need it
// are rare; its coefficients stay in memory so that the others do not hold
// registers for them.
__constant__ double INV_FACTORIAL[13] = {
    1.,         1.,          1. / 2.,      1. / 6.,       1. / 24.,       1. / 120.,      1. / 720.,
    1. / 5040., 1. / 40320., 1. / 362880., 1. / 3628800., 1. / 39916800., 1. / 479001600.};
__device__ __forceinline__ double exp64(double x) {
  const double k = rint(x * 1.4426950408889634);
  const double r = fma(-k, 0.6931471805599453, x);
  double s = 0.;
#pragma unroll 1
  for (int i = 12; i >= 0; --i) s = fma(s, r, INV_FACTORIAL[i]);
  return ldexp(s, (int)fmax(fmin(k, 2000.), -2000.));
}

// LDS floats from a row to the next.  Values lie there as they lie in memory,
// so that a lane moves four at a time without knowing their rows; rows of a
// multiple of 8 (whose 64 starts would share few banks) are 4 floats apart.
__host__ __device__ constexpr int ppo_ld(int na) { return na % 8 == 0 ? na + 4 : na; }

// A logit less the row's largest, no lower than LEAST, whose exponential is 0
// in float32 already: the probability of a logit at float32's lowest value (or
// so far from the largest that the difference overflows) is 0, and so are
// products with it.  FAR_BELOW, lower still, stands for an illegal action.
constexpr float FAR_BELOW = -1e30f, LEAST = -200.f;
__device__ __forceinline__ float below_top(float x, float top) {
  const float d = x - top;  // (a NaN stays one)
  return x == -INFINITY ? FAR_BELOW : d < LEAST ? LEAST : d;
}

// v exp(t) / n for a result that fits float32, also where exp(t) or v exp(t)
// does not: three factors exp(t / 3), in an order in which no product is
// larger than both v and the result (t beyond 264: infinite for any v).
__device__ __forceinline__ float times_exp(float v, float t, float inv_n) {
  const float f = exp32((t > 264.f ? 264.f : t) * (1.f / 3.f));
  const bool large = fabsf(v) > 1.f;
  v = (large ? v * inv_n : v) * f;
  return (large ? v : v * inv_n) * f * f;
}

// A lane's row in LDS -> registers, and back, by the widest pieces that every
// row is aligned to.
template <int NA>
__device__ __forceinline__ void row_in(const float* x, float (&z)[NA]) {
  constexpr int V = NA % 4 == 0 ? 4 : NA % 2 == 0 ? 2 : 1;
  typedef float vec __attribute__((ext_vector_type(V)));
#pragma unroll
  for (int i = 0; i < NA; i += V) {
    const vec v = *reinterpret_cast<const vec*>(x + i);
#pragma unroll
    for (int k = 0; k < V; ++k) z[i + k] = v[k];
  }
}
template <int NA>
__device__ __forceinline__ void row_out(float* x, const float (&z)[NA]) {
  constexpr int V = NA % 4 == 0 ? 4 : NA % 2 == 0 ? 2 : 1;
  typedef float vec __attribute__((ext_vector_type(V)));
#pragma unroll
  for (int i = 0; i < NA; i += V) {
    vec v;
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = z[i + k];
    *reinterpret_cast<vec*>(x + i) = v;
  }
}

// The 64 rows from r0 on, by one wave: gradients written, st added to.  A
// row's values stay in registers (the number of actions is a compile-time
// constant for that).
template <int NA>
__device__ __forceinline__ void ppo_rows(const PpoArgs& p, const PpoNorm& nm, int64_t r0, float* s,
                                         double (&st)[PPO_STATS]) {
  constexpr int LD = ppo_ld(NA), Q = (NA + 3) / 4;  // (16 NA times four values)
  const int lane = threadIdx.x & 63;
  const int live = p.R - r0 < 64 ? (int)(p.R - r0) : 64, vals = live * NA;
  const bool real = lane < live;
  const uint32_t r = real ? lane : live - 1;  // (lanes past the last row read it again and count for nothing)
  const bool counted = real && (!p.mask || (p.mask + r0)[r]);
  const int act_in = (p.actions + r0)[r];
  const float old = (p.logp_old + r0)[r], adv_in = (p.adv + r0)[r], value = (p.value + r0)[r], ret = (p.ret + r0)[r];
  const float value_old = p.value_clip > 0.f ? (p.value_old + r0)[r] : 0.f;
  const float* x_in = p.logits + r0 * NA;
  const uint8_t* l_in = p.legal ? p.legal + r0 * NA : nullptr;
  auto at = [](int v) { return LD == NA ? v : v + (LD - NA) * (v / NA); };  // value v of the 64 rows in LDS
  if (live == 64 && ((reinterpret_cast<uintptr_t>(p.logits) & 15) | (reinterpret_cast<uintptr_t>(p.legal) & 3)) == 0) {
    f32x4 in[Q];
    uint32_t ok[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int v = (q * 64 + lane) * 4;
      if ((q + 1) * 256 <= 64 * NA || v < 64 * NA) {
        in[q] = *reinterpret_cast<const f32x4*>(x_in + v);
        if (l_in) ok[q] = *reinterpret_cast<const uint32_t*>(l_in + v);
      }
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int v = (q * 64 + lane) * 4;
      if (l_in)
#pragma unroll
        for (int k = 0; k < 4; ++k) in[q][k] = ok[q] >> 8 * k & 255 ? in[q][k] : -INFINITY;
      if ((q + 1) * 256 <= 64 * NA || v < 64 * NA) *reinterpret_cast<f32x4*>(s + at(v)) = in[q];
    }
  } else {  // (rows past the last one hold what was there: they count for nothing)
#pragma unroll 4
    for (int v = lane; v < vals; v += 64) {
      const float in = x_in[v];
      s[at(v)] = !l_in || l_in[v] ? in : -INFINITY;
    }
  }
  const int act = counted ? act_in : -1;
  wave_lds_sync();
  float* x = s + lane * LD;
  float z[NA], e[NA], top = -INFINITY;
  row_in<NA>(x, z);
#pragma unroll
  for (int i = 0; i < NA; ++i) top = z[i] > top ? z[i] : top;  // (a NaN is met in the sum)
  const float xa = act >= 0 && act < NA ? x[act] : -INFINITY;
  float sum = 0.f, zsum = 0.f;
#pragma unroll
  for (int i = 0; i < NA; ++i) {
    z[i] = below_top(z[i], top);
    e[i] = exp32(z[i]);
    sum += e[i];
    zsum = fmaf(e[i], z[i], zsum);
  }
  const bool some = !(sum == 0.f);  // a legal action's term is 1, or NaN
  const float logs = some ? log32(sum) : 0.f, inv = some ? rcp32(sum) : 0.f;
  const float ent = logs - zsum * inv;  // -sum p log p, log p = z - logs
  float slope = 0.f, adv = 0.f;         // d policy / d log p_a
  bool rare = false;                    // .. is left to the end
  const double lo64 = uniform(1. - (double)p.clip), hi64 = uniform(1. + (double)p.clip);
  const float lo = uniform((float)lo64), hi = uniform((float)hi64);
  if (!(xa == -INFINITY)) {
    adv = (float)(((double)adv_in - nm.mean) * nm.rstd);
    const double diff64 = (double)xa - top - logs - old;  // (of float32 it may pass the range)
    const float diff = (float)diff64, ratio = exp32(diff > 200.f ? 200.f : diff < -200.f ? -200.f : diff);
    const bool below = ratio < lo, above = ratio > hi;
    // the smaller surrogate is the plain one unless the ratio has left the range on the advantage's side
    const bool plain = adv > 0.f ? !above : adv < 0.f ? !below : true;
    // Near a border the float32 ratio does not say on which side it lies: for u = 2^-24 the sum is off by at most 50 u
    // (a term by u z + 6 u, z exp(-z) <= 0.37; 31 additions), its logarithm by as much and 8 u, the difference by
    // u |log r| <= 88 u more, the exponential by 6 u and the border by u: 153 u, less than tol.  The ratio may also be
    // infinite, or make such a product, where float64's does not.
    const float tol = 1e-5f * ratio, product = ratio * adv;
    rare = fminf(fabsf(ratio - lo), fabsf(ratio - hi)) <= tol || !(fabsf(product) <= 1e30f);
    if (!rare) {
      st[1] -= (double)(plain ? product : (above ? hi : below ? lo : ratio) * adv);
      slope = plain ? -product : 0.f;
      st[4] += kl_term((double)ratio, diff64);
      st[5] += below || above ? 1. : 0.;
    }
  }
  if (counted && some) st[3] += (double)ent;
  double dv = 0.;
  if (counted) {
    const double err = (double)value - ret, off = (double)value - value_old, vc = uniform((double)p.value_clip);
    double loss = 0.5 * err * err;
    dv = err;
    if (vc > 0. && fabs(off) > vc) {
      const double ec = value_old + (off > 0. ? vc : -vc) - ret;
      if (0.5 * ec * ec > loss) {
        loss = 0.5 * ec * ec;
        dv = 0.;
      }
    } else if (vc > 0. && off != off) {  // a NaN among the old values would be lost
      loss = dv = off;
    }
    st[2] += loss;
  }
  if (real) (p.dvalue + r0)[r] = (float)(uniform((double)p.value_coef * nm.inv_n) * dv);
  // slope (onehot - p) + c p (log p + H), over n; where p is 0 so is its part of both
  const float inv_n = uniform((float)nm.inv_n), c = uniform(p.entropy_coef * inv_n), shift = ent - logs;
  const float back = slope * inv_n;
  const bool any = counted && some;
#pragma unroll
  for (int i = 0; i < NA; ++i) {
    const float q = e[i] * inv, d = fmaf(c, q * (z[i] + shift), fmaf(-back, q, i == act ? back : 0.f));
    z[i] = any && !(z[i] == FAR_BELOW) ? d : 0.f;
  }
  if (!rare) row_out<NA>(x, z);
  // the rare rows, each by the whole wave (a lane to an action), in float64
  for (uint64_t left = __ballot(rare); left != 0; left &= left - 1) {
    const int w = __ffsll((unsigned long long)left) - 1, wact = __builtin_amdgcn_readlane(act, w);
    const float wtop = of_lane(top, w), wlogs = of_lane(logs, w), winv = of_lane(inv, w), wadv = of_lane(adv, w);
    const double arg = (double)of_lane(xa, w) - (double)wtop - (double)of_lane(old, w), diff64 = arg - (double)wlogs;
    float* row = s + w * LD;
    const float xi = lane < NA ? row[lane] : -INFINITY;
    // (xa less the log of the sum, less old) against log(1 -+ clip), without logarithms: lane 32 (no action's) has the
    // exponential of all but the sum (e^600 times any advantage fits float64, and is infinite in float32 as it should)
    const double mine = exp64(lane == 32 ? (arg > 600. ? 600. : arg) : (double)xi - (double)wtop);
    double s64 = xi == -INFINITY ? 0. : mine;
    for (int d = 32; d > 0; d >>= 1) s64 += __shfl_xor(s64, d, 64);
    const double e64 = __shfl(mine, 32, 64), ratio = e64 / s64;
    const bool below = e64 < lo64 * s64, above = e64 > hi64 * s64;
    const bool plain = wadv > 0.f ? !above : wadv < 0.f ? !below : true;
    if (lane == w) {
      st[1] -= (plain ? ratio : above ? (double)hi : below ? (double)lo : ratio) * (double)wadv;
      st[4] += kl_term(ratio, diff64);
      st[5] += below || above ? 1. : 0.;
    }
    // slope (onehot - p) with ratio and p by their logarithms
    const float zi = below_top(xi, wtop), q = exp32(zi) * winv, by = plain ? wadv : 0.f, diff = (float)diff64;
    const bool me = lane == wact;
    const float d = times_exp(me ? -by * (1.f - q) : by, me ? diff : diff + (zi - wlogs), inv_n);
    const float wshift = of_lane(shift, w);
    if (lane < NA) row[lane] = zi == FAR_BELOW ? 0.f : fmaf(c, q * (zi + wshift), zi == LEAST && !me ? 0.f : d);
  }
  wave_lds_sync();
  float* out = p.dlogits + r0 * NA;
  if (live == 64 && (reinterpret_cast<uintptr_t>(p.dlogits) & 15) == 0) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int v = (q * 64 + lane) * 4;
      if ((q + 1) * 256 <= 64 * NA || v < 64 * NA)
        *reinterpret_cast<f32x4*>(out + v) = *reinterpret_cast<const f32x4*>(s + at(v));
    }
  } else {
#pragma unroll 4
    for (int v = lane; v < vals; v += 64) out[v] = s[at(v)];
  }
  wave_lds_sync();  // (the next rows overwrite s)
}

__device__ __forceinline__ void ppo_means(const PpoArgs& p, const double (&v)[PPO_STATS], double inv_n) {
  if (threadIdx.x != 0) return;
  for (int i = 1; i < PPO_STATS; ++i) p.stats[i] = (float)(v[i] * inv_n);
  p.stats[0] = (float)((v[1] + (double)p.value_coef * v[2] - (double)p.entropy_coef * v[3]) * inv_n);
}

__global__ __launch_bounds__(PPO_SUM_NT) void ppo_adv_kernel(PpoArgs p, PpoPart* part) {
  __shared__ AdvSum s[PPO_SUM_NT / 64];
  const int64_t first = (int64_t)blockIdx.x * PPO_SUM_NT + threadIdx.x, step = (int64_t)gridDim.x * PPO_SUM_NT;
  const AdvSum v = block_sum(adv_sums4(p, first, step), s);
  if (threadIdx.x == 0) part->adv[blockIdx.x] = v;
}

// LDS bytes of a wave: its rows, or its statistics at the end.
__host__ __device__ constexpr int ppo_wave_bytes(int na) {
  const int rows = 4 * 64 * ppo_ld(na);
  return rows > TURN_BYTES ? rows : TURN_BYTES;
}

// Up to 20 actions the registers are held to what four waves of a SIMD may
// have (two workgroups to a CU; at 20 that spills 3 dwords: 655361 masked rows
// 42 us, 46 without); beyond, too much would be spilled (400000 rows of 22: 41
// us, 36 without; of 24: 55 and 38).
template <int NA>
__global__ __launch_bounds__(PPO_NT, NA <= 20 ? 4 : 1) void ppo_rows_kernel(PpoArgs p, PpoPart* part, int adv_blocks) {
  extern __shared__ double s_dyn[];
  __shared__ double s_stat[16][PPO_STATS];
  PpoNorm nm{1. / (double)p.R, 0., 1.};
  if (adv_blocks) {  // every wave for itself: one partial sum per lane
    const int b = threadIdx.x & 63;  // (PPO_ADV_B <= 64)
    nm = ppo_norm(p, wave_sum(b < adv_blocks ? part->adv[b] : AdvSum{}));
    nm = {uniform(nm.inv_n), uniform(nm.mean), uniform(nm.rstd)};
  }
  double st[PPO_STATS] = {0., 0., 0., 0., 0., 0.};
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), step = blockDim.x;
  char* mine = reinterpret_cast<char*>(s_dyn) + w * ppo_wave_bytes(NA);
  for (int64_t r0 = (int64_t)blockIdx.x * step + w * 64; r0 < p.R; r0 += (int64_t)gridDim.x * step)
    ppo_rows<NA>(p, nm, r0, reinterpret_cast<float*>(mine), st);
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
    for (int b = lane; b < adv_blocks; b += 64) v += part->adv[b].n;
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
template <int NA>
__global__ __launch_bounds__(PPO_NT) void ppo_small_kernel(PpoArgs p) {
  extern __shared__ double s_dyn[];
  __shared__ AdvSum s_adv[PPO_NT / 64];
  __shared__ double s_stat[16][PPO_STATS], s_all[PPO_STATS];
  const PpoNorm nm = ppo_norm(p, block_sum(adv_sums(p, threadIdx.x, blockDim.x), s_adv));
  double st[PPO_STATS] = {0., 0., 0., 0., 0., 0.};
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  char* mine = reinterpret_cast<char*>(s_dyn) + w * ppo_wave_bytes(NA);
  for (int64_t r0 = w * 64; r0 < p.R; r0 += blockDim.x)
    ppo_rows<NA>(p, nm, r0, reinterpret_cast<float*>(mine), st);
  const double t = stats_sum(st, reinterpret_cast<double*>(mine), s_stat);
  if (threadIdx.x < PPO_STATS) s_all[threadIdx.x] = t;
  wave_lds_sync();
  for (int i = 0; i < PPO_STATS; ++i) st[i] = s_all[i];
  ppo_means(p, st, nm.inv_n);
}

template <int NA>
hipError_t run_ppo(const PpoArgs& p, void* workspace, hipStream_t s) {
  const size_t wave = ppo_wave_bytes(NA);
  if (ppo_small(p.R, NA)) {
    const int most = (int)((60u << 10) / wave), rows = (int)((p.R + 63) / 64);  // waves that fit in LDS; row tiles
    const int waves = rows < most ? rows : most;
    const int n = waves < PPO_NT / 64 ? waves : PPO_NT / 64;
    ppo_small_kernel<NA><<<1, 64 * n, wave * n, s>>>(p);
    return hipGetLastError();
  }
  PpoPart* part = static_cast<PpoPart*>(workspace);
  const int nt = wave * (PPO_NT / 64) > 62 * 1024 ? PPO_NT / 2 : PPO_NT;  // (a workgroup has 64 KB of LDS)
  const int64_t tiles = (p.R + nt - 1) / nt, sums = (p.R + 4 * PPO_SUM_NT - 1) / (4 * PPO_SUM_NT);
  const int blocks = (int)(tiles < PPO_ROW_B ? tiles : PPO_ROW_B);
  const int adv_blocks = p.normalize || p.mask ? (int)(sums < PPO_ADV_B ? sums : PPO_ADV_B) : 0;
  if (adv_blocks) ppo_adv_kernel<<<adv_blocks, PPO_SUM_NT, 0, s>>>(p, part);
  ppo_rows_kernel<NA><<<blocks, nt, wave * (nt / 64), s>>>(p, part, adv_blocks);
  ppo_stats_kernel<<<1, STATS_NT, 0, s>>>(p, part, adv_blocks, blocks);
  return hipGetLastError();
}

template <int... N>
hipError_t pick_ppo(std::integer_sequence<int, N...>, const PpoArgs& p, void* workspace, hipStream_t s) {
  static constexpr hipError_t (*run[])(const PpoArgs&, void*, hipStream_t) = {run_ppo<N + 1>...};
  return run[p.NA - 1](p, workspace, s);
}

}  // namespace

size_t ppo_workspace_bytes(int64_t R, int na) { return ppo_small(R, na) ? 0 : sizeof(PpoPart); }

hipError_t launch_ppo(const PpoArgs& p, void* workspace, hipStream_t s) {
  return pick_ppo(std::make_integer_sequence<int, MAX_NA>(), p, workspace, s);
}

}  // namespace rl
