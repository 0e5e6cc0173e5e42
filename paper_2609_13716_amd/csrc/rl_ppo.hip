// Proximal policy optimisation's loss over stored rows and its gradients.
//
// Three launches: partial sums of the advantages (needed when they are
// normalised or rows are masked out), the rows, and the six means.  Sums over
// rows are float64, taken in an order that depends on the sizes only.
#include "rl_internal.h"

namespace rl {
namespace {

constexpr int PPO_NT = 256;
constexpr int PPO_MAXB = 1024;  // workgroups of a launch, at most (partial sums of each go to the workspace)
constexpr int PPO_STATS = 6;

struct PpoPart {  // workspace
  double adv[PPO_MAXB][3];  // rows counted, sum and sum of squares of their advantages
  double stat[PPO_MAXB][PPO_STATS];
};

template <int N>
__device__ __forceinline__ void block_sum(double (&v)[N], double (*s)[N]) {  // result in thread 0
#pragma unroll
  for (int i = 0; i < N; ++i)
    for (int d = 32; d > 0; d >>= 1) v[i] += __shfl_down(v[i], d, 64);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  if (lane == 0)
    for (int i = 0; i < N; ++i) s[w][i] = v[i];
  __syncthreads();
  if (threadIdx.x == 0)
    for (int i = 0; i < N; ++i) {
      v[i] = s[0][i];
      for (int k = 1; k < PPO_NT / 64; ++k) v[i] += s[k][i];
    }
}

__global__ __launch_bounds__(PPO_NT) void ppo_adv_kernel(PpoArgs p, PpoPart* part) {
  __shared__ double s[PPO_NT / 64][3];
  double v[3] = {0., 0., 0.};
  for (int64_t r = (int64_t)blockIdx.x * PPO_NT + threadIdx.x; r < p.R; r += (int64_t)gridDim.x * PPO_NT) {
    if (p.mask && !p.mask[r]) continue;
    const double a = p.adv[r];
    v[0] += 1.;
    v[1] += a;
    v[2] += a * a;
  }
  block_sum<3>(v, s);
  if (threadIdx.x == 0)
    for (int i = 0; i < 3; ++i) part->adv[blockIdx.x][i] = v[i];
}

__global__ __launch_bounds__(PPO_NT) void ppo_rows_kernel(PpoArgs p, PpoPart* part, int adv_blocks) {
  __shared__ double s_adv[PPO_NT / 64][3], s_stat[PPO_NT / 64][PPO_STATS], s_norm[3];
  if (adv_blocks) {
    double v[3] = {0., 0., 0.};
    for (int b = threadIdx.x; b < adv_blocks; b += PPO_NT)
      for (int i = 0; i < 3; ++i) v[i] += part->adv[b][i];
    block_sum<3>(v, s_adv);
    if (threadIdx.x == 0) {
      const double n = v[0] > 0. ? v[0] : 1., mean = v[1] / n, var = v[2] / n - mean * mean;
      s_norm[0] = 1. / n;
      s_norm[1] = mean;
      s_norm[2] = 1. / (sqrt(var > 0. ? var : (var == var ? 0. : var)) + 1e-8);
    }
    __syncthreads();
  } else if (threadIdx.x == 0) {
    s_norm[0] = 1. / (double)p.R;
  }
  __syncthreads();
  const float inv_n = (float)s_norm[0];
  const double mean = p.normalize ? s_norm[1] : 0., rstd = p.normalize ? s_norm[2] : 1.;
  const double lo = 1. - (double)p.clip, hi = 1. + (double)p.clip, vc = p.value_clip;
  double st[PPO_STATS] = {0., 0., 0., 0., 0., 0.};
  const int NA = p.NA;
  for (int64_t r = (int64_t)blockIdx.x * PPO_NT + threadIdx.x; r < p.R; r += (int64_t)gridDim.x * PPO_NT) {
    const float* x = p.logits + r * NA;
    float* dx = p.dlogits + r * NA;
    if (p.mask && !p.mask[r]) {
      for (int i = 0; i < NA; ++i) dx[i] = 0.f;
      p.dvalue[r] = 0.f;
      continue;
    }
    uint32_t legal = 0;
    for (int i = 0; i < NA; ++i)
      if ((!p.legal || p.legal[r * NA + i]) && !(x[i] == -INFINITY)) legal |= 1u << i;
    float top = -INFINITY, sum = 0.f;
    for (int i = 0; i < NA; ++i)
      if (legal >> i & 1) top = fmaxf(top, x[i]);
    for (int i = 0; i < NA; ++i)
      if (legal >> i & 1) sum += expf(x[i] - top);
    const float logs = logf(sum), inv = 1.f / sum;
    float ent = 0.f;
    for (int i = 0; i < NA; ++i)
      if (legal >> i & 1) {
        const float lp = x[i] - top - logs;
        ent -= expf(x[i] - top) * inv * lp;
      }
    const int act = p.actions[r];
    const bool acts = act >= 0 && act < NA && (legal >> act & 1);
    float slope = 0.f;  // d policy / d log p_a
    if (acts) {
      const float old = p.logp_old[r];
      const float adv = (float)(((double)p.adv[r] - mean) * rstd);
      float diff = x[act] - top - logs - old;
      float ratio = expf(diff);
      bool below = (double)ratio < lo, above = (double)ratio > hi;
      // near a border the float32 ratio does not say on which side it lies
      const float tol = 1e-6f * (16.f + fabsf(x[act]) + fabsf(top) + fabsf(old)) * ratio;
      if (fabs((double)ratio - lo) <= tol || fabs((double)ratio - hi) <= tol) {
        double s64 = 0.;
        for (int i = 0; i < NA; ++i)
          if (legal >> i & 1) s64 += exp((double)x[i] - (double)top);
        const double r64 = exp((double)x[act] - (double)top - log(s64) - (double)old);
        below = r64 < lo;
        above = r64 > hi;
      }
      const float clipped = above ? (float)hi : below ? (float)lo : ratio;
      // the smaller surrogate is the plain one unless the ratio has left the range on the advantage's side
      const bool plain = adv > 0.f ? !above : adv < 0.f ? !below : true;
      st[1] -= (double)((plain ? ratio : clipped) * adv);
      slope = plain ? -adv * ratio : 0.f;
      st[4] += (double)(ratio - 1.f - diff);
      st[5] += below || above ? 1. : 0.;
    }
    if (legal) st[3] += (double)ent;
    for (int i = 0; i < NA; ++i) {
      float d = 0.f;
      if (legal >> i & 1) {
        const float lp = x[i] - top - logs, pi = expf(x[i] - top) * inv;
        d = slope * ((i == act ? 1.f : 0.f) - pi) + p.entropy_coef * pi * (lp + ent);
      }
      dx[i] = d * inv_n;
    }
    const double v = p.value[r], ret = p.ret[r], e = v - ret;
    double loss = 0.5 * e * e, dv = e;
    if (p.value_clip > 0.f) {
      const double vo = p.value_old[r];
      if (fabs(v - vo) > vc) {
        const double ec = vo + (v > vo ? vc : -vc) - ret;
        if (0.5 * ec * ec > loss) {
          loss = 0.5 * ec * ec;
          dv = 0.;
        }
      }
    }
    st[2] += loss;
    p.dvalue[r] = (float)((double)p.value_coef * dv * s_norm[0]);
  }
  block_sum<PPO_STATS>(st, s_stat);
  if (threadIdx.x == 0)
    for (int i = 0; i < PPO_STATS; ++i) part->stat[blockIdx.x][i] = st[i];
}

__global__ __launch_bounds__(PPO_NT) void ppo_stats_kernel(PpoArgs p, PpoPart* part, int adv_blocks, int blocks) {
  __shared__ double s_n[PPO_NT / 64][1], s_stat[PPO_NT / 64][PPO_STATS];
  double n[1] = {0.}, v[PPO_STATS] = {0., 0., 0., 0., 0., 0.};
  for (int b = threadIdx.x; b < adv_blocks; b += PPO_NT) n[0] += part->adv[b][0];
  for (int b = threadIdx.x; b < blocks; b += PPO_NT)
    for (int i = 0; i < PPO_STATS; ++i) v[i] += part->stat[b][i];
  block_sum<1>(n, s_n);
  block_sum<PPO_STATS>(v, s_stat);
  if (threadIdx.x == 0) {
    const double cnt = adv_blocks ? (n[0] > 0. ? n[0] : 1.) : (double)p.R;
    for (int i = 1; i < PPO_STATS; ++i) p.stats[i] = (float)(v[i] / cnt);
    p.stats[0] = (float)((v[1] + (double)p.value_coef * v[2] - (double)p.entropy_coef * v[3]) / cnt);
  }
}

int ppo_blocks(int64_t R) {
  const int64_t b = (R + PPO_NT - 1) / PPO_NT;
  return (int)(b < PPO_MAXB ? b : PPO_MAXB);
}

}  // namespace

size_t ppo_workspace_bytes(int64_t) { return sizeof(PpoPart); }

hipError_t launch_ppo(const PpoArgs& p, void* workspace, hipStream_t s) {
  PpoPart* part = static_cast<PpoPart*>(workspace);
  const int blocks = ppo_blocks(p.R), adv_blocks = p.normalize || p.mask ? blocks : 0;
  if (adv_blocks) ppo_adv_kernel<<<adv_blocks, PPO_NT, 0, s>>>(p, part);
  ppo_rows_kernel<<<blocks, PPO_NT, 0, s>>>(p, part, adv_blocks);
  ppo_stats_kernel<<<1, PPO_NT, 0, s>>>(p, part, adv_blocks, blocks);
  return hipGetLastError();
}

}  // namespace rl
