// Newton-Schulz orthogonalisation of a stack of matrices: X = G / |G|_F, then
// X <- a X + (b A + c A A) X with A = X X^T, in float32.  X is stored [m, k]
// with m <= k (transposed where G has more rows than columns).
#include "rl_internal.h"

namespace rl {
namespace {

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr int NORM_NT = 256;

// One workgroup per matrix: 1 / |G|_F (0 for a zero matrix), summed in float64.
template <int DT>
__global__ __launch_bounds__(NORM_NT) void ns_norm_kernel(const void* g, int64_t len, double* inv) {
  __shared__ double s[NORM_NT];
  using E = typename DType<DT>::T;
  const E* x = static_cast<const E*>(g) + (size_t)blockIdx.x * len;
  double v = 0.;
  for (int64_t i = threadIdx.x; i < len; i += NORM_NT) {
    const double f = DType<DT>::to_f32(x[i]);
    v += f * f;
  }
  s[threadIdx.x] = v;
  __syncthreads();
  for (int d = NORM_NT / 2; d > 0; d >>= 1) {
    if (threadIdx.x < d) s[threadIdx.x] += s[threadIdx.x + d];
    __syncthreads();
  }
  if (threadIdx.x == 0) inv[blockIdx.x] = s[0] == 0. ? 0. : 1. / sqrt(s[0]);
}

template <int DT>
__global__ void ns_init_kernel(const void* g, int rows, int cols, const double* inv, float* x) {
  using E = typename DType<DT>::T;
  const size_t base = (size_t)blockIdx.y * rows * cols;
  const bool flip = rows > cols;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < (int64_t)rows * cols;
       i += (int64_t)gridDim.x * blockDim.x) {
    const int r = (int)(i / cols), c = (int)(i - (int64_t)r * cols);
    const float v = (float)((double)DType<DT>::to_f32(static_cast<const E*>(g)[base + i]) * inv[blockIdx.y]);
    x[base + (flip ? (size_t)c * rows + r : (size_t)i)] = v;
  }
}

template <int DT>
__global__ void ns_store_kernel(const float* x, int rows, int cols, void* out) {
  using E = typename DType<DT>::T;
  const size_t base = (size_t)blockIdx.y * rows * cols;
  const bool flip = rows > cols;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < (int64_t)rows * cols;
       i += (int64_t)gridDim.x * blockDim.x) {
    const int r = (int)(i / cols), c = (int)(i - (int64_t)r * cols);
    static_cast<E*>(out)[base + i] = DType<DT>::from_f32(x[base + (flip ? (size_t)c * rows + r : (size_t)i)]);
  }
}

// C [M, N] = alpha P Q' + beta D for each matrix of the stack, Q' = Q^T [N, K] when QT, else Q [K, N];
// 32 x 32 tiles through LDS.
template <bool QT>
__global__ __launch_bounds__(256) void ns_gemm_kernel(const float* P, const float* Q, const float* D, float* C, int M,
                                                      int N, int K, float alpha, float beta) {
  __shared__ float sp[32][33], sq[32][33];
  P += (size_t)blockIdx.z * M * K;
  Q += (size_t)blockIdx.z * N * K;
  D += (size_t)blockIdx.z * M * N;
  C += (size_t)blockIdx.z * M * N;
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, m0 = blockIdx.y * 32, n0 = blockIdx.x * 32;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < K; k0 += 32) {
    for (int i = ty; i < 32; i += 8) {
      const int m = m0 + i, k = k0 + tx;
      sp[i][tx] = m < M && k < K ? P[(size_t)m * K + k] : 0.f;
      if (QT) {  // sq[n][k]
        const int n = n0 + i;
        sq[i][tx] = n < N && k < K ? Q[(size_t)n * K + k] : 0.f;
      } else {
        const int kk = k0 + i, n = n0 + tx;
        sq[tx][i] = n < N && kk < K ? Q[(size_t)kk * N + n] : 0.f;
      }
    }
    __syncthreads();
    for (int k = 0; k < 32; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = fmaf(sp[ty + 8 * j][k], sq[tx][k], acc[j]);
    __syncthreads();
  }
  for (int j = 0; j < 4; ++j) {
    const int m = m0 + ty + 8 * j, n = n0 + tx;
    if (m < M && n < N) {
      const size_t i = (size_t)m * N + n;
      C[i] = alpha * acc[j] + (beta != 0.f ? beta * D[i] : 0.f);
    }
  }
}

struct OrthoLayout {
  size_t off_x, off_y, off_a, off_b, bytes;
};
OrthoLayout ortho_layout(const OrthoArgs& p) {
  const size_t m = p.rows < p.cols ? p.rows : p.cols, k = p.rows < p.cols ? p.cols : p.rows;
  const size_t x = ((size_t)p.n * m * k * 4 + 255) & ~(size_t)255, a = ((size_t)p.n * m * m * 4 + 255) & ~(size_t)255;
  OrthoLayout L;
  L.off_x = ((size_t)p.n * 8 + 255) & ~(size_t)255;
  L.off_y = L.off_x + x;
  L.off_a = L.off_y + x;
  L.off_b = L.off_a + a;
  L.bytes = L.off_b + a;
  return L;
}

}  // namespace

size_t ortho_workspace_bytes(const OrthoArgs& p) { return ortho_layout(p).bytes; }

hipError_t launch_ortho(const OrthoArgs& p, const void* g, void* out, void* workspace, hipStream_t s) {
  const OrthoLayout L = ortho_layout(p);
  char* ws = static_cast<char*>(workspace);
  double* inv = reinterpret_cast<double*>(ws);
  float *x = reinterpret_cast<float*>(ws + L.off_x), *y = reinterpret_cast<float*>(ws + L.off_y);
  float *a = reinterpret_cast<float*>(ws + L.off_a), *b = reinterpret_cast<float*>(ws + L.off_b);
  const int m = p.rows < p.cols ? p.rows : p.cols, k = p.rows < p.cols ? p.cols : p.rows;
  const int64_t len = (int64_t)p.rows * p.cols;
  const dim3 ew((unsigned)((len + 255) / 256 < 1024 ? (len + 255) / 256 : 1024), p.n);
  const auto tiles = [&](int M, int N) { return dim3((N + 31) / 32, (M + 31) / 32, p.n); };
  if (p.dt == DT_F32) {
    ns_norm_kernel<DT_F32><<<p.n, NORM_NT, 0, s>>>(g, len, inv);
    ns_init_kernel<DT_F32><<<ew, 256, 0, s>>>(g, p.rows, p.cols, inv, x);
  } else {
    ns_norm_kernel<DT_BF16><<<p.n, NORM_NT, 0, s>>>(g, len, inv);
    ns_init_kernel<DT_BF16><<<ew, 256, 0, s>>>(g, p.rows, p.cols, inv, x);
  }
  for (int i = 0; i < p.steps; ++i) {
    ns_gemm_kernel<true><<<tiles(m, m), 256, 0, s>>>(x, x, a, a, m, m, k, 1.f, 0.f);
    ns_gemm_kernel<true><<<tiles(m, m), 256, 0, s>>>(a, a, a, b, m, m, m, NS_C, NS_B);
    ns_gemm_kernel<false><<<tiles(m, k), 256, 0, s>>>(b, x, x, y, m, k, m, 1.f, NS_A);
    float* t = x;
    x = y;
    y = t;
  }
  if (p.dt == DT_F32) ns_store_kernel<DT_F32><<<ew, 256, 0, s>>>(x, p.rows, p.cols, out);
  else ns_store_kernel<DT_BF16><<<ew, 256, 0, s>>>(x, p.rows, p.cols, out);
  return hipGetLastError();
}

}  // namespace rl
