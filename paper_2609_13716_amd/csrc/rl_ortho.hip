// Newton-Schulz orthogonalisation of a stack of matrices: X = G / |G|_F, then
// X <- a X + B X with A = X X^T, B = b A + c A A; X is [m, k] with m <= k
// (G transposed where it has more rows than columns).
//
// Arithmetic.  X is kept in float32 and a X is added in float32; every product
// runs on the float16 matrix instructions with both operands split, v = hi +
// lo / 2048 (hi the nearest float16, lo the float16 nearest to 2048 times the
// rest), as hi hi + (hi lo + lo hi) / 2048 accumulated in float32: operands
// keep 22 bits and what is dropped is 2^-22 of a term, at three matrix
// instructions (a float32 matrix instruction has a sixteenth of their rate).
// The splits' errors enter through A and B X only.  Small singular values of X
// grow by `a` a step (485-fold in five), but B X has none of them, so what
// grows with them is the rounding of the float32 X, as in a float32 product.
// Ranges: |X_0|_F = 1 keeps singular values within [0, 1.21], so |X| and |A|
// stay below 1.5 and |B| below 2.9, far inside float16.
//
// Layout.  Operands lie in the workspace as the matrix instruction reads
// them: for 32 rows and 16 columns 1 KB holds lane l's 8 values (row l % 32,
// columns 8 (l / 32) ..), hi followed by lo, so a wave's operand load is 1 KB
// contiguous and needs no LDS.  X is stored once by rows (for X X^T) and once
// by columns (for B X, whose sum runs over X's rows); A and B are symmetric,
// so only tiles on and below the diagonal are computed and written twice.
#include "rl_internal.h"

namespace rl {
namespace {

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float LO_SCALE = 2048.f;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// One operand: [tiles of 32 rows][steps of 16 columns][hi, lo][64 lanes][8].
constexpr int BLOCK = 2 * 512;  // values of a tile and step

__device__ __forceinline__ void split8(const float (&v)[8], f16x8* hi, f16x8* lo) {
  f16x8 h, l;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    h[e] = (_Float16)v[e];
    l[e] = (_Float16)((v[e] - (float)h[e]) * LO_SCALE);
  }
  *hi = h;
  *lo = l;
}

struct NsArgs {
  int rows, cols, dt;  // of G
  int m, k;            // of X: m <= k
  int mp, kp;          // padded with zeros to whole tiles
  _Float16 *x, *t0, *t1, *a, *b;  // operands: X by rows, X by columns (read, written), A, B
  float* xf;           // X [mp, kp]
  const void* g;
  void* out;
  double* part;        // [n, NORM_B] partial sums of squares
};

// ---- norm and first operands ----

constexpr int NORM_NT = 256, NORM_B = 64;

template <int DT>
__global__ __launch_bounds__(NORM_NT) void ns_norm_kernel(NsArgs p) {
  __shared__ double s[NORM_NT / 64];
  using E = typename DType<DT>::T;
  const int64_t len = (int64_t)p.rows * p.cols;
  const E* x = static_cast<const E*>(p.g) + (size_t)blockIdx.y * len;
  double v = 0.;
  for (int64_t i = (int64_t)blockIdx.x * NORM_NT + threadIdx.x; i < len; i += (int64_t)gridDim.x * NORM_NT) {
    const double f = DType<DT>::to_f32(x[i]);
    v += f * f;
  }
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    v = s[0];
    for (int w = 1; w < NORM_NT / 64; ++w) v += s[w];
    p.part[(size_t)blockIdx.y * NORM_B + blockIdx.x] = v;
  }
}

constexpr int TS = 32, LDT = TS + 4;  // a tile of results in LDS, rows 16-byte aligned

// The tile's values (i0.., j0..) as operand rows, columns running along the
// sum: nt threads, 8 values each.
__device__ __forceinline__ void put_rows(const float* s, _Float16* op, int i0, int j0, int steps, int tid) {
  if (tid < TS * TS / 8) {
    const int i = tid & 31, j8 = tid >> 5;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = s[i * LDT + j8 * 8 + e];
    _Float16* q = op + ((size_t)(i0 / 32) * steps + j0 / 16 + j8 / 2) * BLOCK + (i + 32 * (j8 & 1)) * 8;
    split8(v, reinterpret_cast<f16x8*>(q), reinterpret_cast<f16x8*>(q + 512));
  }
}
// The same of the transposed tile: operand rows j, the sum along i.
__device__ __forceinline__ void put_cols(const float* s, _Float16* op, int i0, int j0, int steps, int tid) {
  if (tid < TS * TS / 8) {
    const int j = tid & 31, i8 = tid >> 5;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = s[(i8 * 8 + e) * LDT + j];
    _Float16* q = op + ((size_t)(j0 / 32) * steps + i0 / 16 + i8 / 2) * BLOCK + (j + 32 * (i8 & 1)) * 8;
    split8(v, reinterpret_cast<f16x8*>(q), reinterpret_cast<f16x8*>(q + 512));
  }
}

template <int DT>
__global__ __launch_bounds__(256) void ns_init_kernel(NsArgs p, int norm_blocks) {
  __shared__ float s[TS * LDT];
  using E = typename DType<DT>::T;
  const int tid = threadIdx.x, i0 = blockIdx.y * TS, j0 = blockIdx.x * TS;
  const size_t mat = blockIdx.z, xsz = (size_t)p.mp * p.kp;
  double sum = 0.;
  for (int b = 0; b < norm_blocks; ++b) sum += p.part[mat * NORM_B + b];
  const double inv = sum == 0. ? 0. : 1. / sqrt(sum);
  const E* g = static_cast<const E*>(p.g) + mat * p.rows * p.cols;
  const bool flip = p.rows > p.cols;
  for (int q = tid; q < TS * TS; q += 256) {
    const int c = q & 31, r = q >> 5;  // c runs along G's rows in memory
    const int i = flip ? c : r, j = flip ? r : c;
    float v = 0.f;
    if (i0 + i < p.m && j0 + j < p.k) {
      const size_t at = flip ? (size_t)(j0 + j) * p.cols + i0 + i : (size_t)(i0 + i) * p.cols + j0 + j;
      v = (float)((double)DType<DT>::to_f32(g[at]) * inv);
    }
    s[i * LDT + j] = v;
  }
  __syncthreads();
  for (int q = tid; q < TS * TS; q += 256)
    p.xf[mat * xsz + (size_t)(i0 + (q >> 5)) * p.kp + j0 + (q & 31)] = s[(q >> 5) * LDT + (q & 31)];
  put_rows(s, p.x + mat * xsz * 2, i0, j0, p.kp / 16, tid);
  put_cols(s, p.t0 + mat * xsz * 2, i0, j0, p.mp / 16, tid);
}

// ---- products ----

enum { NS_GRAM = 0, NS_POLY = 1, NS_STEP = 2, NS_LAST = 3 };

// One 32 x 32 tile per workgroup; its waves share out the steps of the sum
// (few tiles and short sums: what counts is how soon a product is done) and
// their partial tiles are added through LDS.
constexpr int NS_W = 4;      // waves of a workgroup
constexpr int NS_AHEAD = 4;  // steps whose operands are loaded ahead

template <int MODE, int DT>
__global__ __launch_bounds__(64 * NS_W) void ns_tile_kernel(NsArgs p) {
  __shared__ float s[NS_W][TS * LDT];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const size_t mat = blockIdx.y, xsz = (size_t)p.mp * p.kp, asz = (size_t)p.mp * p.mp;
  int ti, tj;
  if constexpr (MODE == NS_GRAM || MODE == NS_POLY) {  // the lower triangle, row by row
    const int id = blockIdx.x;
    ti = (int)((sqrtf(8.f * id + 1.f) - 1.f) * 0.5f);
    while ((ti + 1) * (ti + 2) / 2 <= id) ++ti;
    while (ti * (ti + 1) / 2 > id) --ti;
    tj = id - ti * (ti + 1) / 2;
  } else {
    const int nj = p.kp / TS;
    ti = blockIdx.x / nj;
    tj = blockIdx.x - ti * nj;
  }
  const int steps = (MODE == NS_GRAM ? p.kp : p.mp) / 16;
  const _Float16 *P, *Q;
  if constexpr (MODE == NS_GRAM) P = Q = p.x + mat * xsz * 2;
  else if constexpr (MODE == NS_POLY) P = Q = p.a + mat * asz * 2;
  else P = p.b + mat * asz * 2, Q = p.t0 + mat * xsz * 2;
  P += (size_t)ti * steps * BLOCK + lane * 8;
  Q += (size_t)tj * steps * BLOCK + lane * 8;
  const int per = (steps + NS_W - 1) / NS_W, lo = w * per, hi = lo + per < steps ? lo + per : steps;
  f32x16 acc = {}, low = {};
  f16x8 f[NS_AHEAD][4];
  auto fetch = [&](f16x8 (&d)[4], int st) {
    d[0] = *reinterpret_cast<const f16x8*>(P + (size_t)st * BLOCK);
    d[1] = *reinterpret_cast<const f16x8*>(P + (size_t)st * BLOCK + 512);
    d[2] = *reinterpret_cast<const f16x8*>(Q + (size_t)st * BLOCK);
    d[3] = *reinterpret_cast<const f16x8*>(Q + (size_t)st * BLOCK + 512);
  };
#pragma unroll
  for (int q = 0; q < NS_AHEAD; ++q)
    if (lo + q < hi) fetch(f[q], lo + q);
  for (int st = lo; st < hi; st += NS_AHEAD) {
#pragma unroll
    for (int q = 0; q < NS_AHEAD; ++q)
      if (st + q < hi) {
        low = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[q][0], f[q][3], low, 0, 0, 0);
        low = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[q][1], f[q][2], low, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[q][0], f[q][2], acc, 0, 0, 0);
        if (st + q + NS_AHEAD < hi) fetch(f[q], st + q + NS_AHEAD);
      }
  }
#pragma unroll
  for (int r = 0; r < 16; ++r)
    s[w][(8 * (r / 4) + 4 * (lane >> 5) + r % 4) * LDT + (lane & 31)] = fmaf(low[r], 1.f / LO_SCALE, acc[r]);
  __syncthreads();
  // the tile's result in s[0]; a thread's 4 values lie in one row
  const int i0 = ti * TS, j0 = tj * TS;
  float* res = s[0];
  {
    const int i = tid >> 3, j = (tid & 7) * 4;
    f32x4 v = *reinterpret_cast<const f32x4*>(&s[0][i * LDT + j]);
#pragma unroll
    for (int q = 1; q < NS_W; ++q) v += *reinterpret_cast<const f32x4*>(&s[q][i * LDT + j]);
    if constexpr (MODE == NS_POLY) {
      const _Float16* a = p.a + mat * asz * 2 + ((size_t)ti * steps + (j0 + j) / 16) * BLOCK +
                          (i + 32 * (((j0 + j) & 15) / 8)) * 8 + (j & 7);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = NS_C * v[e] + NS_B * ((float)a[e] + (float)a[512 + e] * (1.f / LO_SCALE));
    }
    if constexpr (MODE == NS_STEP || MODE == NS_LAST) {
      f32x4* x = reinterpret_cast<f32x4*>(p.xf + mat * xsz + (size_t)(i0 + i) * p.kp + j0 + j);
      const f32x4 old = *x;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(NS_A, old[e], v[e]);
      if constexpr (MODE == NS_STEP) *x = v;
    }
    *reinterpret_cast<f32x4*>(&res[i * LDT + j]) = v;
  }
  __syncthreads();
  if constexpr (MODE == NS_GRAM || MODE == NS_POLY) {
    _Float16* o = (MODE == NS_GRAM ? p.a : p.b) + mat * asz * 2;
    put_rows(res, o, i0, j0, p.mp / 16, tid);
    if (ti != tj) put_cols(res, o, i0, j0, p.mp / 16, tid);
  } else if constexpr (MODE == NS_STEP) {
    put_rows(res, p.x + mat * xsz * 2, i0, j0, p.kp / 16, tid);
    put_cols(res, p.t1 + mat * xsz * 2, i0, j0, p.mp / 16, tid);
  } else {
    using E = typename DType<DT>::T;
    E* out = static_cast<E*>(p.out) + mat * p.rows * p.cols;
    const bool flip = p.rows > p.cols;
    for (int q = tid; q < TS * TS; q += 64 * NS_W) {
      const int c = q & 31, r = q >> 5;
      const int i = flip ? c : r, j = flip ? r : c;
      if (i0 + i < p.m && j0 + j < p.k)
        out[flip ? (size_t)(j0 + j) * p.cols + i0 + i : (size_t)(i0 + i) * p.cols + j0 + j] =
            DType<DT>::from_f32(res[i * LDT + j]);
    }
  }
}

struct OrthoLayout {
  int m, k, mp, kp;
  size_t off_x, off_t0, off_t1, off_xf, off_a, off_b, bytes;
};
size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
OrthoLayout ortho_layout(const OrthoArgs& p) {
  OrthoLayout L;
  L.m = p.rows < p.cols ? p.rows : p.cols;
  L.k = p.rows < p.cols ? p.cols : p.rows;
  L.mp = round_up(L.m, TS);
  L.kp = round_up(L.k, TS);
  const size_t x = (size_t)p.n * L.mp * L.kp * 4, a = (size_t)p.n * L.mp * L.mp * 4;  // 4 bytes a value, split or not
  L.off_x = round256((size_t)p.n * NORM_B * sizeof(double));
  L.off_t0 = L.off_x + x;
  L.off_t1 = L.off_t0 + x;
  L.off_xf = L.off_t1 + x;
  L.off_a = L.off_xf + x;
  L.off_b = L.off_a + a;
  L.bytes = L.off_b + a;
  return L;
}

template <int DT>
void run_ortho(const OrthoArgs& o, const OrthoLayout& L, NsArgs p, hipStream_t s) {
  const int64_t len = (int64_t)o.rows * o.cols;
  const int nb = (int)((len + 4095) / 4096 < NORM_B ? (len + 4095) / 4096 : NORM_B);
  ns_norm_kernel<DT><<<dim3(nb, o.n), NORM_NT, 0, s>>>(p);
  ns_init_kernel<DT><<<dim3(L.kp / TS, L.mp / TS, o.n), 256, 0, s>>>(p, nb);
  const int mt = L.mp / TS, lower = mt * (mt + 1) / 2, all = mt * (L.kp / TS);
  for (int i = 0; i < o.steps; ++i) {
    ns_tile_kernel<NS_GRAM, DT><<<dim3(lower, o.n), 64 * NS_W, 0, s>>>(p);
    ns_tile_kernel<NS_POLY, DT><<<dim3(lower, o.n), 64 * NS_W, 0, s>>>(p);
    if (i + 1 < o.steps) ns_tile_kernel<NS_STEP, DT><<<dim3(all, o.n), 64 * NS_W, 0, s>>>(p);
    else ns_tile_kernel<NS_LAST, DT><<<dim3(all, o.n), 64 * NS_W, 0, s>>>(p);
    _Float16* t = p.t0;
    p.t0 = p.t1;
    p.t1 = t;
  }
}

}  // namespace

size_t ortho_workspace_bytes(const OrthoArgs& p) { return ortho_layout(p).bytes; }

hipError_t launch_ortho(const OrthoArgs& o, const void* g, void* out, void* workspace, hipStream_t s) {
  const OrthoLayout L = ortho_layout(o);
  char* ws = static_cast<char*>(workspace);
  auto half = [&](size_t off) { return reinterpret_cast<_Float16*>(ws + off); };
  const NsArgs p{o.rows, o.cols, o.dt, L.m, L.k, L.mp, L.kp, half(L.off_x), half(L.off_t0), half(L.off_t1),
                 half(L.off_a), half(L.off_b), reinterpret_cast<float*>(ws + L.off_xf), g, out,
                 reinterpret_cast<double*>(ws)};
  if (o.dt == DT_F32) run_ortho<DT_F32>(o, L, p, s);
  else run_ortho<DT_BF16>(o, L, p, s);
  return hipGetLastError();
}

}  // namespace rl
