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

constexpr int NORM_NT = 256, NORM_B = 256;  // workgroups for a matrix's norm, at most

template <int DT>
__global__ __launch_bounds__(NORM_NT) void ns_norm_kernel(NsArgs p) {
  __shared__ double s[NORM_NT / 64];
  using E = typename DType<DT>::T;
  const int64_t len = (int64_t)p.rows * p.cols;
  const E* x = static_cast<const E*>(p.g) + (size_t)blockIdx.y * len;
  double v = 0.;
#pragma unroll 8
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
// sum: 8 values at a time, by nt threads.
__device__ __forceinline__ void put_rows(const float* s, _Float16* op, int i0, int j0, int steps, int tid, int nt) {
  for (int c = tid; c < TS * TS / 8; c += nt) {
    const int i = c & 31, j8 = c >> 5;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = s[i * LDT + j8 * 8 + e];
    _Float16* q = op + ((size_t)(i0 / 32) * steps + j0 / 16 + j8 / 2) * BLOCK + (i + 32 * (j8 & 1)) * 8;
    split8(v, reinterpret_cast<f16x8*>(q), reinterpret_cast<f16x8*>(q + 512));
  }
}
// The same of the transposed tile: operand rows j, the sum along i.
__device__ __forceinline__ void put_cols(const float* s, _Float16* op, int i0, int j0, int steps, int tid, int nt) {
  for (int c = tid; c < TS * TS / 8; c += nt) {
    const int j = c & 31, i8 = c >> 5;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = s[(i8 * 8 + e) * LDT + j];
    _Float16* q = op + ((size_t)(j0 / 32) * steps + i0 / 16 + i8 / 2) * BLOCK + (j + 32 * (i8 & 1)) * 8;
    split8(v, reinterpret_cast<f16x8*>(q), reinterpret_cast<f16x8*>(q + 512));
  }
}

// X_0 in its three forms, one tile of 32 x 32 per workgroup.
constexpr int INIT_NT = 256;
template <int DT>
__global__ __launch_bounds__(INIT_NT) void ns_init_kernel(NsArgs p, int norm_blocks) {
  __shared__ float s[TS * LDT];
  using E = typename DType<DT>::T;
  const int tid = threadIdx.x, i0 = blockIdx.y * TS, j0 = blockIdx.x * TS;
  const size_t mat = blockIdx.z, xsz = (size_t)p.mp * p.kp;
  const E* g = static_cast<const E*>(p.g) + mat * p.rows * p.cols;
  const bool flip = p.rows > p.cols;
  float in[TS * TS / INIT_NT];
#pragma unroll
  for (int u = 0; u < TS * TS / INIT_NT; ++u) {
    const int q = tid + u * INIT_NT, c = q & 31, r = q >> 5;  // c runs along G's rows in memory
    const int i = flip ? c : r, j = flip ? r : c;
    in[u] = 0.f;
    if (i0 + i < p.m && j0 + j < p.k)
      in[u] = DType<DT>::to_f32(g[flip ? (size_t)(j0 + j) * p.cols + i0 + i : (size_t)(i0 + i) * p.cols + j0 + j]);
  }
  double sum = 0.;
  for (int b = tid & 63; b < norm_blocks; b += 64) sum += p.part[mat * NORM_B + b];  // every wave for itself
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
  const double inv = sum == 0. ? 0. : 1. / sqrt(sum);
#pragma unroll
  for (int u = 0; u < TS * TS / INIT_NT; ++u) {
    const int q = tid + u * INIT_NT, c = q & 31, r = q >> 5;
    s[flip ? c * LDT + r : r * LDT + c] = (float)((double)in[u] * inv);
  }
  __syncthreads();
  for (int q = tid; q < TS * TS; q += INIT_NT)
    p.xf[mat * xsz + (size_t)(i0 + (q >> 5)) * p.kp + j0 + (q & 31)] = s[(q >> 5) * LDT + (q & 31)];
  put_rows(s, p.x + mat * xsz * 2, i0, j0, p.kp / 16, tid, INIT_NT / 2);
  if (tid >= INIT_NT / 2) put_cols(s, p.t0 + mat * xsz * 2, i0, j0, p.mp / 16, tid - INIT_NT / 2, INIT_NT / 2);
}

// ---- products ----

enum { NS_GRAM = 0, NS_POLY = 1, NS_STEP = 2, NS_LAST = 3 };

// Where a product's operands lie: rows of P times rows of Q, `steps` steps of 16.
template <int MODE>
struct Operands {
  const _Float16 *P, *Q;
  int steps;
  __device__ Operands(const NsArgs& p, size_t mat) {
    const size_t xsz = (size_t)p.mp * p.kp * 2, asz = (size_t)p.mp * p.mp * 2;
    steps = (MODE == NS_GRAM ? p.kp : p.mp) / 16;
    if constexpr (MODE == NS_GRAM) P = Q = p.x + mat * xsz;
    else if constexpr (MODE == NS_POLY) P = Q = p.a + mat * asz;
    else {
      P = p.b + mat * asz;
      Q = p.t0 + mat * xsz;
    }
  }
};

// Tile id of a symmetric result: the lower triangle, row by row.
__device__ __forceinline__ void lower_tile(int id, int& ti, int& tj) {
  ti = (int)((sqrtf(8.f * id + 1.f) - 1.f) * 0.5f);
  while ((ti + 1) * (ti + 2) / 2 <= id) ++ti;
  while (ti * (ti + 1) / 2 > id) --ti;
  tj = id - ti * (ti + 1) / 2;
}

// Workgroups of a 1-D grid go to the 8 XCDs in turn, each with an L2 cache of
// its own; this gives each XCD a run of neighbouring tiles instead (and, with
// several matrices, whole matrices), which share operands.
struct Tile {
  size_t mat;
  int ti, tj;
};
template <int MODE>
__device__ __forceinline__ Tile next_tile(int tiles, int nj) {
  const int total = gridDim.x, q = total / 8, r = total % 8, x = blockIdx.x % 8;
  const int id = x * q + (x < r ? x : r) + blockIdx.x / 8, mat = id / tiles, t = id - mat * tiles;
  Tile o{(size_t)mat, 0, 0};
  if constexpr (MODE == NS_GRAM || MODE == NS_POLY) {
    lower_tile(t, o.ti, o.tj);
  } else {
    o.ti = t / nj;
    o.tj = t - o.ti * nj;
  }
  return o;
}

// The 64 lanes' accumulators of a tile -> LDS.
__device__ __forceinline__ void acc_to_lds(const f32x16& acc, const f32x16& low, float* s, int lane) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
    s[(8 * (r / 4) + 4 * (lane >> 5) + r % 4) * LDT + (lane & 31)] = fmaf(low[r], 1.f / LO_SCALE, acc[r]);
}

// What a product's value v (4 of a row: row i, columns j.. of the tile at i0,
// j0) becomes: B from A A, or the new X, which is stored in float32, too.
template <int MODE>
__device__ __forceinline__ f32x4 finish4(const NsArgs& p, size_t mat, int i0, int j0, int i, int j, f32x4 v) {
  if constexpr (MODE == NS_POLY) {
    const _Float16* a = p.a + mat * p.mp * p.mp * 2 + ((size_t)(i0 / 32) * (p.mp / 16) + (j0 + j) / 16) * BLOCK +
                        (i + 32 * (((j0 + j) & 15) / 8)) * 8 + (j & 7);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = NS_C * v[e] + NS_B * ((float)a[e] + (float)a[512 + e] * (1.f / LO_SCALE));
  }
  if constexpr (MODE == NS_STEP || MODE == NS_LAST) {
    f32x4* x = reinterpret_cast<f32x4*>(p.xf + mat * p.mp * p.kp + (size_t)(i0 + i) * p.kp + j0 + j);
    const f32x4 old = *x;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(NS_A, old[e], v[e]);
    if constexpr (MODE == NS_STEP) *x = v;
  }
  return v;
}

// The finished tile in LDS -> its operands, or the caller's matrix.
template <int MODE, int DT>
__device__ __forceinline__ void put_tile(const NsArgs& p, size_t mat, int i0, int j0, const float* res, int tid, int nt) {
  if constexpr (MODE == NS_GRAM || MODE == NS_POLY) {
    _Float16* o = (MODE == NS_GRAM ? p.a : p.b) + mat * p.mp * p.mp * 2;
    put_rows(res, o, i0, j0, p.mp / 16, tid, nt);
    if (i0 != j0) put_cols(res, o, i0, j0, p.mp / 16, tid, nt);
  } else if constexpr (MODE == NS_STEP) {
    put_rows(res, p.x + mat * p.mp * p.kp * 2, i0, j0, p.kp / 16, tid, nt);
    put_cols(res, p.t1 + mat * p.mp * p.kp * 2, i0, j0, p.mp / 16, tid, nt);
  } else {
    using E = typename DType<DT>::T;
    E* out = static_cast<E*>(p.out) + mat * p.rows * p.cols;
    const bool flip = p.rows > p.cols;
    for (int q = tid; q < TS * TS; q += nt) {
      const int c = q & 31, r = q >> 5;
      const int i = flip ? c : r, j = flip ? r : c;
      if (i0 + i < p.m && j0 + j < p.k)
        out[flip ? (size_t)(j0 + j) * p.cols + i0 + i : (size_t)(i0 + i) * p.cols + j0 + j] =
            DType<DT>::from_f32(res[i * LDT + j]);
    }
  }
}

__device__ __forceinline__ void mfma3(const f16x8 (&a)[2], const f16x8 (&b)[2], f32x16& acc, f32x16& low) {
  low = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0], b[1], low, 0, 0, 0);
  low = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[1], b[0], low, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0], b[0], acc, 0, 0, 0);
}
__device__ __forceinline__ void fetch2(const _Float16* p, f16x8 (&d)[2]) {
  d[0] = *reinterpret_cast<const f16x8*>(p);
  d[1] = *reinterpret_cast<const f16x8*>(p + 512);
}

// Few tiles and short sums, where what counts is how soon a product is done:
// one 32 x 32 tile per workgroup, whose waves share out the steps of the sum
// and add their partial tiles through LDS.
constexpr int NS_W = 4;      // waves of a workgroup
constexpr int NS_AHEAD = 4;  // steps whose operands are loaded ahead

template <int MODE, int DT>
__global__ __launch_bounds__(64 * NS_W) void ns_tile_kernel(NsArgs p, int tiles) {
  __shared__ float s[NS_W][TS * LDT];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Tile tile = next_tile<MODE>(tiles, p.kp / TS);
  const size_t mat = tile.mat;
  const int ti = tile.ti, tj = tile.tj;
  const Operands<MODE> op(p, mat);
  const _Float16* P = op.P + (size_t)ti * op.steps * BLOCK + lane * 8;
  const _Float16* Q = op.Q + (size_t)tj * op.steps * BLOCK + lane * 8;
  const int per = (op.steps + NS_W - 1) / NS_W, lo = w * per, hi = lo + per < op.steps ? lo + per : op.steps;
  f32x16 acc = {}, low = {};
  f16x8 a[NS_AHEAD][2], b[NS_AHEAD][2];
#pragma unroll
  for (int q = 0; q < NS_AHEAD; ++q)
    if (lo + q < hi) {
      fetch2(P + (size_t)(lo + q) * BLOCK, a[q]);
      fetch2(Q + (size_t)(lo + q) * BLOCK, b[q]);
    }
  for (int st = lo; st < hi; st += NS_AHEAD) {
#pragma unroll
    for (int q = 0; q < NS_AHEAD; ++q)
      if (st + q < hi) {
        mfma3(a[q], b[q], acc, low);
        if (st + q + NS_AHEAD < hi) {
          fetch2(P + (size_t)(st + q + NS_AHEAD) * BLOCK, a[q]);
          fetch2(Q + (size_t)(st + q + NS_AHEAD) * BLOCK, b[q]);
        }
      }
  }
  acc_to_lds(acc, low, s[w], lane);
  __syncthreads();
  const int i0 = ti * TS, j0 = tj * TS, i = tid >> 3, j = (tid & 7) * 4;
  f32x4 v = *reinterpret_cast<const f32x4*>(&s[0][i * LDT + j]);
#pragma unroll
  for (int q = 1; q < NS_W; ++q) v += *reinterpret_cast<const f32x4*>(&s[q][i * LDT + j]);
  *reinterpret_cast<f32x4*>(&s[0][i * LDT + j]) = finish4<MODE>(p, mat, i0, j0, i, j, v);
  __syncthreads();
  put_tile<MODE, DT>(p, mat, i0, j0, s[0], tid, 64 * NS_W);
}

// Many tiles: each wave takes 64 x 64 values by itself, 12 matrix instructions
// for 8 KB of operands; the four waves of a workgroup form 128 x 128, so that
// every operand block is read by two of them and the second read meets it in
// the L1 cache.  Two-dimensional sizes are padded to 128.
constexpr int WIDE = 128;
constexpr int WIDE_AHEAD = 4;  // (steps are multiples of 8)

template <int MODE, int DT>
__global__ __launch_bounds__(256, 1) void ns_wide_kernel(NsArgs p, int tiles) {
  __shared__ float s[4][TS * LDT];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Tile tile = next_tile<MODE>(tiles, p.kp / WIDE);
  const size_t mat = tile.mat;
  // above the diagonal: wave 2 writes it (no barrier follows)
  if ((MODE == NS_GRAM || MODE == NS_POLY) && tile.ti == tile.tj && w == 1) return;
  const int ti = tile.ti * 4 + (w >> 1) * 2, tj = tile.tj * 4 + (w & 1) * 2;  // in tiles of 32
  const Operands<MODE> op(p, mat);
  const size_t row = (size_t)op.steps * BLOCK;
  const _Float16* P = op.P + ti * row + lane * 8;
  const _Float16* Q = op.Q + tj * row + lane * 8;
  f32x16 acc[2][2] = {}, low[2][2] = {};
  f16x8 a[WIDE_AHEAD][2][2], b[WIDE_AHEAD][2][2];
  auto fetch = [&](int q, int st) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      fetch2(P + h * row + (size_t)st * BLOCK, a[q][h]);
      fetch2(Q + h * row + (size_t)st * BLOCK, b[q][h]);
    }
  };
#pragma unroll
  for (int q = 0; q < WIDE_AHEAD; ++q) fetch(q, q);
  for (int st = 0; st < op.steps; st += WIDE_AHEAD) {
#pragma unroll
    for (int q = 0; q < WIDE_AHEAD; ++q) {
#pragma unroll
      for (int part = 0; part < 3; ++part)  // lo hi, hi lo, hi hi: no instruction waits for the one before
#pragma unroll
        for (int xy = 0; xy < 4; ++xy) {
          const int x = xy >> 1, y = xy & 1;
          f32x16& d = part < 2 ? low[x][y] : acc[x][y];
          d = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[q][x][part == 0], b[q][y][part == 1], d, 0, 0, 0);
        }
      if (st + WIDE_AHEAD < op.steps) fetch(q, st + WIDE_AHEAD + q);
    }
  }
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int i0 = (ti + x) * TS, j0 = (tj + y) * TS;
      if ((MODE == NS_GRAM || MODE == NS_POLY) && j0 > i0) continue;
      acc_to_lds(acc[x][y], low[x][y], s[w], lane);
      wave_lds_sync();
#pragma unroll
      for (int c = lane; c < TS * TS / 4; c += 64) {
        f32x4* v = reinterpret_cast<f32x4*>(&s[w][(c >> 3) * LDT + (c & 7) * 4]);
        *v = finish4<MODE>(p, mat, i0, j0, c >> 3, (c & 7) * 4, *v);
      }
      wave_lds_sync();
      put_tile<MODE, DT>(p, mat, i0, j0, s[w], lane, 64);
      wave_lds_sync();
    }
}

struct OrthoLayout {
  int m, k, mp, kp;
  bool wide;
  size_t off_x, off_t0, off_t1, off_xf, off_a, off_b, bytes;
};
size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
OrthoLayout ortho_layout(const OrthoArgs& p) {
  OrthoLayout L;
  L.m = p.rows < p.cols ? p.rows : p.cols;
  L.k = p.rows < p.cols ? p.cols : p.rows;
  L.wide = (int64_t)p.n * ((L.m + WIDE - 1) / WIDE) * ((L.k + WIDE - 1) / WIDE) >= 128;
  const int pad = L.wide ? WIDE : TS;
  L.mp = round_up(L.m, pad);
  L.kp = round_up(L.k, pad);
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

template <int MODE, int DT>
void run_product(const OrthoArgs& o, const OrthoLayout& L, const NsArgs& p, hipStream_t s) {
  const int t = L.wide ? WIDE : TS, mt = L.mp / t;
  const int tiles = MODE == NS_GRAM || MODE == NS_POLY ? mt * (mt + 1) / 2 : mt * (L.kp / t);
  if (L.wide) ns_wide_kernel<MODE, DT><<<tiles * o.n, 256, 0, s>>>(p, tiles);
  else ns_tile_kernel<MODE, DT><<<tiles * o.n, 64 * NS_W, 0, s>>>(p, tiles);
}

template <int DT>
void run_ortho(const OrthoArgs& o, const OrthoLayout& L, NsArgs p, hipStream_t s) {
  const int64_t len = (int64_t)o.rows * o.cols;
  const int nb = (int)((len + 4095) / 4096 < NORM_B ? (len + 4095) / 4096 : NORM_B);
  ns_norm_kernel<DT><<<dim3(nb, o.n), NORM_NT, 0, s>>>(p);
  ns_init_kernel<DT><<<dim3(L.kp / TS, L.mp / TS, o.n), INIT_NT, 0, s>>>(p, nb);
  for (int i = 0; i < o.steps; ++i) {
    run_product<NS_GRAM, DT>(o, L, p, s);
    run_product<NS_POLY, DT>(o, L, p, s);
    if (i + 1 < o.steps) run_product<NS_STEP, DT>(o, L, p, s);
    else run_product<NS_LAST, DT>(o, L, p, s);
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
