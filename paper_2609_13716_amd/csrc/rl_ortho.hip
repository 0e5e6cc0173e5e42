// Newton-Schulz orthogonalisation of a stack of matrices: X = G / |G|_F, then
// X <- a X + B X with A = X X^T, B = b A + c A A; X is [m, k] with m <= k
// (G transposed where it has more rows than columns).
//
// Arithmetic.  X is kept in float32 and a X is added in float32; every product
// runs on the float16 matrix instructions with both operands split, v = hi +
// lo / 2048 (hi the nearest float16, lo the float16 nearest to 2048 times the
// rest), as hi hi + (hi lo + lo hi) / 2048 accumulated in float32: operands
// keep 22 bits (from 2^-14 on; below, where float16's steps end, they are within
// 2^-36 of the value) and what is dropped is 2^-22 of a term, at three matrix
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
// contiguous, from memory or from LDS.  X is stored once by rows (for X X^T) and once
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
    l[e] = (_Float16)fmaf(-LO_SCALE, (float)h[e], LO_SCALE * v[e]);  // (exact before it is rounded)
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
struct Finish {
  f32x4 old;  // A's or X's values of the same places
  __device__ void load(const NsArgs& p, size_t mat, int i0, int j0, int i, int j) {
    if constexpr (MODE == NS_POLY) {
      const _Float16* a = p.a + mat * p.mp * p.mp * 2 + ((size_t)(i0 / 32) * (p.mp / 16) + (j0 + j) / 16) * BLOCK +
                          (i + 32 * (((j0 + j) & 15) / 8)) * 8 + (j & 7);
#pragma unroll
      for (int e = 0; e < 4; ++e) old[e] = (float)a[e] + (float)a[512 + e] * (1.f / LO_SCALE);
    }
    if constexpr (MODE == NS_STEP || MODE == NS_LAST)
      old = *reinterpret_cast<const f32x4*>(p.xf + mat * p.mp * p.kp + (size_t)(i0 + i) * p.kp + j0 + j);
  }
  __device__ f32x4 operator()(const NsArgs& p, size_t mat, int i0, int j0, int i, int j, f32x4 v) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (MODE == NS_POLY) v[e] = NS_C * v[e] + NS_B * old[e];
      if constexpr (MODE == NS_STEP || MODE == NS_LAST) v[e] = fmaf(NS_A, old[e], v[e]);
    }
    if constexpr (MODE == NS_STEP)
      *reinterpret_cast<f32x4*>(p.xf + mat * p.mp * p.kp + (size_t)(i0 + i) * p.kp + j0 + j) = v;
    return v;
  }
};

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
    // four values of a row of G at a time (r: the tile's row, or column, that runs down G); one store where rows keep
    // to its alignment
    const bool whole = p.cols % 4 == 0 && (reinterpret_cast<uintptr_t>(p.out) & (4 * sizeof(E) - 1)) == 0;
    const int r0 = flip ? j0 : i0, c0 = flip ? i0 : j0;
    for (int q = tid; q < TS * TS / 4; q += nt) {
      const int c = (q & 7) * 4, r = q >> 3;
      if (r0 + r >= p.rows || c0 + c >= p.cols) continue;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = flip ? res[(c + e) * LDT + r] : res[r * LDT + c + e];
      E* o = out + (size_t)(r0 + r) * p.cols + c0 + c;
      if (whole) {
        if constexpr (DT == DT_F32)
          *reinterpret_cast<f32x4*>(o) = f32x4{v[0], v[1], v[2], v[3]};
        else
          *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c0 + c + e < p.cols) o[e] = DType<DT>::from_f32(v[e]);
      }
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
// and add their partial tiles through LDS; 8 waves where that leaves a CU no
// more than two workgroups (1 x 512x658 99 us, with 4 waves 104), else 4.
constexpr int NS_AHEAD = 4;  // steps whose operands are loaded ahead

template <int MODE, int DT, int NS_W>
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
  const int i0 = ti * TS, j0 = tj * TS, i = tid >> 3, j = (tid & 7) * 4;
  const bool ends = w < 4;  // 256 threads finish 4 values each
  Finish<MODE> fin;
  if (ends) fin.load(p, mat, i0, j0, i, j);  // (early: it arrives while the products run)
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
  if (ends) {
    f32x4 v = *reinterpret_cast<const f32x4*>(&s[0][i * LDT + j]);
#pragma unroll
    for (int q = 1; q < NS_W; ++q) v += *reinterpret_cast<const f32x4*>(&s[q][i * LDT + j]);
    *reinterpret_cast<f32x4*>(&s[0][i * LDT + j]) = fin(p, mat, i0, j0, i, j, v);
  }
  __syncthreads();
  put_tile<MODE, DT>(p, mat, i0, j0, s[0], tid, 64 * NS_W);
}

// More tiles: 64 x 64 values per workgroup, again with the sum shared out over
// its waves (12 matrix instructions a step for 8 KB of operands), two
// workgroups per CU, one of which works while the other starts or ends.
constexpr int MID = 64;
constexpr int MID_AHEAD = 3;

template <int MODE, int DT>
__global__ __launch_bounds__(256, 2) void ns_mid_kernel(NsArgs p, int tiles) {
  __shared__ float s[4][4][TS * LDT];  // [wave][32 x 32 tile]
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Tile tile = next_tile<MODE>(tiles, p.kp / MID);
  const size_t mat = tile.mat;
  const Operands<MODE> op(p, mat);
  const size_t row = (size_t)op.steps * BLOCK;
  const _Float16* P = op.P + (size_t)tile.ti * 2 * row + lane * 8;
  const _Float16* Q = op.Q + (size_t)tile.tj * 2 * row + lane * 8;
  const int per = (op.steps + 3) / 4, lo = w * per, hi = lo + per < op.steps ? lo + per : op.steps;
  f32x16 acc[2][2] = {}, low[2][2] = {};
  f16x8 a[MID_AHEAD][2][2], b[MID_AHEAD][2][2];
  auto fetch = [&](int q, int st) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      fetch2(P + h * row + (size_t)st * BLOCK, a[q][h]);
      fetch2(Q + h * row + (size_t)st * BLOCK, b[q][h]);
    }
  };
  auto product = [&](int q) {
#pragma unroll
    for (int part = 0; part < 3; ++part)  // lo hi, hi lo, hi hi: no instruction waits for the one before
#pragma unroll
      for (int xy = 0; xy < 4; ++xy) {
        const int x = xy >> 1, y = xy & 1;
        f32x16& d = part < 2 ? low[x][y] : acc[x][y];
        d = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[q][x][part == 0], b[q][y][part == 1], d, 0, 0, 0);
      }
  };
  // (past its last step a wave loads the last one again: no branch around loads in flight)
  const int end = hi - 1;
#pragma unroll
  for (int q = 0; q < MID_AHEAD; ++q) fetch(q, lo + q < end ? lo + q : end);
  int st = lo;
  for (; st + MID_AHEAD <= hi; st += MID_AHEAD) {
#pragma unroll
    for (int q = 0; q < MID_AHEAD; ++q) {
      product(q);
      fetch(q, st + MID_AHEAD + q < end ? st + MID_AHEAD + q : end);
    }
  }
  if (st < hi) product(0);
  if (st + 1 < hi) product(1);
  const int x = w >> 1, y = w & 1, i0 = tile.ti * MID + x * TS, j0 = tile.tj * MID + y * TS;
  Finish<MODE> fin[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) fin[u].load(p, mat, i0, j0, (lane + u * 64) >> 3, (lane & 7) * 4);
#pragma unroll
  for (int xy = 0; xy < 4; ++xy) acc_to_lds(acc[xy >> 1][xy & 1], low[xy >> 1][xy & 1], s[w][xy], lane);
  __syncthreads();
  if ((MODE == NS_GRAM || MODE == NS_POLY) && j0 > i0) return;  // (no barrier follows)
  // each wave adds up and finishes one of the four
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int i = (lane + u * 64) >> 3, j = (lane & 7) * 4;
    f32x4 v = *reinterpret_cast<const f32x4*>(&s[0][w][i * LDT + j]);
#pragma unroll
    for (int q = 1; q < 4; ++q) v += *reinterpret_cast<const f32x4*>(&s[q][w][i * LDT + j]);
    *reinterpret_cast<f32x4*>(&s[0][w][i * LDT + j]) = fin[u](p, mat, i0, j0, i, j, v);
  }
  wave_lds_sync();
  put_tile<MODE, DT>(p, mat, i0, j0, s[0][w], lane, 64);
}

// Many tiles: a workgroup takes 128 x 128 values, each of its four waves
// 64 x 64 of them.  Both operands go through LDS, where two waves read each
// block; WIDE_STEPS steps are read while the next ones are written, whose
// loads were issued WIDE_STEPS steps before.  What bounds it: a step takes 540
// cycles, 384 of them matrix instructions, and on a full chip (4 x 1024x1024)
// the clock falls from 2.3 to 1.6 GHz; start and end of a workgroup are 15000
// of 50000 cycles there.  (Straight from the L1 cache a step takes 590 cycles:
// 4 x 1024x1024 470 us instead of 460, 1 x 4096x4096 5060 instead of 4710.)
constexpr int WIDE = 128;
constexpr int WIDE_STEPS = 4;            // steps between barriers (sums have a multiple of 8)
constexpr int WIDE_STEP = 16 * 512;      // values of a step: 4 row tiles of P, then of Q, hi and lo

template <int MODE, int DT>
__global__ __launch_bounds__(256, 1) void ns_wide_kernel(NsArgs p, int tiles) {
  __shared__ _Float16 s_op[2][WIDE_STEPS][WIDE_STEP];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Tile tile = next_tile<MODE>(tiles, p.kp / WIDE);
  const size_t mat = tile.mat;
  const int ti = tile.ti * 4 + (w >> 1) * 2, tj = tile.tj * 4 + (w & 1) * 2;  // in tiles of 32
  // above the diagonal: wave 2 writes it
  const bool idle = (MODE == NS_GRAM || MODE == NS_POLY) && tile.ti == tile.tj && w == 1;
  const Operands<MODE> op(p, mat);
  const size_t row = (size_t)op.steps * BLOCK;
  // this wave stages the hi or lo half of every second row tile
  const _Float16* P = op.P + (size_t)(tile.ti * 4 + (w >> 1)) * row + (w & 1) * 512 + lane * 8;
  const _Float16* Q = op.Q + (size_t)(tile.tj * 4 + (w >> 1)) * row + (w & 1) * 512 + lane * 8;
  f16x8 in[WIDE_STEPS * 4];  // loads in flight: piece 4 q + i is block 4 i + w of step q
  auto fetch = [&](int piece, int st) {
    const int i = piece & 3;
    const _Float16* src = (i < 2 ? P : Q) + (i & 1) * 2 * row;
    in[piece] = *reinterpret_cast<const f16x8*>(src + (size_t)(st + piece / 4) * BLOCK);
  };
  auto put = [&](int buf, int piece) {
    *reinterpret_cast<f16x8*>(&s_op[buf][piece / 4][((piece & 3) * 4 + w) * 512 + lane * 8]) = in[piece];
  };
  f32x16 acc[2][2] = {}, low[2][2] = {};
  f16x8 o[2][8];  // operands of a step and of the next: P's two row tiles, then Q's, hi and lo
  const int p0 = (w >> 1) * 4 * 512 + lane * 8, q0 = (8 + (w & 1) * 4) * 512 + lane * 8;
  auto take = [&](int set, int buf, int q, int i) {
    o[set][i] = *reinterpret_cast<const f16x8*>(&s_op[buf][q][(i < 4 ? p0 : q0) + (i & 3) * 512]);
  };
  auto product = [&](int set, int n) {  // lo hi, hi lo, hi hi: no instruction waits for the one before
    const int part = n / 4, x = n >> 1 & 1, y = n & 1;
    f32x16& d = part < 2 ? low[x][y] : acc[x][y];
    d = __builtin_amdgcn_mfma_f32_32x32x16_f16(o[set][x * 2 + (part == 0)], o[set][4 + y * 2 + (part == 1)], d, 0, 0, 0);
  };
  constexpr int PIECES = WIDE_STEPS * 4;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) fetch(i, 0);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    put(0, i);
    fetch(i, WIDE_STEPS);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) take(0, 0, 0, i);
  for (int st = 0; st < op.steps; st += 2 * WIDE_STEPS) {
#pragma unroll
    for (int buf = 0; buf < 2; ++buf) {
      // (past the last step the first ones are loaded and written again: a branch here would make every write
      // wait for all loads in flight)
      const int at = st + buf * WIDE_STEPS, ahead = at + 2 * WIDE_STEPS < op.steps ? at + 2 * WIDE_STEPS : 0;
      int done = 0;  // pieces written
#pragma unroll
      for (int q = 0; q < WIDE_STEPS; ++q) {
        // One memory instruction after each matrix instruction, in this order: several in a row take longer to
        // issue than the matrix instruction before them runs.  The other buffer is whole a step before it is read.
        const bool last = q + 1 == WIDE_STEPS;
        const int upto = last ? PIECES : (PIECES * (q + 1) + WIDE_STEPS - 2) / (WIDE_STEPS - 1);
#pragma unroll
        for (int n = 0; n < 12; ++n) {
          product(q & 1, n);
          __builtin_amdgcn_sched_barrier(0);
          if (n < 8) {
            take((q + 1) & 1, last ? buf ^ 1 : buf, last ? 0 : q + 1, n);
            if (done < upto) put(buf ^ 1, done++);
          } else {
            fetch(q * 4 + n - 8, ahead);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (q + 2 == WIDE_STEPS) __syncthreads();
      }
    }
  }
  __syncthreads();  // (the results go where the operands lie)
  if (idle) return;  // (no barrier follows)
  float* s = reinterpret_cast<float*>(s_op) + w * TS * LDT;
  Finish<MODE> fin[4][4];
#pragma unroll
  for (int xy = 0; xy < 4; ++xy)  // (all at once: one wait; tiles above the diagonal are read and dropped)
#pragma unroll
    for (int u = 0; u < 4; ++u)
      fin[xy][u].load(p, mat, (ti + (xy >> 1)) * TS, (tj + (xy & 1)) * TS, (lane + u * 64) >> 3, (lane & 7) * 4);
#pragma unroll
  for (int xy = 0; xy < 4; ++xy) {
    const int i0 = (ti + (xy >> 1)) * TS, j0 = (tj + (xy & 1)) * TS;
    if ((MODE == NS_GRAM || MODE == NS_POLY) && j0 > i0) continue;
    acc_to_lds(acc[xy >> 1][xy & 1], low[xy >> 1][xy & 1], s, lane);
    wave_lds_sync();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = (lane + u * 64) >> 3, j = (lane & 7) * 4;
      f32x4* v = reinterpret_cast<f32x4*>(&s[i * LDT + j]);
      *v = fin[xy][u](p, mat, i0, j0, i, j, *v);
    }
    wave_lds_sync();
    put_tile<MODE, DT>(p, mat, i0, j0, s, lane, 64);
    wave_lds_sync();
  }
}

// ---- one workgroup per matrix ----
//
// Matrices whose X fits in one CU (policy layers): all steps in one launch.
// X lives in registers, in the layout that the 16 x 16 x 32 matrix instruction
// writes: a wave owns NS strips of 16 columns, all rows (lane l: column l % 16,
// rows 16 it + 4 (l / 16) ..+3).  That is also the layout in which it reads X
// for B X, when the sum over rows takes them in the order (tile 2s: 4 rows of
// the lane's group, tile 2s + 1: 4 rows) -- so X needs LDS only for X X^T, and
// A and B are laid out in LDS with the same order of columns ("fragments":
// 16 rows x 32 columns, 64 lanes x 8 values, hi then lo).  Blocks of 32 x 32 of
// A on and below the diagonal belong to one wave each; where there are more
// waves than blocks, groups of waves share out the columns of X X^T.
// LDS reads bind it: a step reads 8 KB for each block and 32 columns of X, and
// all of B for each strip.

constexpr int FRAG = 2 * 512;  // values of a fragment
constexpr int SMALL_W = 16;    // waves, at most

struct SmallPlan {
  int MT, NS;     // row tiles of 16 (even), strips of a wave
  int W, NB, KS;  // waves, blocks, groups of waves for X X^T
  int kp;         // columns, padded to 32
  size_t lds;
};

// Four halves of a lane (rows r = 0..3 of its column) -> four columns of one
// row: lanes 4q + t exchange so that lane t holds row t, columns 4q ..+3.
__device__ __forceinline__ uint2 quad_turn(uint2 d, int t) {
  const uint32_t sel = t & 1 ? 0x03020706u : 0x05040100u;
  const uint32_t e0 = __builtin_amdgcn_mov_dpp((int)d.x, 0xB1, 0xF, 0xF, true);  // lane t ^ 1
  const uint32_t e1 = __builtin_amdgcn_mov_dpp((int)d.y, 0xB1, 0xF, 0xF, true);
  const uint32_t n0 = __builtin_amdgcn_perm(e0, d.x, sel), n1 = __builtin_amdgcn_perm(e1, d.y, sel);
  const bool low = t < 2;
  const uint32_t x = low ? n0 : n1, y = low ? n1 : n0;
  const uint32_t z = __builtin_amdgcn_mov_dpp((int)y, 0x4E, 0xF, 0xF, true);  // lane t ^ 2
  return low ? make_uint2(x, z) : make_uint2(z, x);
}

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
// Four values split: [hi, lo], two dwords each.
struct Split4 {
  uint2 part[2];
};
__device__ __forceinline__ Split4 split4(f32x4 v) {
  uint32_t h[2], l[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const f32x2 x = {v[2 * e], v[2 * e + 1]};
    const f16x2 hi = __builtin_convertvector(x, f16x2);
    const f32x2 rest = {fmaf(-LO_SCALE, (float)hi[0], LO_SCALE * x[0]), fmaf(-LO_SCALE, (float)hi[1], LO_SCALE * x[1])};
    h[e] = __builtin_bit_cast(uint32_t, hi);
    l[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, f16x2));
  }
  return {make_uint2(h[0], h[1]), make_uint2(l[0], l[1])};
}

// A lane's four values (rows of tile ti, a column of tile tj) -> fragments of
// the matrix itself (rows ti, columns tj; steps of 32 columns) ..
__device__ __forceinline__ void put_frag(_Float16* f, int ti, int tj, int steps, const Split4& v, int lane) {
  const int t = lane & 3, c4 = (lane & 15) >> 2, g = lane >> 4;
#pragma unroll
  for (int part = 0; part < 2; ++part)
    *reinterpret_cast<uint2*>(f + ((ti * steps + tj / 2) * 2 + part) * 512 + ((4 * g + t) + 16 * c4) * 8 + 4 * (tj & 1)) =
        quad_turn(v.part[part], t);
}
// .. and of its transpose (rows tj, columns ti), where the lane's own values
// lie side by side.
__device__ __forceinline__ void put_frag_t(_Float16* f, int ti, int tj, int steps, const Split4& v, int lane) {
#pragma unroll
  for (int part = 0; part < 2; ++part)
    *reinterpret_cast<uint2*>(f + ((tj * steps + ti / 2) * 2 + part) * 512 + lane * 8 + 4 * (ti & 1)) = v.part[part];
}

__device__ __forceinline__ void load_frag(const _Float16* f, int tile, int step, int steps, int lane, f16x8 (&d)[2]) {
  const _Float16* q = f + (tile * steps + step) * FRAG + lane * 8;
  d[0] = *reinterpret_cast<const f16x8*>(q);
  d[1] = *reinterpret_cast<const f16x8*>(q + 512);
}

__device__ __forceinline__ void mfma3_16(const f16x8 (&a)[2], const f16x8 (&b)[2], f32x4& acc, f32x4& low) {
  low = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[0], b[1], low, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[0], b[0], acc, 0, 0, 0);
  low = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[1], b[0], low, 0, 0, 0);
}

// The 32 x 32 block (bi, bj) of F F^T over the steps [lo, hi).
__device__ __forceinline__ void block_product(const _Float16* f, int bi, int bj, int lo, int hi, int steps, int lane,
                                              f32x4 (&out)[2][2]) {
  f32x4 acc[2][2] = {}, low[2][2] = {};
#pragma unroll 1  // (more steps in flight cost registers that the callers need)
  for (int s = lo; s < hi; ++s) {
    f16x8 a[2][2], b[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) load_frag(f, bi * 2 + h, s, steps, lane, a[h]);
    if (bi != bj) {
#pragma unroll
      for (int h = 0; h < 2; ++h) load_frag(f, bj * 2 + h, s, steps, lane, b[h]);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int part = 0; part < 2; ++part) b[h][part] = a[h][part];
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) mfma3_16(a[x], b[y], acc[x][y], low[x][y]);
  }
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int y = 0; y < 2; ++y) out[x][y] = acc[x][y] + low[x][y] * (1.f / LO_SCALE);
}

template <int DT, int MT, int NS, int NT>
__global__ __launch_bounds__(NT) void ns_small_kernel(const void* gp, void* outp, int rows, int cols, int n_steps,
                                                        SmallPlan pl) {
  extern __shared__ char s_raw[];
  __shared__ double s_norm[SMALL_W];
  using E = typename DType<DT>::T;
  constexpr int MS = MT / 2;            // steps of 32 over the rows
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g4 = lane >> 4;
  const bool flip = rows > cols;
  const int m = flip ? cols : rows, k = flip ? rows : cols, strips = pl.kp / 16, ksteps = pl.kp / 32;
  const E* g = static_cast<const E*>(gp) + (size_t)blockIdx.x * rows * cols;
  E* out = static_cast<E*>(outp) + (size_t)blockIdx.x * rows * cols;
  _Float16* fx = reinterpret_cast<_Float16*>(s_raw);           // X's fragments, and (when they are read) ..
  _Float16* fa = fx;                                           // .. A's, ..
  _Float16* fb = fx + MT * MS * FRAG;                          // .. B's, ..
  float* part = reinterpret_cast<float*>(fb);                  // .. or partial blocks of A before B is there

  // a lane's place in G: element (i, j) of X
  auto at = [&](int i, int j) { return (uint32_t)(flip ? j * cols + i : i * cols + j); };
  f32x4 x[NS][MT];
  double sum = 0.;
#pragma unroll
  for (int ns = 0; ns < NS; ++ns)
#pragma unroll
    for (int it = 0; it < MT; ++it)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = it * 16 + 4 * g4 + r, j = (w * NS + ns) * 16 + c;
        x[ns][it][r] = i < m && j < k ? DType<DT>::to_f32(g[at(i, j)]) : 0.f;
      }
#pragma unroll
  for (int ns = 0; ns < NS; ++ns)
#pragma unroll
    for (int it = 0; it < MT; ++it)
#pragma unroll
      for (int r = 0; r < 4; ++r) sum += (double)x[ns][it][r] * (double)x[ns][it][r];
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
  if (lane == 0) s_norm[w] = sum;
  __syncthreads();
  sum = s_norm[0];
  for (int q = 1; q < pl.W; ++q) sum += s_norm[q];
  const double inv = sum == 0. ? 0. : 1. / sqrt(sum);
#pragma unroll
  for (int ns = 0; ns < NS; ++ns)
#pragma unroll
    for (int it = 0; it < MT; ++it)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[ns][it][r] = (float)((double)x[ns][it][r] * inv);

  // this wave's block of the lower triangle, and (KS > 1) its part of the sum
  int bi, bj;
  lower_tile(w % pl.NB, bi, bj);
  const int group = w / pl.NB, per = (ksteps + pl.KS - 1) / pl.KS;  // (groups from KS on have nothing to do)
  const int lo = group < pl.KS ? group * per : ksteps, hi = lo + per < ksteps ? lo + per : ksteps;
  auto put_block = [&](_Float16* f, const f32x4 (&v)[2][2]) {
#pragma unroll
    for (int xy = 0; xy < 4; ++xy) {
      const int ti = bi * 2 + (xy >> 1), tj = bj * 2 + (xy & 1);
      const Split4 parts = split4(v[xy >> 1][xy & 1]);
      put_frag_t(f, ti, tj, MS, parts, lane);
      if (bi != bj) put_frag(f, ti, tj, MS, parts, lane);
    }
  };
  u32x4 xo[NS][MS][2];  // X as an operand: tiles 2s and 2s + 1 make a step
  auto operand = [&](int ns, int it, const Split4& parts) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      xo[ns][it / 2][q][it % 2 * 2] = parts.part[q].x;
      xo[ns][it / 2][q][it % 2 * 2 + 1] = parts.part[q].y;
    }
  };
  for (int step = 0; step < n_steps; ++step) {
#pragma unroll
    for (int ns = 0; ns < NS; ++ns)
      if (w * NS + ns < strips)
#pragma unroll
        for (int it = 0; it < MT; ++it) {
          const Split4 parts = split4(x[ns][it]);
          put_frag(fx, it, w * NS + ns, ksteps, parts, lane);
          operand(ns, it, parts);
        }
    __syncthreads();
    // A = X X^T
    f32x4 a[2][2];
    block_product(fx, bi, bj, lo, hi, ksteps, lane, a);
    __syncthreads();
    if (pl.KS > 1) {
      float* at = part + (group - 1) * pl.NB * 1024 + (w % pl.NB) * 1024 + lane * 4;
      if (group > 0 && group < pl.KS)
#pragma unroll
        for (int xy = 0; xy < 4; ++xy) *reinterpret_cast<f32x4*>(at + xy * 256) = a[xy >> 1][xy & 1];
      __syncthreads();
      if (group == 0)
        for (int h = 1; h < pl.KS; ++h)
#pragma unroll
          for (int xy = 0; xy < 4; ++xy)
            a[xy >> 1][xy & 1] += *reinterpret_cast<const f32x4*>(at + h * pl.NB * 1024 + xy * 256);
    }
    if (group == 0) put_block(fa, a);
    __syncthreads();
    // B = b A + c A A (over the partial blocks, which have been read)
    if (group == 0) {
      f32x4 v[2][2];
      block_product(fa, bi, bj, 0, MS, MS, lane, v);
#pragma unroll
      for (int xy = 0; xy < 4; ++xy) v[xy >> 1][xy & 1] = NS_C * v[xy >> 1][xy & 1] + NS_B * a[xy >> 1][xy & 1];
      put_block(fb, v);
    }
    __syncthreads();
    // X <- a X + B X, strip by strip
    if (w * NS < strips) {
#pragma unroll
      for (int it = 0; it < MT; ++it) {
        f32x4 acc[NS] = {}, low[NS] = {};
#pragma unroll
        for (int s = 0; s < MS; ++s) {
          f16x8 b[2];
          load_frag(fb, it, s, MS, lane, b);
#pragma unroll
          for (int ns = 0; ns < NS; ++ns) {
            const f16x8 v[2] = {__builtin_bit_cast(f16x8, xo[ns][s][0]), __builtin_bit_cast(f16x8, xo[ns][s][1])};
            mfma3_16(b, v, acc[ns], low[ns]);
          }
        }
#pragma unroll
        for (int ns = 0; ns < NS; ++ns) x[ns][it] = NS_A * x[ns][it] + (acc[ns] + low[ns] * (1.f / LO_SCALE));
        __builtin_amdgcn_sched_barrier(0);  // (B's tiles one at a time: what is read ahead holds registers)
      }
    }
    __syncthreads();
  }
  // (the lane's place is made anew: offsets and bounds kept from the loads above would hold registers all the way)
  int lane_again = lane;
  asm volatile("" : "+v"(lane_again));
  const int c_out = lane_again & 15, g_out = lane_again >> 4;
#pragma unroll
  for (int ns = 0; ns < NS; ++ns)
#pragma unroll
    for (int it = 0; it < MT; ++it)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = it * 16 + 4 * g_out + r, j = (w * NS + ns) * 16 + c_out;
        if (i < m && j < k) out[at(i, j)] = DType<DT>::from_f32(x[ns][it][r]);
      }
}

// Whether (and how) a matrix of this size runs in one workgroup.  As many
// waves as there are strips and blocks (up to 16): a wave's chain of LDS reads,
// products and exchanges is what takes the time (128 x 192, a step: 12 waves
// 21200, 6 waves of two strips 25400, 4 of three 32300 cycles).
bool small_plan(const OrthoArgs& o, SmallPlan* p) {
  const int m = o.rows < o.cols ? o.rows : o.cols, k = o.rows < o.cols ? o.cols : o.rows;
  if (m > 128) return false;
  const int MB = (m + 31) / 32;
  p->MT = 2 * MB;
  p->kp = round_up(k, 32);
  const int strips = p->kp / 16;
  p->NS = 1;
  while (p->NS * SMALL_W < strips) p->NS *= 2;
  if (p->NS * p->MT > 8) return false;  // X's registers
  p->NB = MB * (MB + 1) / 2;
  const int need = (strips + p->NS - 1) / p->NS;
  p->W = need > p->NB ? need : p->NB;
  if (p->W < 4) p->W = 4;
  if (MB > 2 && p->W > 12) return false;  // (128 registers a wave are too few there)
  p->KS = p->W / p->NB < p->kp / 32 ? p->W / p->NB : p->kp / 32;
  const size_t x = (size_t)p->MT * (p->kp / 32) * FRAG * 2, a = (size_t)p->MT * MB * FRAG * 2;
  const size_t b = a > (size_t)(p->KS - 1) * p->NB * 4096 ? a : (size_t)(p->KS - 1) * p->NB * 4096;
  p->lds = x > a + b ? x : a + b;
  return true;
}

template <int DT, int MT, int NS, int NT>
hipError_t run_small(const OrthoArgs& o, const SmallPlan& p, const void* g, void* out, hipStream_t s) {
  if (p.lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)ns_small_kernel<DT, MT, NS, NT>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.lds);
    if (e != hipSuccess) return e;
  }
  ns_small_kernel<DT, MT, NS, NT><<<o.n, 64 * p.W, p.lds, s>>>(g, out, o.rows, o.cols, o.steps, p);
  return hipGetLastError();
}
// The registers that so many waves leave to each.
template <int DT, int MT, int NS>
hipError_t pick_small(const OrthoArgs& o, const SmallPlan& p, const void* g, void* out, hipStream_t s) {
  if (p.W <= 8) return run_small<DT, MT, NS, 512>(o, p, g, out, s);
  if constexpr (MT <= 4)
    if (p.W > 12) return run_small<DT, MT, NS, 1024>(o, p, g, out, s);
  return run_small<DT, MT, NS, 768>(o, p, g, out, s);
}
template <int DT>
hipError_t launch_small(const OrthoArgs& o, const SmallPlan& p, const void* g, void* out, hipStream_t s) {
  switch (p.MT * 16 + p.NS) {
    case 2 * 16 + 1: return pick_small<DT, 2, 1>(o, p, g, out, s);
    case 2 * 16 + 2: return pick_small<DT, 2, 2>(o, p, g, out, s);
    case 2 * 16 + 4: return pick_small<DT, 2, 4>(o, p, g, out, s);
    case 4 * 16 + 1: return pick_small<DT, 4, 1>(o, p, g, out, s);
    case 4 * 16 + 2: return pick_small<DT, 4, 2>(o, p, g, out, s);
    case 6 * 16 + 1: return pick_small<DT, 6, 1>(o, p, g, out, s);
    default: return pick_small<DT, 8, 1>(o, p, g, out, s);
  }
}

// ---- many workgroups per matrix ----

struct OrthoLayout {
  int m, k, mp, kp;
  int tile;
  size_t off_x, off_t0, off_t1, off_xf, off_a, off_b, bytes;
};
size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
OrthoLayout ortho_layout(const OrthoArgs& p) {
  OrthoLayout L;
  L.m = p.rows < p.cols ? p.rows : p.cols;
  L.k = p.rows < p.cols ? p.cols : p.rows;
  // Larger tiles where there are enough of them (two workgroups of 64 x 64 to a CU, one of 128 x 128) and padding to
  // them adds little.  Measured (us; 32 / 64 / 128): 12 x 512x512 255 / 237 / 287, 4 x 1024x1024 560 / 473 / 460,
  // 1 x 4096x4096 - / 6460 / 4710, 64 x 130x140 (padded to 160, 192, 256) 112 / 165 / 240; with fewer tiles,
  // 2 x 700x900 157 / 199 / -.
  auto count = [&](int t) { return (int64_t)p.n * ((L.m + t - 1) / t) * ((L.k + t - 1) / t); };
  auto work = [&](int t) { return (double)round_up(L.m, t) * round_up(L.m, t) * (3. * round_up(L.k, t) + round_up(L.m, t)); };
  L.tile = TS;
  if (count(MID) >= 512 && work(MID) <= 1.15 * work(TS)) L.tile = MID;
  if (count(WIDE) >= 256 && work(WIDE) <= 1.15 * work(L.tile)) L.tile = WIDE;
  const int pad = L.tile;
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
  const int t = L.tile, mt = L.mp / t;
  const int tiles = MODE == NS_GRAM || MODE == NS_POLY ? mt * (mt + 1) / 2 : mt * (L.kp / t);
  if (t == MID) ns_mid_kernel<MODE, DT><<<tiles * o.n, 256, 0, s>>>(p, tiles);
  else if (t == WIDE) ns_wide_kernel<MODE, DT><<<tiles * o.n, 256, 0, s>>>(p, tiles);
  else if (tiles * o.n <= 512) ns_tile_kernel<MODE, DT, 8><<<tiles * o.n, 512, 0, s>>>(p, tiles);
  else ns_tile_kernel<MODE, DT, 4><<<tiles * o.n, 256, 0, s>>>(p, tiles);
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

size_t ortho_workspace_bytes(const OrthoArgs& p) {
  SmallPlan sp;
  return small_plan(p, &sp) ? 0 : ortho_layout(p).bytes;
}

hipError_t launch_ortho(const OrthoArgs& o, const void* g, void* out, void* workspace, hipStream_t s) {
  SmallPlan sp;
  if (small_plan(o, &sp))
    return o.dt == DT_F32 ? launch_small<DT_F32>(o, sp, g, out, s) : launch_small<DT_BF16>(o, sp, g, out, s);
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
