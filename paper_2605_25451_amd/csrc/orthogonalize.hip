// Orthogonalised updates: the quintic Newton-Schulz iteration
//   X0 = G / (|G|_F + eps),   A = X X^T,   B = b A + c A A,   X' = a X + B X
// on matrices of m rows and n >= m columns (a taller G is transposed on the way in and out).
//
// Three products a step, of m^2 n + m^3 + 2 m^2 n operations: A and B are symmetric, so only the tiles on
// and above the diagonal are computed, and stored twice.  Bound by the matrix cores where m is large, by launches where it is
// small.
//
// Numbers.  Operands are fp16, whose products the matrix cores add up in fp32.  bf16 would round eight times as coarsely:
// 1-6 % off after five steps, against 0.2 % of the one rounding that a bf16 result needs anyway.  What decides is X: a
// small singular value has few of X's bits, and five steps enlarge it 500 times.  So X is kept as hi + lo (22 bits)
// until the last two steps, where it enters the sum a X in full and the products as hi alone: 0.08-0.16 % off on noise and on spectra that
// fall over three decades (hi alone all the time: 0.14 and 0.4-0.7 %).  Few rows need more, see there.  For fp32 results all
// of X, A and B are hi + lo and every product is three, hi hi + hi lo + lo hi: 3e-7 to 3e-6 off, as in fp32 arithmetic.  Where one
// direction is 1000 times all others, both are off by more: 0.22 to 0.28 % and 5e-5 to 1e-4 (fp32 arithmetic 8e-5 to 3e-4).
// fp16's range: with powers of two s, t and u the buffers hold s X, t A and u B (see Scales).
#include "gemm_phases.h"
#include "train.h"

#include <algorithm>
#include <atomic>
#include <cmath>

namespace bm {

namespace {

typedef _Float16 half_t;
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

constexpr int PAD = 64;                        // rows and columns of the buffers are whole 64, the rest zeros

struct Split { half_t *hi, *lo; };             // lo may be null: hi alone

enum { GRAM = 0, POLY, STEP, LAST };

struct Product {
  Split A, B, C, old;                          // old: A of POLY, X of STEP and LAST
  int M, N, K, lda, ldb, ldc;                  // multiples of 64
  size_t stride_a, stride_b, stride_c;         // of the batch
  int terms;                                   // 1: hi hi;  3: and hi lo, lo hi
  float alpha, beta;                           // C = alpha * product + beta * old
  void* out; long ld_o, stride_o;              // LAST: [rows, cols] or, transposed, [cols, rows]
  int rows, cols, transposed, out_fp32;
};

__device__ inline half8 as_half(const bf16x8& v) { return __builtin_bit_cast(half8, v); }

// up to 8 values of a row of the result
__device__ inline void store_result(const Product& p, long at, int count, const float (&v)[8]) {
  if (p.out_fp32) {
    float* o = (float*)p.out + at;
    if (count == 8 && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
      *reinterpret_cast<f32x4*>(o) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4*>(o + 4) = f32x4{v[4], v[5], v[6], v[7]};
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < count) o[e] = v[e];
  } else {
    bf16_t* o = (bf16_t*)p.out + at;
    if (count == 8 && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
      store16(o, v);
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < count) o[e] = (bf16_t)v[e];
  }
}

// 8 values of a row as hi and lo
struct Halves { half8 hi, lo; };
__device__ inline void split8(const float (&v)[8], half8* hi, half8* lo) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    (*hi)[e] = (half_t)v[e];
    (*lo)[e] = (half_t)(v[e] - (float)(*hi)[e]);
  }
}

// ---- norm and conversion ----------------------------------------------------------------------

constexpr int NORM_PARTS = 1024;               // at most

// sums of squares of parts of every matrix, in fp64: squares of fp32 values neither overflow nor vanish there.  A row is `per_row`
// pieces of VEC elements.
template <int VEC>
__global__ __launch_bounds__(256) void norm_kernel(const float* __restrict__ g, long ld, long stride, uint32_t per_row, uint32_t pieces,
                                                   int parts, double* __restrict__ sums) {
  __shared__ double sm[4];
  const int b = blockIdx.x / parts, part = blockIdx.x % parts;
  const float* x = g + b * stride;
  double s = 0.0;
  const uint32_t step = parts * 256u;
#pragma unroll 4
  for (uint32_t i = part * 256u + threadIdx.x; i < pieces; i += step) {
    const uint32_t r = i / per_row, c = (i - r * per_row) * VEC;
    if constexpr (VEC == 4) {
      const float4 v = *reinterpret_cast<const float4*>(x + r * ld + c);
      s += (double)v.x * v.x + (double)v.y * v.y + (double)v.z * v.z + (double)v.w * v.w;
    } else {
      const double v = x[r * ld + c];
      s += v * v;
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, WAVE);
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) sums[blockIdx.x] = sm[0] + sm[1] + sm[2] + sm[3];
}

// The sum of a matrix's parts, in every thread: four wavefronts.
__device__ inline double sum_parts(const double* __restrict__ sums, int parts, double* sm) {
  double s = 0.0;
  for (int p = threadIdx.x; p < parts; p += 256) s += sums[p];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, WAVE);
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = s;
  __syncthreads();
  return sm[0] + sm[1] + sm[2] + sm[3];
}

// x[m, n] = s G / (|G| + eps), transposed where the rows of G are the columns of x.  A workgroup: `across` runs of 64 x 64 of x.
// VEC: rows of G start on 16 bytes
template <bool TRANSPOSED, bool VEC>
__global__ __launch_bounds__(256) void convert_kernel(const float* __restrict__ g, long ld, long stride, int M, int N,
                                                      const double* __restrict__ sums, int parts, float eps, float s, Split x,
                                                      int ldx, size_t stride_x, int tiles_n, int runs_n, int across, int runs) {
  __shared__ float tile[TRANSPOSED ? PAD : 1][PAD + 4];
  __shared__ double sm[4];
  const int b = blockIdx.x / runs, t = blockIdx.x % runs;
  const int r0 = t / runs_n * PAD, first = t % runs_n * across, last = min(tiles_n, first + across);
  const double scale = (double)s / (sqrt(sum_parts(sums + (size_t)b * parts, parts, sm)) + (double)eps);
  g += b * stride;
  x.hi += b * stride_x;
  if (x.lo) x.lo += b * stride_x;
  // four elements of a row of G
  auto fetch = [&](int r, int c, float (&v)[4]) {
    if (VEC && r < M && c + 4 <= N) {
      const float4 q = *reinterpret_cast<const float4*>(g + r * ld + c);
      v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = r < M && c + e < N ? g[r * ld + c + e] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)((double)v[e] * scale);
  };
  for (int ct = first; ct < last; ++ct) {
    const int c0 = ct * PAD;
    if (TRANSPOSED) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = threadIdx.x / 16 + i * 16, c = threadIdx.x % 16 * 4;   // of G: its rows are columns of x
        float v[4];
        fetch(c0 + r, r0 + c, v);
        *reinterpret_cast<float4*>(&tile[r][c]) = float4{v[0], v[1], v[2], v[3]};
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = threadIdx.x / 8 + i * 32, c = threadIdx.x % 8 * 8;       // of x
      float v[8];
      if (TRANSPOSED) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[c + e][r];
      } else {
        float lo[4], hi[4];
        fetch(r0 + r, c0 + c, lo);
        fetch(r0 + r, c0 + c + 4, hi);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = lo[e]; v[4 + e] = hi[e]; }
      }
      half8 h, l;
      split8(v, &h, &l);
      const size_t at = (size_t)(r0 + r) * ldx + c0 + c;
      *reinterpret_cast<half8*>(x.hi + at) = h;
      if (x.lo) *reinterpret_cast<half8*>(x.lo + at) = l;
    }
  }
}

// ---- products -----------------------------------------------------------------------------------

// the tile of the upper triangle of n x n tiles, row by row
__device__ inline void triangle_tile(int id, int n, int* tm, int* tn) {
  // rows before row r hold r n - r (r - 1) / 2 tiles
  int r = (int)((2 * n + 1 - sqrtf(fmaxf((float)(2 * n + 1) * (2 * n + 1) - 8.f * id, 0.f))) * 0.5f);
  r = max(0, min(r, n - 1));
  while (r > 0 && r * n - r * (r - 1) / 2 > id) --r;
  while ((r + 1) * n - (r + 1) * r / 2 <= id) ++r;
  *tm = r;
  *tn = r + id - (r * n - r * (r - 1) / 2);
}

// ---- epilogue of one wavefront: FM x FN blocks of 16 x 16, in strips of 16 rows.  The MFMAs run with swapped operands: of
// block (i, j) a lane holds row l % 16 and 4 columns from 4 (l / 16) on.  A strip goes through the wavefront's own LDS, so that
// rows are read and written 16 bytes per lane; a tile above the diagonal, or a result that is transposed, is read
// back by columns from there.  Sizes are whole 64, so a strip lies inside the matrix or outside.
//   row_of(i)  first row of strip i;  col0  first column;  mirror  the tile lies above the diagonal
//   stage      16 x (16 FN + 4) floats of LDS, free once `last` has returned
// `old` is requested two strips ahead, the first two strips before the tile's last MFMAs (`last`).
template <int KIND, int FM, int FN, typename RowOf, typename Last>
__device__ inline void finish(const Product& p, int b, f32x4 (&acc)[FM][FN], float* stage, int lane, int col0, bool mirror,
                              RowOf row_of, Last last) {
  constexpr int W = FN * 16, SLD = W + 4;
  constexpr int LPR = W / 8, RPI = 64 / LPR, TPS = 16 / RPI;            // lanes of a row, rows of an access, accesses of a strip
  constexpr int DOWN = 16 * W / 64;                                     // rows of a lane in a column
  const int m_in = lane & 15, q4 = (lane >> 4) * 4;
  const int rcol = (lane % LPR) * 8, rrow = lane / LPR;
  const int down_col = lane % W, down_row = lane / W * DOWN;
  const size_t at0 = b * p.stride_c;
  Halves pre[2][TPS];
  auto request = [&](auto i_t) {
    constexpr int i = decltype(i_t)::value;
    if (KIND == GRAM || i >= FM) return;
    if (row_of(i) >= p.M || col0 >= p.N) return;
#pragma unroll
    for (int t = 0; t < TPS; ++t) {
      const size_t at = at0 + (size_t)(row_of(i) + t * RPI + rrow) * p.ldc + col0 + rcol;
      pre[i & 1][t].hi = *reinterpret_cast<const half8*>(p.old.hi + at);
      if (p.old.lo) pre[i & 1][t].lo = *reinterpret_cast<const half8*>(p.old.lo + at);
      else pre[i & 1][t].lo = half8{};
    }
  };
  request(std::integral_constant<int, 0>{});
  request(std::integral_constant<int, 1>{});
  last();
  if (col0 >= p.N) return;
  const bool down = mirror || (KIND == LAST && p.transposed);
  const long out0 = b * p.stride_o;
  static_for<FM>([&](auto i_t) {
    constexpr int i = decltype(i_t)::value;
    if (row_of(i) >= p.M) return;
#pragma unroll
    for (int j = 0; j < FN; ++j) *reinterpret_cast<f32x4*>(stage + m_in * SLD + j * 16 + q4) = acc[i][j];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int t = 0; t < TPS; ++t) {
      const int row = t * RPI + rrow, r = row_of(i) + row, c = col0 + rcol;
      float* piece = stage + row * SLD + rcol;
      const f32x4 x0 = *reinterpret_cast<const f32x4*>(piece), x1 = *reinterpret_cast<const f32x4*>(piece + 4);
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = p.alpha * (e < 4 ? x0[e] : x1[e - 4]);
        if (KIND != GRAM) v[e] += p.beta * ((float)pre[i & 1][t].hi[e] + (float)pre[i & 1][t].lo[e]);
      }
      if (down) {
        *reinterpret_cast<f32x4*>(piece) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4*>(piece + 4) = f32x4{v[4], v[5], v[6], v[7]};
      }
      if constexpr (KIND == LAST) {
        if (!p.transposed && r < p.rows) store_result(p, out0 + r * p.ld_o + c, min(8, p.cols - c), v);
      } else {
        half8 hi, lo;
        split8(v, &hi, &lo);
        const size_t at = at0 + (size_t)r * p.ldc + c;
        *reinterpret_cast<half8*>(p.C.hi + at) = hi;
        if (p.C.lo) *reinterpret_cast<half8*>(p.C.lo + at) = lo;
      }
    }
    if (down) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const int r = col0 + down_col, c0 = row_of(i) + down_row;           // of the transposed matrix
#pragma unroll
      for (int q = 0; q < DOWN; q += 8) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = stage[(down_row + q + e) * SLD + down_col];
        if constexpr (KIND == LAST) {
          if (r < p.cols) store_result(p, out0 + r * p.ld_o + c0 + q, min(8, p.rows - c0 - q), v);
        } else {
          half8 hi, lo;
          split8(v, &hi, &lo);
          const size_t at = at0 + (size_t)r * p.ldc + c0 + q;
          *reinterpret_cast<half8*>(p.C.hi + at) = hi;
          if (p.C.lo) *reinterpret_cast<half8*>(p.C.lo + at) = lo;
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    request(std::integral_constant<int, i + 2>{});
  });
}

// Where a workgroup's tile lies.  Workgroups of one XCD have neighbouring tiles.
struct Place { int b, tm, tn; };
template <bool SYMMETRIC>
__device__ inline Place place(int tiles_m, int tiles_n, int tiles) {
  const int id = xcd_run(blockIdx.x, gridDim.x), t = id % tiles;
  Place q;
  q.b = id / tiles;
  if (SYMMETRIC) triangle_tile(t, tiles_n, &q.tm, &q.tn);
  else grouped_tile<4>(t, tiles_m, tiles_n, &q.tm, &q.tn);
  q.tm = __builtin_amdgcn_readfirstlane(q.tm);              // (the root is taken in vector registers)
  q.tn = __builtin_amdgcn_readfirstlane(q.tn);
  return q;
}

// A slice's operands: terms of K / 64 slices each, hi hi, hi lo, lo hi.
template <bool B_TR>
struct Operands {
  const bf16_t *a[2], *b[2];
  int slices;                                  // of a term
  size_t b_step;
  __device__ inline Operands(const Product& p, const Place& q, int m0, int n0) {
    const size_t ao = q.b * p.stride_a + (size_t)m0 * p.lda, bo = q.b * p.stride_b + (B_TR ? (size_t)n0 : (size_t)n0 * p.ldb);
    a[0] = reinterpret_cast<const bf16_t*>(p.A.hi + ao);
    b[0] = reinterpret_cast<const bf16_t*>(p.B.hi + bo);
    a[1] = p.terms > 1 ? reinterpret_cast<const bf16_t*>(p.A.lo + ao) : a[0];
    b[1] = p.terms > 1 ? reinterpret_cast<const bf16_t*>(p.B.lo + bo) : b[0];
    slices = p.K / BK;
    b_step = B_TR ? (size_t)BK * p.ldb : (size_t)BK;
  }
  __device__ inline const bf16_t* a_at(int j) const {
    const int t = (j >= slices) + (j >= 2 * slices);
    return (t == 2 ? a[1] : a[0]) + (size_t)(j - t * slices) * BK;
  }
  __device__ inline const bf16_t* b_at(int j) const {
    const int t = (j >= slices) + (j >= 2 * slices);
    return (t == 1 ? b[1] : b[0]) + (size_t)(j - t * slices) * b_step;
  }
};

// ---- TILE x TILE (64 or 128), GROUPS times four wavefronts of a quarter each: group g multiplies the slices g, g + GROUPS, ...
// of the contraction, and group 0 adds up their sums.  Each has DEPTH slices of LDS: DEPTH - 1 are on their way while one is
// multiplied, with one barrier a slice.  FULL: a slice holds hi and lo of both operands, for three products each (as slices of their own
// the products would fetch six operands instead of four).
constexpr int small_lds(int tile, int depth, int groups, bool full) { return groups * depth * 2 * tile * BK * 2 * (full ? 2 : 1); }

template <int KIND, int TILE, int DEPTH, int GROUPS, bool FULL>
__global__ __launch_bounds__(256 * GROUPS) void small_product_kernel(Product p, int tiles_m, int tiles_n, int tiles) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr bool NN = KIND == STEP || KIND == LAST;
  using RegA = Region<TILE, false, 4>;
  using RegB = Region<TILE, NN, 4>;
  constexpr int PARTS = FULL ? 2 : 1;                        // hi, lo
  constexpr uint32_t B0 = PARTS * RegA::BYTES, BUF = B0 + PARTS * RegB::BYTES;
  constexpr int LOADS = PARTS * (RegA::LOADS + RegB::LOADS), F = TILE / 32, HALF = TILE / 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) & 3);
  const int group = GROUPS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
  const int wm = wave >> 1, wn = wave & 1;
  const Place q = place<!NN>(tiles_m, tiles_n, tiles);
  const int m0 = q.tm * TILE, n0 = q.tn * TILE;
  const Operands<NN> op(p, q, m0, n0);
  const int n = (op.slices - group + GROUPS - 1) / GROUPS;
  RegA ra;
  RegB rb;
  ra.init(p.lda, 0, p.M - m0, wave, lane);
  rb.init(p.ldb, 0, p.N - n0, wave, lane);
  const uint32_t base = group * (DEPTH * BUF);
  auto load = [&](int j, uint32_t buf) {
    const size_t k = (size_t)(group + j * GROUPS);
#pragma unroll
    for (int h = 0; h < PARTS; ++h) {
      rb.template load<false>(op.b[h] + k * op.b_step, p.ldb, BK, base + buf + B0 + h * RegB::BYTES, wave, lane);
      ra.template load<false>(op.a[h] + k * BK, p.lda, BK, base + buf + h * RegA::BYTES, wave, lane);
    }
  };
  Fragments<TILE, false, F> fa;
  Fragments<TILE, NN, F> fb;
  fa.init(wm * HALF, lane);
  fb.init(wn * HALF, lane);
  f32x4 acc[F][F] = {};
#pragma unroll
  for (int s = 0; s < DEPTH - 1; ++s)
    if (s < n) load(s, s * BUF);
  uint32_t cur = 0, free = (DEPTH - 1) * BUF;
  for (int j = 0; j * GROUPS < op.slices; ++j) {
    // slice j has landed; later ones need not have
    const int later = n - 1 - j;
    if (later >= DEPTH - 2) wait_loads<(DEPTH - 2) * LOADS>();
    else if (DEPTH > 3 && later == 1) wait_loads<LOADS>();
    else wait_loads<0>();
    end_phase();                                             // for all; and all have read slice j - 1
    if (j >= n) break;                                       // (only in the last round)
    if (j + DEPTH - 1 < n) load(j + DEPTH - 1, free);
    bf16x8 a[PARTS][2][F], bb[PARTS][2][F];
#pragma unroll
    for (int h = 0; h < PARTS; ++h)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int f = 0; f < F; ++f) {
          bb[h][ks][f] = fb.read(smem, f, ks, base + cur + B0 + h * RegB::BYTES);
          a[h][ks][f] = fa.read(smem, f, ks, base + cur + h * RegA::BYTES);
        }
    auto multiply = [&](int ha, int hb) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
          for (int c = 0; c < F; ++c)
            acc[i][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_half(bb[hb][ks][c]), as_half(a[ha][ks][i]), acc[i][c], 0, 0, 0);
    };
    multiply(0, 0);
    if constexpr (FULL) {
      multiply(0, 1);
      multiply(1, 0);
    }
    wait_fragments();
    free = cur;
    cur = cur == (DEPTH - 1) * BUF ? 0 : cur + BUF;
  }
  end_phase();                                               // sums and strips overlay the slices
  constexpr int SUM = TILE * TILE;                           // floats of a group's sums
  float* sums = reinterpret_cast<float*>(smem);
  static_assert(((GROUPS - 1) * SUM + 4 * 16 * (F * 16 + 4)) * 4 <= small_lds(TILE, DEPTH, GROUPS, FULL), "sums and strips fit");
  if constexpr (GROUPS > 1) {
    auto at = [&](int g, int i, int c) {
      return reinterpret_cast<f32x4*>(sums + (g - 1) * SUM + (((wave * F + i) * F + c) * 64 + lane) * 4);
    };
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < F; ++i)
#pragma unroll
        for (int c = 0; c < F; ++c) *at(group, i, c) = acc[i][c];
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int g = 1; g < GROUPS; ++g)
#pragma unroll
      for (int i = 0; i < F; ++i)
#pragma unroll
        for (int c = 0; c < F; ++c) acc[i][c] += *at(g, i, c);
  }
  finish<KIND, F, F>(p, q.b, acc, sums + (GROUPS - 1) * SUM + wave * 16 * (F * 16 + 4), lane, n0 + wn * HALF, !NN && q.tm != q.tn,
                     [&](int i) { return m0 + wm * HALF + i * 16; }, [] {});
}

// ---- 256 x 256: two groups of four wavefronts that take turns between MFMAs and everything else, as in the bf16 kernels.
__device__ inline void mfma16_half(f32x4& acc, const bf16x8& a, const bf16x8& b) {
  asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}

template <int KIND>
__global__ __launch_bounds__(512, 2) void large_product_kernel(Product p, int tiles_m, int tiles_n, int tiles) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr bool NN = KIND == STEP || KIND == LAST;
  using RegA = Region<128, false>;
  using RegB = Region<256, NN>;
  constexpr uint32_t A1 = RegA::BYTES, B0 = 2 * RegA::BYTES, BUF = B0 + RegB::BYTES;
  constexpr int LATE = RegA::LOADS, EARLY = RegA::LOADS + RegB::LOADS;   // loads of a slice's two parts
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 2, wn = wave & 3;                                 // wm is the group
  const Place q = place<!NN>(tiles_m, tiles_n, tiles);
  const int m0 = q.tm * 256, n0 = q.tn * 256;
  const Operands<NN> op(p, q, m0, n0);
  const int n = op.slices * p.terms;
  RegA ra0, ra1;
  RegB rb;
  ra0.init(p.lda, 0, p.M - m0, wave, lane);
  ra1.init(p.lda, 128, p.M - m0, wave, lane);
  rb.init(p.ldb, 0, p.N - n0, wave, lane);
  auto load_early = [&](int j, uint32_t buf) {
    rb.template load<false>(op.b_at(j), p.ldb, BK, buf + B0, wave, lane);
    ra0.template load<false>(op.a_at(j), p.lda, BK, buf, wave, lane);
  };
  auto load_late = [&](int j, uint32_t buf) { ra1.template load<false>(op.a_at(j), p.lda, BK, buf + A1, wave, lane); };
  Fragments<128, false, 4> fa;
  Fragments<256, NN, 4> fb;
  fa.init(wm * 64, lane);
  fb.init(wn * 64, lane);
  bf16x8 af[2][4], bf[2][4];
  f32x4 acc[8][4];
  auto multiply = [&](auto half_t_) {
    constexpr int H = decltype(half_t_)::value * 4;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) mfma16_half(acc[H + i][j], bf[ks][j], af[ks][i]);
  };
  // COME: slices that follow this one (2: two or more, 0: this is the last)
  auto slice = [&](auto come_t, int j) {
    constexpr int COME = decltype(come_t)::value;
    const uint32_t buf = (j & 1) * BUF;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int f = 0; f < 4; ++f) bf[ks][f] = fb.read(smem, f, ks, buf + B0);
#pragma unroll
      for (int f = 0; f < 4; ++f) af[ks][f] = fa.read(smem, f, ks, buf);
    }
    if (COME >= 1) load_late(j + 1, buf ^ BUF);
    wait_fragments();
    // the second half of A of this slice is read next: everything older than the next slice's two parts must have landed
    wait_loads<COME >= 1 ? EARLY + LATE : 0>();
    end_phase();
    multiply(Int<0>{});
    wait_loads<COME >= 1 ? EARLY + LATE : 0>();
    end_phase();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int f = 0; f < 4; ++f) af[ks][f] = fa.read(smem, f, ks, buf + A1);
    if (COME >= 2) load_early(j + 2, buf);
    wait_fragments();
    if (COME == 0) { end_phase(); return; }                 // the last MFMAs belong to the epilogue
    wait_loads<COME >= 2 ? EARLY + LATE : LATE>();
    end_phase();
    multiply(Int<1>{});
    wait_loads<COME >= 2 ? EARLY + LATE : LATE>();
    end_phase();
  };
  load_early(0, 0);
  load_late(0, 0);
  if (n > 1) load_early(1, BUF);
  {
    bf16x8 z = {};
    asm volatile("s_nop 7" : "+v"(z));
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) mfma16_first(acc[i][j], z, z);
  }
  if (n > 1) wait_loads<EARLY + LATE>();
  else wait_loads<0>();
  end_phase();
  if (wm == 1) end_phase();                                 // group 1 stays one phase behind
  for (int j = 0; j < n - 2; ++j) slice(Int<2>{}, j);
  if (n > 1) slice(Int<1>{}, n - 2);
  slice(Int<0>{}, n - 1);
  finish<KIND, 8, 4>(p, q.b, acc, reinterpret_cast<float*>(smem) + wave * 16 * 68, lane, n0 + wn * 64, !NN && q.tm != q.tn,
                     [&](int i) { return m0 + (i >> 2) * 128 + wm * 64 + (i & 3) * 16; },
                     [&] {
                       multiply(Int<1>{});
                       if (wm == 0) end_phase();            // its strips overlay what group 1 has just read
                       settle(acc);
                     });
}

// ---- 192 x 192 and 96 x 96, of the symmetric products: twelve wavefronts of 48 x 64, or twice six of 48 x 32 that share the slices
// as above; three slices of LDS each, with one barrier a slice.
constexpr int MIDDLE_DEPTH = 3;
constexpr size_t middle_lds(int tile) { return (size_t)(tile == 96 ? 2 : 1) * MIDDLE_DEPTH * 2 * tile * BK * sizeof(half_t); }

template <int KIND, int TILE>
__global__ __launch_bounds__(768) void middle_product_kernel(Product p, int tiles_m, int tiles_n, int tiles) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  static_assert(KIND == GRAM || KIND == POLY, "operands whose k is contiguous");
  static_assert(TILE == 96 || TILE == 192, "48 rows a wavefront");
  constexpr int GROUPS = TILE == 96 ? 2 : 1, WAVES = 12 / GROUPS, WM = TILE / 48, FM = 3, FN = TILE / 48;
  using Reg = Region<TILE, false, WAVES>;
  constexpr uint32_t BUF = 2 * Reg::BYTES;
  constexpr int LOADS = 2 * Reg::LOADS;
  const int lane = threadIdx.x & 63, id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = GROUPS > 1 ? id / WAVES : 0, wave = id - group * WAVES, wm = wave % WM, wn = wave / WM;
  const Place q = place<true>(tiles_m, tiles_n, tiles);
  const int m0 = q.tm * TILE, n0 = q.tn * TILE;
  const Operands<false> op(p, q, m0, n0);
  const int all = op.slices * p.terms, n = (all - group + GROUPS - 1) / GROUPS;
  Reg ra, rb;
  ra.init(p.lda, 0, p.M - m0, wave, lane);
  rb.init(p.ldb, 0, p.N - n0, wave, lane);
  const uint32_t base = group * (MIDDLE_DEPTH * BUF);
  auto load = [&](int j, uint32_t buf) {
    rb.template load<false>(op.b_at(group + j * GROUPS), p.ldb, BK, base + buf + Reg::BYTES, wave, lane);
    ra.template load<false>(op.a_at(group + j * GROUPS), p.lda, BK, base + buf, wave, lane);
  };
  Fragments<TILE, false, FM> fa;
  Fragments<TILE, false, FN> fb;
  fa.init(wm * FM * 16, lane);
  fb.init(wn * FN * 16, lane);
  f32x4 acc[FM][FN] = {};
  if (n > 0) load(0, 0);
  if (n > 1) load(1, BUF);
  uint32_t cur = 0, free = 2 * BUF;
  for (int j = 0; j * GROUPS < all; ++j) {
    if (j + 1 < n) wait_loads<LOADS>();
    else wait_loads<0>();
    end_phase();                                             // slice j is there for all, and all have read slice j - 1
    if (j >= n) break;                                       // (only in the last round)
    if (j + 2 < n) load(j + 2, free);
    bf16x8 a[2][FM], b[2][FN];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int f = 0; f < FN; ++f) b[ks][f] = fb.read(smem, f, ks, base + cur + Reg::BYTES);
#pragma unroll
      for (int f = 0; f < FM; ++f) a[ks][f] = fa.read(smem, f, ks, base + cur);
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int c = 0; c < FN; ++c)
          acc[i][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_half(b[ks][c]), as_half(a[ks][i]), acc[i][c], 0, 0, 0);
    wait_fragments();
    free = cur;
    cur = cur == 2 * BUF ? 0 : cur + BUF;
  }
  end_phase();                                               // sums and strips overlay the slices
  constexpr int SUM = (GROUPS - 1) * TILE * TILE, STRIP = 16 * (FN * 16 + 4);
  float* sums = reinterpret_cast<float*>(smem);
  static_assert((SUM + WAVES * STRIP) * 4 <= middle_lds(TILE), "sums and strips fit");
  if constexpr (GROUPS > 1) {
    auto at = [&](int i, int c) { return reinterpret_cast<f32x4*>(sums + (((wave * FM + i) * FN + c) * 64 + lane) * 4); };
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int c = 0; c < FN; ++c) *at(i, c) = acc[i][c];
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int c = 0; c < FN; ++c) acc[i][c] += *at(i, c);
  }
  finish<KIND, FM, FN>(p, q.b, acc, sums + SUM + wave * STRIP, lane, n0 + wn * FN * 16, q.tm != q.tn,
                       [&](int i) { return m0 + (wm * FM + i) * 16; }, [] {});
}

// ---- few rows: 32, 64 or 128 of X at most ----------------------------------------------------------------
//
// A and B fit the LDS of a workgroup, so that a whole step is one launch: a workgroup holds a chunk of X's columns, has A from the sums
// of all chunks, computes B for itself, moves its chunk on and adds up the chunk's share of the next A.  Where X is one
// chunk (32 x 1024, 64 x 512, 128 x 128), all steps are one launch.  The tiled kernels would be three
// launches a step of one to a few workgroups: 192 x 64 59 us, here 23; 29 x 2350 93 and 47; 100 x 4096 127 and 96.
//
// Roundings average out less the fewer rows there are: with A and B of 11 bits a bf16 result would be 0.3 % off at 35 x 704 and
// 0.18 % at 64 x 192, beside 0.17 % of its own rounding.  So A and B are hi + lo here for all results: 0.08 and 0.1 % (22.7 us at 192 x 64
// instead of 20.4, 96 at 100 x 4096 instead of 88), and X, too, up to 32 rows (16 x 64: up to 0.18 % with a single product).
//
// LDS: X and then A or B in blocks of MP rows x 64 columns, 128 bytes a row, 16-byte chunk c of row r at c ^ ((r >> 1) & 7); hi, and lo
// behind it.  A chunk lies in the workspace as it does in LDS.
constexpr int TINY_THREADS = 1024, TINY_WAVES = TINY_THREADS / WAVE;
enum { SOLO = 0, FIRST, NEXT };                // all steps; conversion and the first sums; one step

struct Tiny {
  const float* g; long ld_g, stride_g;
  int M, N, tall;
  const double* norms; int parts;
  float eps, s, t, u;                          // Scales
  float a, b, c;
  int steps, step, full_from;                  // X entering step i has a lo part while i < full_from
  int blocks, chunks, summands;                // 64-column blocks of a chunk, chunks of a matrix, and how many sums there are of them
  unsigned char* image;                        // [batch, chunks] chunks
  float4 *sums, *sums_next;                    // [batch, chunks, blocks of A, 64]
  void* out; long ld_o, stride_o;
  int out_fp32;
};

// the most 64-column blocks of a chunk: of a matrix that is one, and of others.  A CU runs one workgroup of a step: 64 rows leave 4
// wavefronts a SIMD their registers (B's fragments take 64 of 112), 32 rows take 88 KiB of LDS.  Short chunks are faster while a matrix
// is fewer of them than there are CUs, long ones beyond; what is taken lies between.  bf16, us, with 128 / 256 / 512 over the rows:
//   64 x 1024 39, 46, 60    64 x 8192 69, 61, 70    64 x 131072 426, 267, 190    128 of 64 x 2048 385, 276, 229
//   32 x 2350 37, 46, 62    29 x 16384 51, 52, 65    32 x 81920 147, 97, 92    256 of 32 x 2048 205, 252, 216
constexpr int tiny_blocks(int mp, bool solo) { return mp == 128 ? 2 : solo ? 512 / mp : 256 / mp; }
// blocks of 16 x 16 on and above the diagonal of A
constexpr int tiny_gram_blocks(int mp) { return (mp / 16) * (mp / 16 + 1) / 2; }
constexpr size_t tiny_x_bytes(int mp, int blocks) { return (size_t)blocks * mp * 64 * 2 * 2; }
constexpr uint32_t tiny_ab_bytes(int mp) { return (mp + 63) / 64 * mp * 128; }
constexpr uint32_t tiny_norm_bytes(bool solo) { return solo ? 256 : 0; }
constexpr size_t tiny_lds(int mp, int blocks, bool solo) {
  return tiny_x_bytes(mp, blocks) + tiny_ab_bytes(mp) * 2 + tiny_norm_bytes(solo) + (mp == 32 ? 16 * 1024 : 0);
}

template <int MP, bool FULL, int MODE>
__global__ __launch_bounds__(TINY_THREADS) void tiny_kernel(Tiny t) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int MB = MP / 16, GB = tiny_gram_blocks(MP), PER_WAVE = (GB + TINY_WAVES - 1) / TINY_WAVES;
  constexpr int MAX_BLOCKS = tiny_blocks(MP, MODE == SOLO);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = blockIdx.x / t.chunks, chunk = blockIdx.x % t.chunks;
  const uint32_t x_half = t.blocks * (MP * 128), ab0 = 2 * x_half;
  constexpr uint32_t ab_half = tiny_ab_bytes(MP);
  double* sm = reinterpret_cast<double*>(smem + ab0 + ab_half * 2);
  const int m_in = lane & 15, q4 = (lane >> 4) * 4;
  auto at = [](int block, int row, int c) { return (uint32_t)((block * MP + row) * 128 + ((c ^ ((row >> 1) & 7)) << 4)); };
  // 16 rows x 32 k of an operand whose k is contiguous; k step ks of 32
  auto rows16 = [&](uint32_t base, int row0, int ks) {
    return *reinterpret_cast<const half8*>(smem + base + at(ks >> 1, row0 + m_in, (ks & 1) * 4 + (lane >> 4)));
  };
  // 16 columns x 32 k of X, whose k are the rows
  auto cols16 = [&](uint32_t base, int col0, int ks) {
    const int s = lane & 15, k = ks * 32 + (lane >> 4) * 8 + (s >> 2), c = (col0 & 63) / 8 + ((s & 3) >> 1);
    const unsigned char* p0 = smem + base + at(col0 >> 6, k, c) + (s & 1) * 8;
    const unsigned char* p1 = smem + base + at(col0 >> 6, k + 4, c) + (s & 1) * 8;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)p0);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)p1);
    union { struct { s16x4 a, b; } h; half8 v; } u;
    u.h.a = lo; u.h.b = hi;
    return u.v;
  };
  auto mfma = [](const half8& x, const half8& y, f32x4& acc) { acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, acc, 0, 0, 0); };
  // a lane's four neighbours of a row
  auto four = [&](uint32_t base, int row, int col) {
    return reinterpret_cast<half_t*>(smem + base + at(col >> 6, row, (col & 63) >> 3) + (col & 4) * 2);
  };
  typedef _Float16 half4 __attribute__((ext_vector_type(4)));
  // block i of this wavefront: its place among the GB, and its first row and column
  auto block_of = [&](int i, int* r, int* c) {
    const int id = wave + i * TINY_WAVES;
    int tm = 0, left = min(id, GB - 1);
    while (left >= MB - tm) { left -= MB - tm; ++tm; }
    *r = tm * 16;
    *c = (tm + left) * 16;
    return id;
  };
  // a block of the symmetric product of the rows at `base`, over k steps from .. to - 1; of both parts of their values or of hi alone
  auto gram_block = [&](auto parts_t, uint32_t base, uint32_t half, int r, int c, int from, int to) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    auto step = [&](int ks) {
      const half8 x = rows16(base, r, ks), y = rows16(base, c, ks);
      mfma(y, x, v);
      if constexpr (decltype(parts_t)::value > 1) {
        mfma(rows16(base + half, c, ks), x, v);
        mfma(y, rows16(base + half, r, ks), v);
      }
    };
    // (two a trip; the compiler unrolls no loop of MFMAs whose length it does not know)
    int ks = from;
    for (; ks + 2 <= to; ks += 2) { step(ks); step(ks + 1); }
    if (ks < to) step(ks);
    return v;
  };
  auto gram = [&](auto parts_t, uint32_t base, uint32_t half, int steps, f32x4 (&acc)[PER_WAVE]) {
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
      int r, c;
      acc[i] = block_of(i, &r, &c) < GB ? gram_block(parts_t, base, half, r, c, 0, steps) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  // that of X, whose columns are shared by as many wavefronts as there are for a block
  constexpr int X_PARTS = FULL ? 2 : 1, SHARE = TINY_WAVES / GB > 1 ? TINY_WAVES / GB : 1;
  auto gram_x = [&](f32x4 (&acc)[PER_WAVE]) {
    if constexpr (SHARE == 1) {
      gram(Int<X_PARTS>{}, 0, x_half, t.blocks * 2, acc);
    } else {
      static_assert(PER_WAVE == 1, "a block a wavefront");
      f32x4* shares = reinterpret_cast<f32x4*>(smem + ab0 + ab_half * 2 + tiny_norm_bytes(MODE == SOLO));
      const int part = wave / GB, block = wave % GB, per = (t.blocks * 2 + SHARE - 1) / SHARE;
      int r = 0, left = block;
      while (left >= MB - r) { left -= MB - r; ++r; }
      acc[0] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (part < SHARE) acc[0] = gram_block(Int<X_PARTS>{}, 0, x_half, r * 16, (r + left) * 16, part * per, min(t.blocks * 2, part * per + per));
      if (part > 0 && part < SHARE) shares[((part - 1) * GB + block) * WAVE + lane] = acc[0];
      __syncthreads();
      if (part == 0) {
#pragma unroll
        for (int p = 1; p < SHARE; ++p) acc[0] += shares[((p - 1) * GB + block) * WAVE + lane];
      }
    }
  };
  // a symmetric matrix into the place of A and B
  auto put_symmetric = [&](const f32x4 (&v)[PER_WAVE]) {
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
      int r, c;
      if (block_of(i, &r, &c) >= GB) continue;
      half4 hi, lo;
#pragma unroll
      for (int e = 0; e < 4; ++e) { hi[e] = (half_t)v[i][e]; lo[e] = (half_t)(v[i][e] - (float)hi[e]); }
      *reinterpret_cast<half4*>(four(ab0, r + m_in, c + q4)) = hi;
      *reinterpret_cast<half4*>(four(ab0 + ab_half, r + m_in, c + q4)) = lo;
      if (r == c) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = c + q4 + e, col = r + m_in;
        const uint32_t o = ab0 + at(col >> 6, row, (col & 63) >> 3) + (col & 7) * 2;
        *reinterpret_cast<half_t*>(smem + o) = hi[e];
        *reinterpret_cast<half_t*>(smem + o + ab_half) = lo[e];
      }
    }
  };

  // ---- X: converted from the gradient, or as the last step has left it
  // a thread's elements of a 64-column block in the gradient and the result, and their steps: neighbours have neighbours of a row
  constexpr int EACH = MP * 64 / TINY_THREADS;
  const int first_col = chunk * t.blocks * 64;
  auto element = [&](int k, int r, int c) { return at(k, r, c >> 3) + (c & 7) * 2; };
  auto each_element = [&](auto body) {
    if (t.tall) body(Int<1>{}, tid % MP, tid / MP);
    else body(Int<0>{}, tid / 64, tid % 64);
  };
  unsigned char* image = t.image + (size_t)blockIdx.x * tiny_x_bytes(MP, t.blocks);
  if (MODE == NEXT) {
    for (uint32_t o = tid * 16; o < 2 * x_half; o += TINY_THREADS * 16)
      *reinterpret_cast<u32x4*>(smem + o) = *reinterpret_cast<const u32x4*>(image + o);
  } else {
    each_element([&](auto tall_t, int r0, int c0) {
      constexpr bool TALL = decltype(tall_t)::value;
      constexpr int DR = TALL ? 0 : TINY_THREADS / 64, DC = TALL ? TINY_THREADS / MP : 0;
      const float* g = t.g + b * t.stride_g + (TALL ? (first_col + c0) * t.ld_g + r0 : r0 * t.ld_g + first_col + c0);
      const int m = TALL ? t.N : t.M, n = TALL ? t.M : t.N;
      float v[MAX_BLOCKS][EACH];
      double sum = 0.0;
#pragma unroll
      for (int k = 0; k < MAX_BLOCKS; ++k)
#pragma unroll
        for (int e = 0; e < EACH && k < t.blocks; ++e)
          v[k][e] = r0 + e * DR < m && first_col + k * 64 + c0 + e * DC < n ? g[TALL ? (k * 64 + e * DC) * t.ld_g : e * DR * t.ld_g + k * 64] : 0.f;
      if (MODE == SOLO) {
#pragma unroll
        for (int k = 0; k < MAX_BLOCKS; ++k)
#pragma unroll
          for (int e = 0; e < EACH && k < t.blocks; ++e) sum += (double)v[k][e] * v[k][e];
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, WAVE);
        if (lane == 0) sm[wave] = sum;
        __syncthreads();
        sum = 0.0;
        for (int w = 0; w < TINY_WAVES; ++w) sum += sm[w];
      } else {
        for (int p = lane; p < t.parts; p += WAVE) sum += t.norms[(size_t)b * t.parts + p];
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, WAVE);
      }
      const double scale = (double)t.s / (sqrt(sum) + (double)t.eps);
#pragma unroll
      for (int k = 0; k < MAX_BLOCKS; ++k)
#pragma unroll
        for (int e = 0; e < EACH && k < t.blocks; ++e) {
          // (what lies outside of the matrix stays 0 whatever the scale is)
          const float x = r0 + e * DR < m && first_col + k * 64 + c0 + e * DC < n ? (float)((double)v[k][e] * scale) : 0.f;
          const half_t hi = (half_t)x;
          const uint32_t o = element(k, r0 + e * DR, c0 + e * DC);
          *reinterpret_cast<half_t*>(smem + o) = hi;
          *reinterpret_cast<half_t*>(smem + x_half + o) = (half_t)(x - (float)hi);
        }
    });
  }
  __syncthreads();

  const size_t sums_of = (size_t)GB * WAVE;    // float4 of a chunk
  f32x4 acc[PER_WAVE];
  const int first = MODE == NEXT ? t.step : 0, last = MODE == SOLO ? t.steps : MODE == NEXT ? t.step + 1 : 0;
  for (int step = first; step < last; ++step) {
    // A
    if (MODE == SOLO) {
      gram_x(acc);
    } else {
#pragma unroll
      for (int i = 0; i < PER_WAVE; ++i) {
        acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int id = wave + i * TINY_WAVES;
        if (id >= GB) continue;
        const float4* from = t.sums + (size_t)b * t.chunks * sums_of + id * WAVE + lane;
#pragma unroll 8
        for (int k = 0; k < t.summands; ++k) {
          const float4 v = from[k * sums_of];
          acc[i][0] += v.x; acc[i][1] += v.y; acc[i][2] += v.z; acc[i][3] += v.w;
        }
      }
    }
    const float alpha = t.t / (t.s * t.s);
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) acc[i] *= alpha;
    put_symmetric(acc);
    __syncthreads();
    // B in its place
    f32x4 square[PER_WAVE];
    gram(Int<2>{}, ab0, ab_half, MP / 32, square);
    const float cs = t.c * (t.u / t.t) / t.t, bs = t.b * (t.u / t.t);
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) square[i] = cs * square[i] + bs * acc[i];
    __syncthreads();
    put_symmetric(square);
    __syncthreads();
    // X, 16 columns at a time; no other wavefront reads them
    const bool old_lo = step < t.full_from, new_lo = step + 1 < t.full_from, end = step + 1 == t.steps;
    const float as = end ? t.a / t.s : t.a, us = (end ? 1.f / t.s : 1.f) / t.u;
    // (B's fragments stay in registers where there is room)
    constexpr bool HELD = MP <= 64;
    half8 w_hi[HELD ? MP / 32 : 1][HELD ? MB : 1], w_lo[HELD ? MP / 32 : 1][HELD ? MB : 1];
    if constexpr (HELD) {
#pragma unroll
      for (int ks = 0; ks < MP / 32; ++ks)
#pragma unroll
        for (int i = 0; i < MB; ++i) {
          w_hi[ks][i] = rows16(ab0, i * 16, ks);
          w_lo[ks][i] = rows16(ab0 + ab_half, i * 16, ks);
        }
    }
    for (int strip = wave; strip < t.blocks * 4; strip += TINY_WAVES) {
      const int col0 = strip * 16;
      f32x4 y[MB] = {};
#pragma unroll
      for (int ks = 0; ks < MP / 32; ++ks) {
        const half8 x = cols16(0, col0, ks);
        half8 xl;
        if (FULL) xl = cols16(x_half, col0, ks);
#pragma unroll
        for (int i = 0; i < MB; ++i) {
          half8 w, wl;
          if constexpr (HELD) w = w_hi[ks][i]; else w = rows16(ab0, i * 16, ks);
          if constexpr (HELD) wl = w_lo[ks][i]; else wl = rows16(ab0 + ab_half, i * 16, ks);
          mfma(x, w, y[i]);
          mfma(x, wl, y[i]);
          if constexpr (FULL) mfma(xl, w, y[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const int r = i * 16 + m_in, c = col0 + q4;
        half4* hi_at = reinterpret_cast<half4*>(four(0, r, c));
        half4* lo_at = reinterpret_cast<half4*>(four(x_half, r, c));
        half4 hi = *hi_at, lo = {};
        if (old_lo) lo = *lo_at;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = as * ((float)hi[e] + (float)lo[e]) + us * y[i][e];
        if (!end) {
#pragma unroll
          for (int e = 0; e < 4; ++e) { hi[e] = (half_t)v[e]; lo[e] = (half_t)(v[e] - (float)hi[e]); }
          *hi_at = hi;
          if (new_lo) *lo_at = lo;
          continue;
        }
        // the result's bits in their place, to be stored by whole rows
        typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));
        u16x4 up, low;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t bits = __builtin_bit_cast(uint32_t, v[e]);
          up[e] = t.out_fp32 ? (unsigned short)(bits >> 16) : __builtin_bit_cast(unsigned short, (bf16_t)v[e]);
          low[e] = (unsigned short)bits;
        }
        *reinterpret_cast<u16x4*>(hi_at) = up;
        if (t.out_fp32) *reinterpret_cast<u16x4*>(lo_at) = low;
      }
    }
    __syncthreads();
  }
  if (MODE == SOLO || (MODE == NEXT && t.step + 1 == t.steps)) {
    each_element([&](auto tall_t, int r0, int c0) {
      constexpr bool TALL = decltype(tall_t)::value;
      constexpr int DR = TALL ? 0 : TINY_THREADS / 64, DC = TALL ? TINY_THREADS / MP : 0;
      const long to = b * t.stride_o + (TALL ? (first_col + c0) * t.ld_o + r0 : r0 * t.ld_o + first_col + c0);
      const int m = TALL ? t.N : t.M, n = TALL ? t.M : t.N;
#pragma unroll
      for (int k = 0; k < MAX_BLOCKS; ++k)
#pragma unroll
        for (int e = 0; e < EACH && k < t.blocks; ++e) {
          if (!(r0 + e * DR < m && first_col + k * 64 + c0 + e * DC < n)) continue;
          const uint32_t o = element(k, r0 + e * DR, c0 + e * DC);
          const long i = to + (TALL ? (k * 64 + e * DC) * t.ld_o : e * DR * t.ld_o + k * 64);
          const uint32_t up = *reinterpret_cast<const unsigned short*>(smem + o);
          if (t.out_fp32)
            ((uint32_t*)t.out)[i] = up << 16 | *reinterpret_cast<const unsigned short*>(smem + x_half + o);
          else
            ((unsigned short*)t.out)[i] = (unsigned short)up;
        }
    });
    return;
  }
  // the chunk's share of the next A, and the chunk
  gram_x(acc);
#pragma unroll
  for (int i = 0; i < PER_WAVE; ++i) {
    const int id = wave + i * TINY_WAVES;
    if (id >= GB) continue;
    t.sums_next[(size_t)blockIdx.x * sums_of + id * WAVE + lane] = float4{acc[i][0], acc[i][1], acc[i][2], acc[i][3]};
  }
  for (uint32_t o = tid * 16; o < 2 * x_half; o += TINY_THREADS * 16)
    *reinterpret_cast<u32x4*>(image + o) = *reinterpret_cast<const u32x4*>(smem + o);
}

// The sums of a matrix's chunks in the place of the first one's: where there are many, every workgroup would add up all of them.
__global__ __launch_bounds__(256) void tiny_sum_kernel(float4* __restrict__ sums, int chunks, int per_chunk) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= per_chunk) return;
  float4* from = sums + (size_t)blockIdx.y * chunks * per_chunk + i;
  float4 s = from[0];
#pragma unroll 8
  for (int k = 1; k < chunks; ++k) {
    const float4 v = from[(size_t)k * per_chunk];
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  from[0] = s;
}

// ---- host -----------------------------------------------------------------------------------------

struct Shape {
  int m, n, mp, np;                            // of X, and of its buffer
  bool tall;
  size_t x, a;                                 // elements of a matrix
  Shape(int M, int N)
      : m(std::min(M, N)), n(std::max(M, N)), mp((int)align_up(m, PAD)), np((int)align_up(n, PAD)), tall(M > N),
        x((size_t)mp * np), a((size_t)mp * mp) {}
};

// Where the buffers' powers of two lie: no entry of X exceeds its largest singular value, no entry of A its square, and fp16
// ends at 65504.
struct Scales {
  float s, t, u;
  bool ok;
  Scales(const Shape& q, const float* c, int steps) {
    // the largest singular value that a step can make out of [0, top], on a grid fine enough for a polynomial of degree 5
    double top = 1.0, most = 1.0;
    ok = std::isfinite(c[0]) && std::isfinite(c[1]) && std::isfinite(c[2]);
    for (int k = 0; ok && k < steps; ++k) {
      double next = 0.0;
      for (int i = 1; i <= 2048; ++i) {
        const double x = top * i / 2048.0, y = x * x;
        next = std::max(next, std::fabs(x * (c[0] + y * (c[1] + y * c[2]))));
      }
      top = next * 1.001;
      most = std::max(most, top);
      if (!(top <= 8.0)) ok = false;
    }
    if (!ok) return;
    auto below = [](double v) { return (float)std::exp2(std::floor(std::log2(v))); };
    const double y = most * most;
    s = below(std::min(std::sqrt((double)q.m * q.n), 32000.0 / most));   // entries of about 1
    t = below(60000.0 / y);
    u = below(60000.0 / std::max(y * (std::fabs((double)c[1]) + std::fabs((double)c[2]) * y), 1e-3));
  }
};

constexpr size_t MAX_ELEMENTS = (size_t)1 << 31;

// How few rows are cut: 64-column blocks of a chunk, and chunks; none where X has too many rows.
struct TinyPlan {
  int mp = 0, blocks = 0, chunks = 0;
  TinyPlan(const Shape& q) {
    if (q.m > 128) return;
    mp = q.m <= 32 ? 32 : q.m <= 64 ? 64 : 128;
    const int all = cdiv(q.n, 64);
    blocks = all <= tiny_blocks(mp, true) ? all : tiny_blocks(mp, false);
    chunks = cdiv(all, blocks);
  }
};

struct Workspace {
  double* sums = nullptr;
  Split X[2], A, B;
  unsigned char* image = nullptr;
  float4* partial[2] = {nullptr, nullptr};
  int most;                                    // matrices of a launch: a grid has fewer than 2^32 threads
  size_t bytes;
  Workspace(void* scratch, int dtype, int batch, const Shape& q, const TinyPlan& tiny)
      : most((int)std::max((size_t)1, ((size_t)1 << 21) / (q.x / (PAD * PAD)))) {
    Arena w(scratch);
    batch = std::min(batch, most);
    const bool full = dtype == BM_DTYPE_FP32;
    if (tiny.chunks != 1) sums = w.take<double>((size_t)batch * NORM_PARTS * sizeof(double));
    if (tiny.chunks) {
      if (tiny.chunks > 1) {
        const size_t chunks = (size_t)batch * tiny.chunks;
        image = w.take<unsigned char>(chunks * tiny_x_bytes(tiny.mp, tiny.blocks));
        for (float4*& s : partial) s = w.take<float4>(chunks * tiny_gram_blocks(tiny.mp) * WAVE * sizeof(float4));
      }
    } else {
      for (Split& x : X) {
        x.hi = w.take<half_t>(batch * q.x * sizeof(half_t));
        x.lo = w.take<half_t>(batch * q.x * sizeof(half_t));
      }
      for (Split* x : {&A, &B}) {
        x->hi = w.take<half_t>(batch * q.a * sizeof(half_t));
        x->lo = full ? w.take<half_t>(batch * q.a * sizeof(half_t)) : nullptr;
      }
    }
    bytes = std::max(w.off, (size_t)256);
  }
};

// dynamic LDS beyond 64 KiB, allowed once on each device
template <typename Kernel>
bm_status allow_lds(Kernel kern, size_t lds, std::atomic<uint64_t>* done) {
  int dev = 0;
  BM_CHECK_HIP(hipGetDevice(&dev));
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (done->load(std::memory_order_relaxed) & bit)) return BM_OK;
  BM_CHECK_HIP(hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
  if (dev < 64) done->fetch_or(bit, std::memory_order_relaxed);
  return BM_OK;
}

// GROUPS = 0: the kernel of two groups that take turns
template <int KIND, int TILE, int DEPTH, int GROUPS, bool FULL>
bm_status launch_tile(const Product& p, int batch, hipStream_t st) {
  constexpr bool SYMMETRIC = KIND == GRAM || KIND == POLY;
  constexpr size_t lds = GROUPS ? small_lds(TILE, DEPTH, GROUPS, FULL) : 2 * 2 * TILE * BK * sizeof(half_t);
  void (*kern)(Product, int, int, int);
  if constexpr (GROUPS == 0) kern = large_product_kernel<KIND>;
  else kern = small_product_kernel<KIND, TILE, DEPTH, GROUPS, FULL>;
  static std::atomic<uint64_t> done{0};
  BM_RETURN_IF(allow_lds(kern, lds, &done));
  const int tm = cdiv(p.M, TILE), tn = cdiv(p.N, TILE), tiles = SYMMETRIC ? tm * (tm + 1) / 2 : tm * tn;
  ProfScope prof(SYMMETRIC ? PROF_GEMM_NT : PROF_GEMM_NN, (SYMMETRIC ? 1.0 : 2.0) * batch * p.terms * p.M * p.N * p.K, st);
  hipLaunchKernelGGL(kern, dim3((unsigned)((long)tiles * batch)), dim3(GROUPS ? 256 * GROUPS : 512), lds, st, p, tm, tn, tiles);
  BM_CHECK_LAUNCH("orthogonalize product");
  return BM_OK;
}

template <int KIND, int TILE>
bm_status launch_middle(const Product& p, int batch, hipStream_t st) {
  static std::atomic<uint64_t> done{0};
  auto kern = middle_product_kernel<KIND, TILE>;
  BM_RETURN_IF(allow_lds(kern, middle_lds(TILE), &done));
  const int t = cdiv(p.M, TILE), tiles = t * (t + 1) / 2;
  ProfScope prof(PROF_GEMM_NT, (double)batch * p.terms * p.M * p.N * p.K, st);
  hipLaunchKernelGGL(kern, dim3((unsigned)((long)tiles * batch)), dim3(768), middle_lds(TILE), st, p, t, t, tiles);
  BM_CHECK_LAUNCH("orthogonalize product");
  return BM_OK;
}

// Operands come from L2 at 50-60 bytes per ns and CU whatever the kernel (deeper prefetch, fragments read ahead, wavefronts with whole
// tiles of their own and a compact order of the tiles in an XCD changed nothing), so tiles are as large as leaves one for every CU.
// A whole update in us, 256x256 / 128x128 / 64x64 two workgroups a CU / 64x64 two groups:
//   1024 x 1024 420, 243, 160, 149     1536 x 1536 555, 325, 282, 335     2048 x 2048 704, 424, 499, 575     16 of 1024 x 1024 598, 757, 805, 1060
// A CU fetches the operands of one tile after the other, so a symmetric product takes the rounds of the chip times the tile's size:
// 4096 rows are 136 tiles of 256 for 256 CUs, but 253 of 192.  A whole update without and with 192 x 192:
//   4096 x 4096 1448, 1374 (fp32 3822, 3682)     4096 x 14336 3900, 3769     3584 x 3584 1153, 1033     50 of 300 x 300 246, 217
// and with 96 x 96:
//   2048 x 2048 359, 317     2048 x 8192 840, 732     1792 x 7168 611, 573     1536 x 1536 224, 227
template <int KIND>
bm_status launch(const Product& p, int batch, hipStream_t st) {
  constexpr bool SYMMETRIC = KIND == GRAM || KIND == POLY;
  auto tiles = [&](int size) {
    const long tm = cdiv(p.M, size), tn = cdiv(p.N, size);
    return (SYMMETRIC ? tm * (tm + 1) / 2 : tm * tn) * batch;
  };
  constexpr int NUM_CU = 256;
  if constexpr (SYMMETRIC) {
    auto rounds = [&](int size) { return (tiles(size) + NUM_CU - 1) / NUM_CU * size; };
    if (tiles(192) > NUM_CU / 2 && rounds(192) < std::min(rounds(128), rounds(256))) return launch_middle<KIND, 192>(p, batch, st);
    if (p.terms == 1 && tiles(96) > NUM_CU / 2 && tiles(64) > NUM_CU && rounds(96) < std::min(rounds(128), rounds(256)))
      return launch_middle<KIND, 96>(p, batch, st);
  }
  if (tiles(256) >= NUM_CU / 2) return launch_tile<KIND, 256, 2, 0, false>(p, batch, st);
  if (p.terms > 1) {
    if (tiles(64) <= NUM_CU) return launch_tile<KIND, 64, 2, 2, true>(p, batch, st);
    if (tiles(128) <= NUM_CU / 2) return launch_tile<KIND, 64, 2, 1, true>(p, batch, st);
    return launch_tile<KIND, 128, 2, 1, true>(p, batch, st);
  }
  if (tiles(64) <= NUM_CU) return launch_tile<KIND, 64, 4, 2, false>(p, batch, st);
  if (tiles(128) <= NUM_CU / 2) return launch_tile<KIND, 64, 4, 1, false>(p, batch, st);
  return launch_tile<KIND, 128, 2, 2, false>(p, batch, st);
}

template <int MP, bool FULL, int MODE>
bm_status launch_tiny(const Tiny& t, int batch, hipStream_t st) {
  auto kern = tiny_kernel<MP, FULL, MODE>;
  static std::atomic<uint64_t> done{0};
  constexpr int MOST = tiny_blocks(MP, MODE == SOLO);
  static_assert(tiny_lds(MP, MOST, MODE == SOLO) <= 160 * 1024, "a chunk with A or B");
  BM_RETURN_IF(allow_lds(kern, tiny_lds(MP, MOST, MODE == SOLO), &done));
  hipLaunchKernelGGL(kern, dim3((unsigned)((long)batch * t.chunks)), dim3(TINY_THREADS), tiny_lds(MP, t.blocks, MODE == SOLO), st, t);
  BM_CHECK_LAUNCH("orthogonalize few rows");
  return BM_OK;
}

// Chunks whose sums every workgroup adds up for itself.  A whole update in us without and with a launch that does it once:
//   128 x 512 (4 chunks) 80.2, 81.3    128 x 896 (7) 93.8, 86.1    100 x 4096 (32) 125.4, 96.7
//   64 x 8192 (32) 62.0, 68.9    64 x 16384 (64) 82.2, 82.3    64 x 32768 (128) 115.9, 103.7
//   32 x 131072 (256) 135.3, 143.2    32 x 262144 (512) 391, 257
constexpr int tiny_summands(int mp) { return mp == 128 ? 4 : mp == 64 ? 64 : 256; }

template <int MP, bool FULL>
bm_status run_tiny(Tiny t, int batch, const Workspace& w, hipStream_t st) {
  if (t.chunks == 1) return launch_tiny<MP, FULL, SOLO>(t, batch, st);
  t.sums_next = w.partial[0];
  BM_RETURN_IF((launch_tiny<MP, FULL, FIRST>(t, batch, st)));
  for (t.step = 0; t.step < t.steps; ++t.step) {
    t.sums = w.partial[t.step & 1];
    t.sums_next = w.partial[(t.step + 1) & 1];
    t.summands = t.chunks;
    if (t.chunks > tiny_summands(MP) && batch < 65536) {
      constexpr int per_chunk = tiny_gram_blocks(MP) * WAVE;
      hipLaunchKernelGGL(tiny_sum_kernel, dim3(cdiv(per_chunk, 256), batch), dim3(256), 0, st, w.partial[t.step & 1], t.chunks, per_chunk);
      BM_CHECK_LAUNCH("orthogonalize sums");
      t.summands = 1;
    }
    BM_RETURN_IF((launch_tiny<MP, FULL, NEXT>(t, batch, st)));
  }
  return BM_OK;
}

bool sizes_ok(int dtype, int batch, int M, int N) {
  if (!good_dtype(dtype) || batch <= 0 || M <= 0 || N <= 0) return false;
  if (M > (1 << 20) || N > (1 << 20)) return false;
  const Shape q(M, N);
  return q.x < MAX_ELEMENTS && (double)batch * (q.mp / 64) * (q.np / 64) < 2147483648.0;
}

bm_status run(bool full, int batch, int M, int N, const Shape& q, const TinyPlan& tiny, const Scales& k, const Workspace& w,
              const float* grad, int32_t ld_g, int64_t stride_g, void* out, int32_t ld_o, int64_t stride_o,
              const float* coefficients, int32_t steps, float eps, hipStream_t st) {
  const int terms = full ? 3 : 1;
  const float a = coefficients[0], b = coefficients[1], c = coefficients[2];
  // X that enters step i is kept in 22 bits where that step's result still feeds two more
  auto in_full = [&](int i) { return full || i + 2 < steps; };
  auto view = [](Split x, bool lo) { if (!lo) x.lo = nullptr; return x; };

  // rows of G that start on 16 bytes are read four elements at a time (matrices of an odd stride start where they like); rows without a
  // gap are one long row
  const bool vec = aligned16(grad) && ld_g % 4 == 0 && N % 4 == 0 && (batch == 1 || stride_g % 4 == 0);
  const uint32_t pieces = (uint32_t)((size_t)M * N / (vec ? 4 : 1)), per_row = ld_g == N ? pieces : (uint32_t)(vec ? N / 4 : N);
  // enough parts for 8 workgroups a CU, none without 4 pieces a thread
  const int parts = std::max(1, std::min({NORM_PARTS, cdiv(2048, batch), cdiv(pieces, 1024)}));
  auto norms = [&]() -> bm_status {
    hipLaunchKernelGGL((vec ? norm_kernel<4> : norm_kernel<1>), dim3((unsigned)batch * parts), dim3(256), 0, st, grad, (long)ld_g,
                       (long)stride_g, per_row, pieces, parts, w.sums);
    BM_CHECK_LAUNCH("orthogonalize norm");
    return BM_OK;
  };
  if (tiny.chunks) {
    ProfScope prof(PROF_GEMM_NT, steps * (double)batch * terms * ((double)q.m * q.m * (3.0 * q.n + q.m)), st);
    if (tiny.chunks > 1) BM_RETURN_IF(norms());
    Tiny t{};
    t.g = grad; t.ld_g = ld_g; t.stride_g = stride_g;
    t.M = M; t.N = N; t.tall = q.tall;
    t.norms = w.sums; t.parts = parts;
    t.eps = eps; t.s = k.s; t.t = k.t; t.u = k.u;
    t.a = a; t.b = b; t.c = c;
    t.steps = steps;
    t.full_from = full || tiny.mp == 32 ? steps : std::max(0, steps - 2);
    t.blocks = tiny.blocks; t.chunks = tiny.chunks;
    t.image = w.image;
    t.out = out; t.ld_o = ld_o; t.stride_o = stride_o;
    t.out_fp32 = full;
    if (tiny.mp == 32) return run_tiny<32, true>(t, batch, w, st);
    if (tiny.mp == 64) return full ? run_tiny<64, true>(t, batch, w, st) : run_tiny<64, false>(t, batch, w, st);
    return full ? run_tiny<128, true>(t, batch, w, st) : run_tiny<128, false>(t, batch, w, st);
  }
  BM_RETURN_IF(norms());
  const int tiles_n = q.np / PAD, across = std::max(1, std::min(4, (int)((long)tiles_n * (q.mp / PAD) * batch / 2048)));
  const int runs_n = cdiv(tiles_n, across), runs = q.mp / PAD * runs_n;
  const bool rows_vec = aligned16(grad) && ld_g % 4 == 0 && (batch == 1 || stride_g % 4 == 0);
  const auto convert = q.tall ? (rows_vec ? convert_kernel<true, true> : convert_kernel<true, false>)
                              : (rows_vec ? convert_kernel<false, true> : convert_kernel<false, false>);
  hipLaunchKernelGGL(convert, dim3((unsigned)((long)batch * runs)), dim3(256), 0, st, grad, (long)ld_g, (long)stride_g, M, N, w.sums, parts,
                     eps, k.s, view(w.X[0], in_full(0)), q.np, q.x, tiles_n, runs_n, across, runs);
  BM_CHECK_LAUNCH("orthogonalize convert");
  for (int i = 0; i < steps; ++i) {
    const Split x = view(w.X[i & 1], in_full(i)), next = view(w.X[(i + 1) & 1], in_full(i + 1));
    Product p{};
    p.terms = terms;
    p.A = x; p.B = x; p.C = w.A;
    p.M = p.N = q.mp; p.K = q.np;
    p.lda = p.ldb = q.np; p.ldc = q.mp;
    p.stride_a = p.stride_b = q.x; p.stride_c = q.a;
    p.alpha = k.t / (k.s * k.s);
    BM_RETURN_IF(launch<GRAM>(p, batch, st));
    p.A = w.A; p.B = w.A; p.C = w.B; p.old = w.A;
    p.K = q.mp; p.lda = p.ldb = q.mp;
    p.stride_a = p.stride_b = q.a;
    p.alpha = c * (k.u / k.t) / k.t;
    p.beta = b * (k.u / k.t);
    BM_RETURN_IF(launch<POLY>(p, batch, st));
    p.A = w.B; p.B = x; p.C = next; p.old = x;
    p.N = q.np; p.ldb = p.ldc = q.np;
    p.stride_b = p.stride_c = q.x;
    p.alpha = 1.f / k.u;
    p.beta = a;
    if (i + 1 < steps) {
      BM_RETURN_IF(launch<STEP>(p, batch, st));
    } else {
      p.alpha /= k.s;
      p.beta /= k.s;
      p.out = out; p.ld_o = ld_o; p.stride_o = stride_o;
      p.rows = q.m; p.cols = q.n; p.transposed = q.tall; p.out_fp32 = full;
      BM_RETURN_IF(launch<LAST>(p, batch, st));
    }
  }
  return BM_OK;
}

}  // namespace
}  // namespace bm

using namespace bm;

extern "C" size_t bm_orthogonalize_scratch_bytes(int32_t dtype, int32_t batch, int32_t M, int32_t N) {
  return sizes_ok(dtype, batch, M, N) ? Workspace(nullptr, dtype, batch, Shape(M, N), TinyPlan(Shape(M, N))).bytes : 0;
}

extern "C" bm_status bm_orthogonalize(int32_t dtype, int32_t batch, int32_t M, int32_t N, const float* grad, int32_t ld_g,
                                      int64_t stride_g, void* out, int32_t ld_o, int64_t stride_o, const float* coefficients,
                                      int32_t steps, float eps, void* scratch, size_t scratch_bytes, void* hip_stream) {
  BM_ARG_CHECK(good_dtype(dtype), "bm_orthogonalize: dtype %d", dtype);
  BM_ARG_CHECK(batch >= 0 && M > 0 && N > 0, "bm_orthogonalize: bad sizes");
  BM_ARG_CHECK(ld_g >= N && ld_o >= N, "bm_orthogonalize: leading dimension too small");
  BM_ARG_CHECK(stride_g >= 0 && stride_o >= 0, "bm_orthogonalize: negative stride");
  // one behind the other, or side by side in wider rows
  BM_ARG_CHECK(batch <= 1 || stride_o >= (int64_t)(M - 1) * ld_o + N || (stride_o >= N && (batch - 1) * stride_o + N <= ld_o),
               "bm_orthogonalize: the results of a batch overlap");
  BM_ARG_CHECK(steps >= 1 && steps <= 64, "bm_orthogonalize: %d steps", steps);
  BM_ARG_CHECK(eps >= 0.f && std::isfinite(eps), "bm_orthogonalize: bad eps");
  BM_ARG_CHECK(coefficients, "bm_orthogonalize: NULL coefficients");
  if (batch == 0) return BM_OK;
  BM_ARG_CHECK(sizes_ok(dtype, batch, M, N), "bm_orthogonalize: %d matrices of %d x %d are too large", batch, M, N);
  BM_ARG_CHECK(grad && out && aligned16(grad) && aligned16(out) && aligned16(scratch), "bm_orthogonalize: NULL or misaligned tensor");
  const Shape q(M, N);
  const Scales k(q, coefficients, steps);
  if (!k.ok) {
    set_error("bm_orthogonalize: singular values do not stay below 8 under these coefficients");
    return BM_ERR_UNSUPPORTED;
  }
  const TinyPlan tiny(q);
  const Workspace w(scratch, dtype, batch, q, tiny);
  if (!scratch || scratch_bytes < w.bytes) {
    set_error("bm_orthogonalize needs %zu scratch bytes, got %zu", w.bytes, scratch_bytes);
    return BM_ERR_WORKSPACE_TOO_SMALL;
  }
  const bool full = dtype == BM_DTYPE_FP32;
  // matrices of few rows are read and written by a workgroup each, without regard to the others
  const bool same = full && (const void*)grad == out && ld_o == ld_g && (batch == 1 || stride_o == stride_g);
  auto end_of = [&](const void* p, int64_t stride, int ld, int bytes) {
    return reinterpret_cast<uintptr_t>(p) + (uintptr_t)((batch - 1) * stride + (int64_t)(M - 1) * ld + N) * bytes;
  };
  BM_ARG_CHECK(same || end_of(grad, stride_g, ld_g, 4) <= reinterpret_cast<uintptr_t>(out) ||
                   end_of(out, stride_o, ld_o, full ? 4 : 2) <= reinterpret_cast<uintptr_t>(grad),
               "bm_orthogonalize: the result overlaps the gradient without being it");
  for (int first = 0; first < batch; first += std::min(w.most, batch - first))
    BM_RETURN_IF(run(full, std::min(w.most, batch - first), M, N, q, tiny, k, w, grad + first * stride_g, ld_g, stride_g,
                     (char*)out + first * stride_o * (full ? 4 : 2), ld_o, stride_o, coefficients, steps, eps, (hipStream_t)hip_stream));
  return BM_OK;
}
