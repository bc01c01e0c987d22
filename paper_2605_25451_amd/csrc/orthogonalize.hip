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
// until the last two steps, where it enters the sum a X in full and the products as hi alone: 0.08-0.14 % off on noise and on spectra that
// fall over three decades (hi alone all the time: 0.14 and 0.4-0.7 %).  For fp32 results all of X, A and B are hi + lo and every
// product is three, hi hi + hi lo + lo hi: 3e-7 to 1.3e-6 off.
// fp16's range: with powers of two s, t and u the buffers hold s X, t A and u B (see Scales).
#include "train.h"

#include <algorithm>
#include <cmath>

namespace bm {

namespace {

typedef _Float16 half_t;
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int PAD = 64;                        // rows and columns of the buffers are whole 64, the rest zeros

struct Split { half_t *hi, *lo; };             // lo may be null: hi alone

__device__ inline void put(const Split& d, size_t i, float v) {
  const half_t h = (half_t)v;
  d.hi[i] = h;
  if (d.lo) d.lo[i] = (half_t)(v - (float)h);
}
__device__ inline float get(const Split& d, size_t i) { return (float)d.hi[i] + (d.lo ? (float)d.lo[i] : 0.f); }

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

// ---- norm and conversion ----------------------------------------------------------------------

constexpr int NORM_PARTS = 64;

// sums of squares of parts of every matrix, in fp64: squares of fp32 values neither overflow nor vanish there
__global__ __launch_bounds__(256) void norm_kernel(const float* __restrict__ g, long ld, long stride, int M, int N, int parts,
                                                   double* __restrict__ sums) {
  __shared__ double sm[4];
  const int b = blockIdx.x / parts, part = blockIdx.x % parts;
  const float* x = g + b * stride;
  double s = 0.0;
  for (int r = part; r < M; r += parts)
    for (int c = threadIdx.x; c < N; c += 256) {
      const double v = x[r * ld + c];
      s += v * v;
    }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, WAVE);
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) sums[blockIdx.x] = sm[0] + sm[1] + sm[2] + sm[3];
}

// x[m, n] = s G / (|G| + eps), transposed where the rows of G are the columns of x.  A workgroup: 64 x 64 of x.
__global__ __launch_bounds__(256) void convert_kernel(const float* __restrict__ g, long ld, long stride, int M, int N, int transposed,
                                                      const double* __restrict__ sums, int parts, float eps, float s, Split x,
                                                      int ldx, size_t stride_x, int tiles_n, int tiles) {
  __shared__ float tile[PAD][PAD + 1];
  const int b = blockIdx.x / tiles, t = blockIdx.x % tiles;
  const int r0 = (t / tiles_n) * PAD, c0 = (t % tiles_n) * PAD;          // of x
  double sum = 0.0;
  for (int p = 0; p < parts; ++p) sum += sums[(size_t)b * parts + p];
  const double scale = (double)s / (sqrt(sum) + (double)eps);
  const int gr0 = transposed ? c0 : r0, gc0 = transposed ? r0 : c0;
  for (int i = threadIdx.x; i < PAD * PAD; i += 256) {
    const int r = i / PAD, c = i % PAD;
    float v = 0.f;
    if (gr0 + r < M && gc0 + c < N) v = (float)((double)g[b * stride + (gr0 + r) * ld + gc0 + c] * scale);
    if (transposed) tile[c][r] = v; else tile[r][c] = v;
  }
  __syncthreads();
  x.hi += b * stride_x;
  if (x.lo) x.lo += b * stride_x;
  for (int i = threadIdx.x; i < PAD * PAD; i += 256) {
    const int r = i / PAD, c = i % PAD;
    put(x, (size_t)(r0 + r) * ldx + c0 + c, tile[r][c]);
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

// One 64 x 64 tile: four wavefronts of 32 x 32.  NN: B lies [K, N], else [N, K].
template <int KIND>
__global__ __launch_bounds__(256) void small_product_kernel(Product p, int tiles, int tiles_n) {
  constexpr bool NN = KIND == STEP || KIND == LAST, SYMMETRIC = !NN;
  constexpr int LD = 72;                       // halves of an LDS row: 144 bytes, so that rows differ in their banks
  __shared__ __attribute__((aligned(16))) half_t sa[64 * LD], sb[64 * LD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b = blockIdx.x / tiles, t = blockIdx.x % tiles;
  int tm, tn;
  if (SYMMETRIC) triangle_tile(t, tiles_n, &tm, &tn);
  else { tm = t / tiles_n; tn = t % tiles_n; }
  const int m0 = tm * 64, n0 = tn * 64;
  f32x4 acc[2][2] = {};
  for (int term = 0; term < p.terms; ++term) {
    const half_t* A = (term == 2 ? p.A.lo : p.A.hi) + b * p.stride_a;
    const half_t* B = (term == 1 ? p.B.lo : p.B.hi) + b * p.stride_b;
    for (int k0 = 0; k0 < p.K; k0 += 64) {
      half8 ra[2], rb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int id = threadIdx.x + i * 256, r = id >> 3, c = (id & 7) * 8;
        ra[i] = *reinterpret_cast<const half8*>(A + (size_t)(m0 + r) * p.lda + k0 + c);
        rb[i] = *reinterpret_cast<const half8*>(NN ? B + (size_t)(k0 + r) * p.ldb + n0 + c : B + (size_t)(n0 + r) * p.ldb + k0 + c);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int id = threadIdx.x + i * 256, r = id >> 3, c = (id & 7) * 8;
        *reinterpret_cast<half8*>(sa + r * LD + c) = ra[i];
        if (NN) {
#pragma unroll
          for (int e = 0; e < 8; ++e) sb[(c + e) * LD + r] = rb[i][e];
        } else {
          *reinterpret_cast<half8*>(sb + r * LD + c) = rb[i];
        }
      }
      __syncthreads();
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        half8 fa[2], fb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          fa[i] = *reinterpret_cast<const half8*>(sa + ((wave >> 1) * 32 + i * 16 + (lane & 15)) * LD + ks * 32 + (lane >> 4) * 8);
          fb[i] = *reinterpret_cast<const half8*>(sb + ((wave & 1) * 32 + i * 16 + (lane & 15)) * LD + ks * 32 + (lane >> 4) * 8);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[i], fb[j], acc[i][j], 0, 0, 0);
      }
    }
  }
  Split C = p.C, old = p.old;
  if (KIND != LAST) { C.hi += b * p.stride_c; if (C.lo) C.lo += b * p.stride_c; }
  if (KIND != GRAM) { old.hi += b * p.stride_c; if (old.lo) old.lo += b * p.stride_c; }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = m0 + (wave >> 1) * 32 + i * 16 + (lane >> 4) * 4 + e, c = n0 + (wave & 1) * 32 + j * 16 + (lane & 15);
        const size_t at = (size_t)r * p.ldc + c;
        float v = p.alpha * acc[i][j][e];
        if (KIND != GRAM) v += p.beta * get(old, at);
        if (KIND == LAST) {
          if (r < p.rows && c < p.cols) {
            const long o = b * p.stride_o + (p.transposed ? c * p.ld_o + r : r * p.ld_o + c);
            if (p.out_fp32) ((float*)p.out)[o] = v;
            else ((bf16_t*)p.out)[o] = (bf16_t)v;
          }
        } else {
          put(C, at, v);
          if (SYMMETRIC && tm != tn) put(C, (size_t)c * p.ldc + r, v);
        }
      }
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

struct Workspace {
  double* sums;
  Split X[2], A, B;
  size_t bytes;
  Workspace(void* scratch, int dtype, int batch, const Shape& q) {
    Arena w(scratch);
    const bool full = dtype == BM_DTYPE_FP32;
    sums = w.take<double>((size_t)batch * NORM_PARTS * sizeof(double));
    for (Split& x : X) {
      x.hi = w.take<half_t>(batch * q.x * sizeof(half_t));
      x.lo = w.take<half_t>(batch * q.x * sizeof(half_t));
    }
    for (Split* x : {&A, &B}) {
      x->hi = w.take<half_t>(batch * q.a * sizeof(half_t));
      x->lo = full ? w.take<half_t>(batch * q.a * sizeof(half_t)) : nullptr;
    }
    bytes = w.off;
  }
};

template <int KIND>
bm_status launch(const Product& p, int batch, hipStream_t st) {
  const int tm = p.M / 64, tn = p.N / 64;
  const int tiles = KIND == GRAM || KIND == POLY ? tm * (tm + 1) / 2 : tm * tn;
  ProfScope prof(KIND == GRAM || KIND == POLY ? PROF_GEMM_NT : PROF_GEMM_NN, 2.0 * batch * p.M * p.N * p.K, st);
  hipLaunchKernelGGL(small_product_kernel<KIND>, dim3((unsigned)((long)tiles * batch)), dim3(256), 0, st, p, tiles, tn);
  BM_CHECK_LAUNCH("orthogonalize product");
  return BM_OK;
}

bool sizes_ok(int dtype, int batch, int M, int N) {
  if (!good_dtype(dtype) || batch <= 0 || M <= 0 || N <= 0) return false;
  if (M > (1 << 20) || N > (1 << 20)) return false;
  const Shape q(M, N);
  return q.x < MAX_ELEMENTS && (double)batch * (q.mp / 64) * (q.np / 64) < 2147483648.0;
}

}  // namespace
}  // namespace bm

using namespace bm;

extern "C" size_t bm_orthogonalize_scratch_bytes(int32_t dtype, int32_t batch, int32_t M, int32_t N) {
  return sizes_ok(dtype, batch, M, N) ? Workspace(nullptr, dtype, batch, Shape(M, N)).bytes : 0;
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
  const Workspace w(scratch, dtype, batch, q);
  if (!scratch || scratch_bytes < w.bytes) {
    set_error("bm_orthogonalize needs %zu scratch bytes, got %zu", w.bytes, scratch_bytes);
    return BM_ERR_WORKSPACE_TOO_SMALL;
  }
  hipStream_t st = (hipStream_t)hip_stream;
  const bool full = dtype == BM_DTYPE_FP32;
  const int terms = full ? 3 : 1;
  const float a = coefficients[0], b = coefficients[1], c = coefficients[2];
  // X that enters step i is kept in 22 bits where that step's result still feeds two more
  auto in_full = [&](int i) { return full || i + 2 < steps; };
  auto view = [](Split x, bool lo) { if (!lo) x.lo = nullptr; return x; };

  hipLaunchKernelGGL(norm_kernel, dim3(batch * NORM_PARTS), dim3(256), 0, st, grad, (long)ld_g, (long)stride_g, M, N, NORM_PARTS, w.sums);
  BM_CHECK_LAUNCH("orthogonalize norm");
  const int tiles_n = q.np / PAD, tiles = q.mp / PAD * tiles_n;
  hipLaunchKernelGGL(convert_kernel, dim3((unsigned)((long)batch * tiles)), dim3(256), 0, st, grad, (long)ld_g, (long)stride_g, M, N,
                     (int)q.tall, w.sums, NORM_PARTS, eps, k.s, view(w.X[0], in_full(0)), q.np, q.x, tiles_n, tiles);
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
