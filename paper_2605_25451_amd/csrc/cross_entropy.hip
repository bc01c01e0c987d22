// Cross-entropy of a vocabulary and its gradient: with m the largest logit of a row and s the sum of exp(z - m),
//   loss = w (m + log s - z[label]),   dz = w (exp(z - m) / s - onehot(label)).
// m and s come from one pass: a thread rescales its sum when its maximum grows, and pairs (m, s) are joined.
// A row whose label is negative is never read.  Bound by HBM.
//
// Rows that fit the registers of a workgroup are read once (row_kernel).  Wider ones, and a few wide ones, which would leave the chip
// idle, are cut into parts: one launch for the parts' (m, s), one that joins those of a row and writes its gradient; the
// second read of the logits comes from the memory-side cache where they fit.
// 4096 x 128000 bf16: 2.10 GB in 389 us, 5.4 TB/s (a copy of 2 GB moves 4.9 TB/s).
#include "train.h"

#include <float.h>

#include <algorithm>

namespace bm {

namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// exp(x - m) with the difference first: its rounding does not grow with the logits
__device__ inline float exp_diff(float x, float m) { return __builtin_amdgcn_exp2f((x - m) * LOG2E); }

// running maximum and sum.  The maximum starts at the lowest finite value, so that -inf adds exp(-inf) = 0.
struct Stat {
  float m, s;
  static __device__ inline Stat none() { return Stat{-FLT_MAX, 0.f}; }
  template <int N> __device__ inline void add(const float (&x)[N]) {
    float top = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) top = fmaxf(top, x[e]);
    top = fmaxf(top, m);
    s *= exp_diff(m, top);
#pragma unroll
    for (int e = 0; e < N; ++e) s += exp_diff(x[e], top);
    m = top;
  }
  __device__ inline void join(const Stat& o) {
    const float top = fmaxf(m, o.m);
    s = s * exp_diff(m, top) + o.s * exp_diff(o.m, top);
    m = top;
  }
};

__device__ inline Stat wave_join(Stat a) {
  Stat r;
  r.m = wave_max(a.m);
  r.s = wave_sum(a.s * exp_diff(a.m, r.m));
  return r;
}

// The statistics of a workgroup, in every thread; sm: one of every wavefront.  Ends in a barrier.
template <int THREADS>
__device__ inline Stat block_join(Stat a, Stat* sm) {
  a = wave_join(a);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = a;
  __syncthreads();
  a = sm[0];
#pragma unroll 1
  for (int w = 1; w < THREADS / WAVE; ++w) a.join(sm[w]);
  return a;
}

// A row in 16-byte vectors: `head` elements up to the first boundary, whole vectors, the rest.
template <typename T>
struct Span {
  static constexpr int W = Elt<T>::VEC;
  int head, vecs, tail;                                     // tail: the first element behind the vectors
  __device__ inline Span(const T* row, int V) {
    head = min(V, (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(T));
    vecs = (V - head) / W;
    tail = head + vecs * W;
  }
};

template <typename T>
__device__ inline float label_logit(const T* row, int label, int V) {
  return label < V ? Elt<T>::to_f(row[label]) : __builtin_nanf("");
}

// ---- parts of rows ------------------------------------------------------------------------------

constexpr int PART_THREADS = 256;

template <typename T>
__global__ __launch_bounds__(PART_THREADS) void part_stats_kernel(const T* __restrict__ logits, long ld, const int32_t* __restrict__ labels,
                                                                  int V, int parts, Stat* __restrict__ stats, float* __restrict__ at_label) {
  __shared__ Stat sm[PART_THREADS / WAVE];
  const int row = blockIdx.x / parts, part = blockIdx.x % parts;
  const int label = labels[row];
  if (label < 0) return;
  const T* x = logits + (size_t)row * ld;
  const Span<T> sp(x, V);
  const int per = (sp.vecs + parts - 1) / parts, first = min(sp.vecs, part * per), last = min(sp.vecs, first + per);
  Stat a = Stat::none();
#pragma unroll 4
  for (int i = first + threadIdx.x; i < last; i += PART_THREADS) {
    float v[Span<T>::W];
    load16(x + sp.head + i * Span<T>::W, v);
    a.add(v);
  }
  if (part == 0) {
    const int i = threadIdx.x < sp.head ? (int)threadIdx.x : sp.tail + (int)threadIdx.x - sp.head;
    if (i < V) {
      const float v[1] = {Elt<T>::to_f(x[i])};
      a.add(v);
    }
    if (threadIdx.x == 0) at_label[row] = label_logit(x, label, V);
  }
  a = block_join<PART_THREADS>(a, sm);
  if (threadIdx.x == 0) stats[(size_t)row * parts + part] = a;
}

// writes: parts of a row that write the gradient; 0 with dlogits == nullptr, where the grid holds one workgroup of a row
template <typename T>
__global__ __launch_bounds__(PART_THREADS) void part_finish_kernel(const T* logits, long ld, const int32_t* __restrict__ labels,
                                                                   const float* __restrict__ weight, int V, int parts, int writes,
                                                                   const Stat* __restrict__ stats, const float* __restrict__ at_label,
                                                                   float* __restrict__ loss, T* dlogits, long ld_d) {
  constexpr int W = Span<T>::W;
  const int wgs = max(writes, 1);
  const int row = blockIdx.x / wgs, part = blockIdx.x % wgs;
  const int label = labels[row];
  const T* x = logits + (size_t)row * ld;
  T* g = dlogits + (size_t)row * ld_d;
  Stat a = Stat::none();
  float scale = 0.f, w = 0.f, xl = 0.f;
  if (label >= 0) {
    for (int p = 0; p < parts; ++p) a.join(stats[(size_t)row * parts + p]);
    xl = at_label[row];
    w = weight ? weight[row] : 1.f;
    if (label >= V) w = xl;                                 // NaN
    scale = w / a.s;
  }
  if (part == 0 && threadIdx.x == 0 && loss) loss[row] = label >= 0 ? w * (a.m - xl + logf(a.s)) : 0.f;
  if (!writes) return;
  const Span<T> sp(g, V);                                   // vectors of what is written
  const bool same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15) == 0;
  const int per = (sp.vecs + writes - 1) / writes, first = min(sp.vecs, part * per), last = min(sp.vecs, first + per);
  auto one = [&](int i) {
    float v = label >= 0 ? exp_diff(Elt<T>::to_f(x[i]), a.m) * scale : 0.f;
    if (i == label) v -= w;
    g[i] = Elt<T>::from_f(v);
  };
#pragma unroll 4
  for (int i = first + threadIdx.x; i < last; i += PART_THREADS) {
    const int c = sp.head + i * W;
    float v[W];
    if (label < 0) {
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] = 0.f;
    } else {
      if (same) {
        load16(x + c, v);
      } else {
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] = Elt<T>::to_f(x[c + e]);
      }
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] = exp_diff(v[e], a.m) * scale - (c + e == label ? w : 0.f);
    }
    store16(g + c, v);
  }
  if (part == 0) {
    const int i = threadIdx.x < sp.head ? (int)threadIdx.x : sp.tail + (int)threadIdx.x - sp.head;
    if (i < V) one(i);
  }
}

// ---- whole rows -----------------------------------------------------------------------------------

typedef unsigned int Quad __attribute__((ext_vector_type(4)));

// The same statistics with an instruction less per element: exp(x - m) as 2^(x L - c), c = m L rounded once, which makes 2^(m L - c)
// a common factor of all terms.  m L - c is half a step of c at most: 1/2 up to |m| = MOST, but from 1e9 on the factor can leave fp32's
// range.  So the maximum starts at -MOST (a thread whose words are all masked with -1e30 or -inf adds nothing), and a row whose
// largest logit is not between -MOST and MOST is done again with the difference first.
struct Stat2 {
  static constexpr float MOST = 0x1p23f;
  float m, c, s;
  // (the same rounded product wherever it is taken, never part of a fused multiply-add)
  static __device__ inline float scaled(float m) {
#pragma clang fp contract(off)
    return m * LOG2E;
  }
  static __device__ inline Stat2 none() { return Stat2{-MOST, -MOST * LOG2E, 0.f}; }
  static __device__ inline float term(float x, float c) { return __builtin_amdgcn_exp2f(fmaf(x, LOG2E, -c)); }
  template <int N> __device__ inline void add(const float (&x)[N]) {
    float top = m;
#pragma unroll
    for (int e = 0; e < N; ++e) top = fmaxf(top, x[e]);
    const float c1 = scaled(top);
    s *= __builtin_amdgcn_exp2f(c - c1);
#pragma unroll
    for (int e = 0; e < N; ++e) s += term(x[e], c1);
    m = top;
    c = c1;
  }
};
template <int THREADS>
__device__ inline Stat2 block_join(Stat2 a, Stat2* sm) {
  const float m = wave_max(a.m), c = Stat2::scaled(m);
  const float s = wave_sum(a.s * __builtin_amdgcn_exp2f(a.c - c));
  if (THREADS == WAVE) return Stat2{m, c, s};
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = Stat2{m, c, s};
  __syncthreads();
  // every wavefront joins those of all, one per lane
  constexpr int WAVES = THREADS / WAVE;
  Stat2 r = sm[threadIdx.x % WAVES];
  float top = r.m;
#pragma unroll
  for (int off = 1; off < WAVES; off <<= 1) top = fmaxf(top, __shfl_xor(top, off, WAVE));
  const float c1 = Stat2::scaled(top);
  r.s *= __builtin_amdgcn_exp2f(r.c - c1);
#pragma unroll
  for (int off = 1; off < WAVES; off <<= 1) r.s += __shfl_xor(r.s, off, WAVE);
  r.m = top;
  r.c = c1;
  return r;
}

// A workgroup holds a row in its registers, NV vectors per thread, so that the logits are read once.  Neither they nor the gradient are
// used again before a cache has lost them: with non-temporal accesses 256 x 128000 take 26 us instead of 31.  One workgroup per
// row: persistent ones that fetch the next row under the gradient of the last keep in step with one another, so that all read, compute
// and write at the same time (4096 x 64000 249 us, this 186; 8192 x 8000 93 and 47), and have more to do where fewer rows are ignored.
// Rows of logits and gradient start at the same place between two 16-byte boundaries.
template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void row_kernel(const T* logits, long ld, const int32_t* __restrict__ labels,
                                                      const float* __restrict__ weight, int V, float* __restrict__ loss, T* dlogits,
                                                      long ld_d) {
  constexpr int W = Span<T>::W;
  __shared__ Stat2 sm[THREADS / WAVE];
  __shared__ Stat sm_far[THREADS / WAVE];
  const int tid = threadIdx.x, row = blockIdx.x, label = labels[row];
  const T* x = logits + (size_t)row * ld;
  T* g = dlogits + (size_t)row * ld_d;
  const Span<T> sp(x, V);
  // the element of a thread outside of the vectors: in front of them, behind them, or none
  const int at = tid < sp.head ? tid : tid >= W && sp.tail + tid - W < V ? sp.tail + tid - W : -1;
  // vector tid + k THREADS of a row: a uniform address and one offset of the thread, or every vector holds two registers
  const uint32_t off = tid * 16u;
  auto vec = [&](auto* p, int k) {
    return reinterpret_cast<Quad*>(reinterpret_cast<char*>(const_cast<T*>(p) + sp.head) + k * (THREADS * 16) + off);
  };
  if (label < 0) {
    if (tid == 0 && loss) loss[row] = 0.f;
    if (!dlogits) return;
    for (int k = 0; k < NV && tid < sp.vecs - k * THREADS; ++k) __builtin_nontemporal_store(Quad{0u, 0u, 0u, 0u}, vec(g, k));
    if (at >= 0) g[at] = Elt<T>::from_f(0.f);
    return;
  }
  Vec16<T> v[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (tid < sp.vecs - k * THREADS) v[k] = __builtin_bit_cast(Vec16<T>, __builtin_nontemporal_load(vec(x, k)));
  const float extra = at >= 0 ? Elt<T>::to_f(x[at]) : 0.f, xl = label_logit(x, label, V);
  const float w = label >= V ? xl : weight ? weight[row] : 1.f;           // (NaN)
  Stat2 a = Stat2::none();
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (tid < sp.vecs - k * THREADS) {
      float f[W];
#pragma unroll
      for (int e = 0; e < W; ++e) f[e] = Elt<T>::to_f(v[k].v[e]);
      a.add(f);
    }
  }
  if (at >= 0) {
    const float f[1] = {extra};
    a.add(f);
  }
  a = block_join<THREADS>(a, sm);
  if (!(fabsf(a.m) < Stat2::MOST)) {
    Stat b = Stat::none();
#pragma unroll 1
    for (int i = tid; i < V; i += THREADS) {
      const float f[1] = {Elt<T>::to_f(x[i])};
      b.add(f);
    }
    b = block_join<THREADS>(b, sm_far);                      // (no element is written before all have been read)
    const float scale = w / b.s;
    if (tid == 0 && loss) loss[row] = w * (b.m - xl + logf(b.s));
    if (!dlogits) return;
#pragma unroll 1
    for (int i = tid; i < V; i += THREADS)
      g[i] = Elt<T>::from_f(exp_diff(Elt<T>::to_f(x[i]), b.m) * scale - (i == label ? w : 0.f));
    return;
  }
  const float scale = w / a.s;
  // log of the terms' sum without their common factor, to what the label is behind: c itself would round the loss at the logits' size
  if (tid == 0 && loss) loss[row] = w * ((a.m - xl) + (__builtin_amdgcn_logf(a.s) - fmaf(a.m, LOG2E, -a.c)) * LN2);
  if (!dlogits) return;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (tid < sp.vecs - k * THREADS) {
      Vec16<T> f;
#pragma unroll
      for (int e = 0; e < W; ++e) f.v[e] = Elt<T>::from_f(Stat2::term(Elt<T>::to_f(v[k].v[e]), a.c) * scale);
      __builtin_nontemporal_store(__builtin_bit_cast(Quad, f), vec(g, k));
    }
  }
  if (at >= 0) g[at] = Elt<T>::from_f(Stat2::term(extra, a.c) * scale);
  // the label's element again, by the thread that has just written it
  const int in = label - sp.head;
  const bool owner = in < 0 ? tid == label : in / W < sp.vecs ? tid == in / W % THREADS : tid == label - sp.tail + W;
  if (label < V && owner) g[label] = Elt<T>::from_f(Stat2::term(xl, a.c) * scale - w);
}

// ---- host ----------------------------------------------------------------------------------------

// workgroups of a row: enough for four of every CU, with a whole pass of 4 vectors per thread each
int row_parts(int dtype, int T, int V) {
  const int vecs = V / (dtype == BM_DTYPE_BF16 ? 8 : 4);
  const int most = cdiv(vecs, PART_THREADS * 4), want = cdiv(1024, T);
  return std::max(1, std::min(most, want));
}

struct Workspace {
  Stat* stats;
  float* at_label;
  size_t bytes;
  Workspace(void* scratch, int dtype, int T, int V) {
    Arena a(scratch);
    stats = a.take<Stat>((size_t)T * row_parts(dtype, T, V) * sizeof(Stat));
    at_label = a.take<float>((size_t)T * sizeof(float));
    bytes = a.off;
  }
};

constexpr int NUM_CU = 256;

// The kernel for T rows of V words, or -1: parts of rows.  Wide rows have all wavefronts of a CU or half of them; narrower ones fewer
// wavefronts, so that several share a CU, once there are rows enough for that.  Measured with bf16 words (us):
//   1024 x 16000: 512x8 12.1, 256x16 13.6, 1024x4 15.6; 256 rows: 512x8 6.3, 1024x4 5.9     4096 x 4000: 256x4 14.9, 512x8 18.1
//   1024 x 64000: 1024x8 47.4, 512x16 48.7     4096 x 1500: 64x4 8.1, 256x4 10.9
//   x 128000: 1 row 9.6 in 16 parts, 15.5 in registers; 48 rows 14.8 and 16.7, 128 rows 26.4 and 17.4, 4096 rows 618 and 389
int row_plan(int dtype, int T, int V) {
  const int vecs = V / (dtype == BM_DTYPE_BF16 ? 8 : 4);
  if (vecs <= 64 * 4) return 0;
  if (vecs <= 256 * 4) return 1;
  if (vecs <= 512 * 8) return T <= 2 * NUM_CU ? 3 : 2;
  if (vecs <= 1024 * 8) return 4;
  return vecs > 1024 * 24 || T <= 32 ? -1 : 5;
}

template <typename T>
bm_status run_rows(int plan, int n, int V, const T* logits, int ld, const int32_t* labels, const float* weight, float* loss,
                   T* dlogits, int ld_d, hipStream_t st) {
  constexpr decltype(&row_kernel<T, 64, 4>) kernels[] = {row_kernel<T, 64, 4>,   row_kernel<T, 256, 4>,  row_kernel<T, 512, 8>,
                                                         row_kernel<T, 1024, 4>, row_kernel<T, 1024, 8>, row_kernel<T, 1024, 24>};
  constexpr int threads[] = {64, 256, 512, 1024, 1024, 1024};
  hipLaunchKernelGGL(kernels[plan], dim3(n), dim3(threads[plan]), 0, st, logits, (long)ld, labels, weight, V, loss, dlogits, (long)ld_d);
  BM_CHECK_LAUNCH("cross entropy rows");
  return BM_OK;
}

template <typename T>
bm_status run(int dtype, int n, int V, const void* logits, int ld, const int32_t* labels, const float* weight, float* loss,
              void* dlogits, int ld_d, const Workspace& w, hipStream_t st) {
  const int plan = row_plan(dtype, n, V);
  if (plan >= 0 && (!dlogits || (size_t)std::abs(ld - ld_d) * sizeof(T) % 16 == 0))
    return run_rows<T>(plan, n, V, (const T*)logits, ld, labels, weight, loss, (T*)dlogits, ld_d, st);
  const int parts = row_parts(dtype, n, V);
  hipLaunchKernelGGL(part_stats_kernel<T>, dim3((unsigned)((long)n * parts)), dim3(PART_THREADS), 0, st, (const T*)logits, (long)ld,
                     labels, V, parts, w.stats, w.at_label);
  BM_CHECK_LAUNCH("cross entropy statistics");
  const int writes = dlogits ? parts : 0;
  hipLaunchKernelGGL(part_finish_kernel<T>, dim3((unsigned)((long)n * std::max(1, writes))), dim3(PART_THREADS), 0, st,
                     (const T*)logits, (long)ld, labels, weight, V, parts, writes, w.stats, w.at_label, loss, (T*)dlogits, (long)ld_d);
  BM_CHECK_LAUNCH("cross entropy gradient");
  return BM_OK;
}

}  // namespace
}  // namespace bm

using namespace bm;

extern "C" size_t bm_cross_entropy_scratch_bytes(int32_t dtype, int32_t T, int32_t V) {
  if (!good_dtype(dtype) || T <= 0 || V <= 0) return 0;
  return Workspace(nullptr, dtype, T, V).bytes;
}

extern "C" bm_status bm_cross_entropy(int32_t dtype, int32_t T, int32_t V, const void* logits, int32_t ld, const int32_t* labels,
                                      const float* weight, float* loss, void* dlogits, int32_t ld_d, void* scratch,
                                      size_t scratch_bytes, void* hip_stream) {
  BM_ARG_CHECK(good_dtype(dtype), "bm_cross_entropy: dtype %d", dtype);
  BM_ARG_CHECK(T >= 0 && V > 0, "bm_cross_entropy: bad sizes");
  BM_ARG_CHECK(ld >= V && (!dlogits || ld_d >= V), "bm_cross_entropy: leading dimension too small");
  BM_ARG_CHECK(V < INT32_MAX - 4096, "bm_cross_entropy: %d words are too many", V);
  BM_ARG_CHECK(dlogits != logits || ld_d == ld, "bm_cross_entropy: a gradient in place of the logits has their row stride");
  if (T == 0) return BM_OK;
  BM_ARG_CHECK(logits && labels && (loss || dlogits), "bm_cross_entropy: NULL tensor");
  BM_ARG_CHECK(aligned16(logits) && aligned16(labels) && aligned16(weight) && aligned16(loss) && aligned16(dlogits) && aligned16(scratch),
               "bm_cross_entropy: misaligned tensor");
  const Workspace w(scratch, dtype, T, V);
  if (w.bytes && (!scratch || scratch_bytes < w.bytes)) {
    set_error("bm_cross_entropy needs %zu scratch bytes, got %zu", w.bytes, scratch_bytes);
    return BM_ERR_WORKSPACE_TOO_SMALL;
  }
  hipStream_t st = (hipStream_t)hip_stream;
  ProfScope prof(PROF_ELEMENTWISE, (dlogits ? 2.0 : 1.0) * T * V * elt_size(dtype), st);
  // (a grid has fewer than 2^32 threads; what is left of the rows has no more parts than all of them together)
  constexpr int MOST = 1 << 21;
  const size_t elt = elt_size(dtype);
  for (int first = 0; first < T; first += std::min(MOST, T - first)) {
    const int n = std::min(MOST, T - first);
    const void* x = (const char*)logits + (size_t)first * ld * elt;
    void* g = dlogits ? (char*)dlogits + (size_t)first * ld_d * elt : nullptr;
    const float* f = weight ? weight + first : nullptr;
    float* l = loss ? loss + first : nullptr;
    BM_RETURN_IF(dtype == BM_DTYPE_BF16 ? run<bf16_t>(dtype, n, V, x, ld, labels + first, f, l, g, ld_d, w, st)
                                        : run<float>(dtype, n, V, x, ld, labels + first, f, l, g, ld_d, w, st));
  }
  return BM_OK;
}
