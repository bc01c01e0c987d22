// Cross-entropy of a vocabulary and its gradient: with m the largest logit of a row and s the sum of exp(z - m),
//   loss = w (m + log s - z[label]),   dz = w (exp(z - m) / s - onehot(label)).
// m and s come from one pass: a thread rescales its sum when its maximum grows, and pairs (m, s) are joined.
// A row whose label is negative is never read.  Bound by HBM.
//
// Two launches: parts of rows leave their (m, s), then every part of a row joins those of the whole row and writes its
// gradient.  The second read of the logits comes from the memory-side cache where they fit.
#include "train.h"

#include <float.h>

#include <algorithm>

namespace bm {

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

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
#pragma unroll
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

template <typename T>
bm_status run(int dtype, int n, int V, const void* logits, int ld, const int32_t* labels, const float* weight, float* loss,
              void* dlogits, int ld_d, const Workspace& w, hipStream_t st) {
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
  return dtype == BM_DTYPE_BF16 ? run<bf16_t>(dtype, T, V, logits, ld, labels, weight, loss, dlogits, ld_d, w, st)
                                : run<float>(dtype, T, V, logits, ld, labels, weight, loss, dlogits, ld_d, w, st);
}
