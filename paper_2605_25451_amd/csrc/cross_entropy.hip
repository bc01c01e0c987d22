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

// The same statistics with an instruction less per element: exp(x - m) as 2^(x L - c), c = m L rounded once, which is a
// common factor of all terms.  c is kept inside fp32's range, which makes rows whose largest logit is past 1e38 in
// magnitude wrong (a row of nothing but the lowest finite value, say); those are done again with the difference first.
struct Stat2 {
  float m, c, s;
  static __device__ inline float bound(float m) { return __builtin_amdgcn_fmed3f(m * LOG2E, -3e38f, 3e38f); }
  static __device__ inline Stat2 none() { return Stat2{-FLT_MAX, -3e38f, 0.f}; }
  static __device__ inline float term(float x, float c) { return __builtin_amdgcn_exp2f(fmaf(x, LOG2E, -c)); }
  template <int N> __device__ inline void add(const float (&x)[N]) {
    float top = m;
#pragma unroll
    for (int e = 0; e < N; ++e) top = fmaxf(top, x[e]);
    const float c1 = bound(top);
    s *= __builtin_amdgcn_exp2f(c - c1);
#pragma unroll
    for (int e = 0; e < N; ++e) s += term(x[e], c1);
    m = top;
    c = c1;
  }
};
template <int THREADS>
__device__ inline Stat2 block_join(Stat2 a, Stat2* sm) {
  const float m = wave_max(a.m), c = Stat2::bound(m);
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
  const float c1 = Stat2::bound(top);
  r.s *= __builtin_amdgcn_exp2f(r.c - c1);
#pragma unroll
  for (int off = 1; off < WAVES; off <<= 1) r.s += __shfl_xor(r.s, off, WAVE);
  r.m = top;
  r.c = c1;
  return r;
}

// The rows of a workgroup where there are more rows than workgroups: of LIST rows each, those that are read are dealt out one by one,
// then those that are ignored, so that all have as much to do wherever the ignored ones stand (30 % of them at random, 16 rows per
// workgroup: the busiest would read 16, now all read 11 or 12).
constexpr int LIST = 64;
template <int THREADS>
struct RowList {
  int live[THREADS / WAVE], row[LIST];
  // rows first .. end - 1, shares of them in a grid of 2^log_grid; how many there are for this workgroup
  __device__ inline int fill(const int32_t* __restrict__ labels, int first, int end, int log_grid) {
    constexpr int WAVES = THREADS / WAVE;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per = (end - first + WAVES * WAVE - 1) / (WAVES * WAVE) * WAVE;
    const int from = min(end, first + wave * per), to = min(end, from + per);
    int count = 0;
    for (int i = from + lane; i - lane < to; i += WAVE) count += __popcll(__ballot(i < to && labels[i] >= 0));
    __syncthreads();                                         // the list is no longer read
    if (lane == 0) live[wave] = count;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll 1
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) before += live[w];
      all += live[w];
    }
    const int grid = 1 << log_grid, me = blockIdx.x;
    int rest = all + from - first - before;
    for (int i = from + lane; i - lane < to; i += WAVE) {
      const bool in = i < to, is = in && labels[i] >= 0;
      const uint64_t m = __ballot(is), r = __ballot(in && !is), lower = (1ull << lane) - 1;
      const int rank = is ? before + __popcll(m & lower) : rest + __popcll(r & lower);
      if (in && (rank & (grid - 1)) == me) row[rank >> log_grid] = i;
      before += __popcll(m);
      rest += __popcll(r);
    }
    __syncthreads();
    return (end - first - me + grid - 1) >> log_grid;
  }
};

// A workgroup holds a row in its registers, NV vectors per thread, so that the logits are read once; while it writes a row's
// gradient, every register that has been used is filled from the next row, so that memory is never idle for the
// exponentials.  Rows of logits and gradient start at the same place between two 16-byte boundaries.
template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void row_kernel(const T* logits, long ld, const int32_t* __restrict__ labels,
                                                      const float* __restrict__ weight, int V, int rows, int log_grid,
                                                      float* __restrict__ loss, T* dlogits, long ld_d) {
  constexpr int W = Span<T>::W;
  __shared__ RowList<THREADS> list;
  __shared__ Stat2 sm[THREADS / WAVE];
  __shared__ Stat sm_far[THREADS / WAVE];
  Vec16<T> v[NV];
  const int tid = threadIdx.x;
  // the element of a thread outside of the vectors: in front of them, behind them, or none
  auto loose = [&](const Span<T>& sp) { return tid < sp.head ? tid : tid >= W && sp.tail + tid - W < V ? sp.tail + tid - W : -1; };
  float extra = 0.f;
  // vector tid + k THREADS of a row: a uniform address and one offset of the thread, or every vector holds two registers
  const uint32_t off = tid * 16u;
  auto fetch = [&](const T* x, const Span<T>& sp, int k) {
    if (tid < sp.vecs - k * THREADS)
      v[k] = *reinterpret_cast<const Vec16<T>*>(reinterpret_cast<const char*>(x + sp.head) + k * (THREADS * 16) + off);
  };
  // log_grid < 0: a row for every workgroup
  long segment = 0;
  int items = 1, item = 0, row = blockIdx.x;
  if (log_grid >= 0) {
    items = list.fill(labels, 0, min(rows, LIST << log_grid), log_grid);
    row = __builtin_amdgcn_readfirstlane(list.row[0]);        // (rows are not fewer than workgroups)
  }
  int label = labels[row];
  const T* x = logits + (size_t)row * ld;
  Span<T> sp(x, V);
  auto whole = [&] {
    const int at = loose(sp);
    if (at >= 0) extra = Elt<T>::to_f(x[at]);
#pragma unroll
    for (int k = 0; k < NV; ++k) fetch(x, sp, k);
  };
  if (label >= 0) whole();
  for (;;) {
    const bool more = item + 1 < items;
    const int next = more ? log_grid < 0 ? 0 : __builtin_amdgcn_readfirstlane(list.row[item + 1]) : 0;
    const int next_label = more ? labels[next] : -1;
    const int at = loose(sp);
    Stat2 a = Stat2::none();
    float scale = 0.f, w = 0.f, p_label = 0.f;
    bool far = false;
    if (label >= 0) {
      const float xl = label_logit(x, label, V);
      w = weight ? weight[row] : 1.f;
      if (label >= V) w = xl;                               // NaN
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
      far = !(fabsf(a.m) <= 1e38f);
      float nll = (a.c + __builtin_amdgcn_logf(a.s)) * LN2 - xl;
      if (far) {
        Stat b = Stat::none();
#pragma unroll 1
        for (int i = tid; i < V; i += THREADS) {
          const float f[1] = {Elt<T>::to_f(x[i])};
          b.add(f);
        }
        b = block_join<THREADS>(b, sm_far);                 // (no element is written before all have been read)
        a.m = b.m;
        a.s = b.s;
        nll = b.m - xl + logf(b.s);
      }
      scale = w / a.s;
      p_label = (far ? exp_diff(xl, a.m) : Stat2::term(xl, a.c)) * scale - w;
      if (tid == 0 && loss) loss[row] = w * nll;
    } else if (tid == 0 && loss) {
      loss[row] = 0.f;
    }
    const T* xn = logits + (size_t)(more ? next : row) * ld;
    const Span<T> spn(xn, V);
    T* g = dlogits + (size_t)row * ld_d;
    const bool writes = dlogits && !far;
    if (dlogits && far) {
#pragma unroll 1
      for (int i = tid; i < V; i += THREADS)
        g[i] = Elt<T>::from_f(i == label ? p_label : exp_diff(Elt<T>::to_f(x[i]), a.m) * scale);
    }
    auto gradient = [&](float z) { return label < 0 ? 0.f : Stat2::term(z, a.c) * scale; };
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (writes && tid < sp.vecs - k * THREADS) {
        float f[W];
#pragma unroll
        for (int e = 0; e < W; ++e) f[e] = gradient(Elt<T>::to_f(v[k].v[e]));
        store16(reinterpret_cast<T*>(reinterpret_cast<char*>(g + sp.head) + k * (THREADS * 16) + off), f);
      }
      if (next_label >= 0) fetch(xn, spn, k);
    }
    if (writes) {
      if (at >= 0) g[at] = Elt<T>::from_f(gradient(extra));
      // the label's element again, by the thread that has just written it
      const int in = label - sp.head;
      const bool owner = in < 0 ? tid == label : in / W < sp.vecs ? tid == in / W % THREADS : tid == label - sp.tail + W;
      if (label >= 0 && label < V && owner) g[label] = Elt<T>::from_f(p_label);
    }
    if (!more) {
      // the next rows, if there are any
      segment += (long)LIST << max(log_grid, 0);
      if (log_grid < 0 || segment >= rows) break;
      items = list.fill(labels, (int)segment, (int)min((long)rows, segment + (LIST << log_grid)), log_grid);
      if (items == 0) break;                                // (only at the last of the rows)
      item = 0;
      row = __builtin_amdgcn_readfirstlane(list.row[0]);
      label = labels[row];
      x = logits + (size_t)row * ld;
      sp = Span<T>(x, V);
      if (label >= 0) whole();
      continue;
    }
    ++item;
    row = next; label = next_label; x = xn; sp = spn;
    if (label >= 0) {
      const int to = loose(sp);
      if (to >= 0) extra = Elt<T>::to_f(x[to]);
    }
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

// threads and vectors per thread of a row that stays in registers; workgroups that a CU holds
struct RowPlan { int threads, vectors, per_cu; };
constexpr RowPlan ROW_PLANS[] = {{64, 4, 32}, {256, 4, 8}, {256, 16, 4}, {512, 16, 2}, {1024, 16, 1}, {1024, 20, 1}, {1024, 4, 2}, {1024, 8, 1}};
constexpr int NUM_CU = 256;

// The plan for rows of V words, or -1: parts of rows.  Measured with T rows of V bf16 words (us):
//   few rows       more threads per row: 1 x 32000 256x16 10.5, 512x16 8.5, 1024x4 7.3; 256 rows 14.7, 12.3, 11.4
//   many rows      more rows per CU: 1024 x 32000 256x16 31.2, 512x16 36.3, 1024x4 39.5; 4096 rows 133, 138, 145
//   between them   the one whose last round is full: 512 x 32000 20.8, 18.5, 21.9; 700 x 64000 512x16 56.8, 1024x8 54.5
//   wide rows      one fills a CU: 1 x 128000 18.7 against 9.3 of 16 parts, 128 rows 25.5 and 26.2, 256 33 and 45, 300 66 and 52,
//                  400 69 and 65, 512 66 and 85
int row_plan(int dtype, int T, int V) {
  const int vecs = V / (dtype == BM_DTYPE_BF16 ? 8 : 4);
  if (vecs <= 64 * 4) return 0;
  if (vecs <= 256 * 4) return 1;
  if (vecs <= 1024 * 4) return T <= NUM_CU ? 6 : T <= 2 * NUM_CU ? 3 : 2;
  if (vecs <= 1024 * 8) return T < NUM_CU / 4 ? -1 : T <= NUM_CU || (T > 2 * NUM_CU && T <= 3 * NUM_CU) ? 7 : 3;
  if (vecs > 1024 * 20 || T < NUM_CU / 2 || (T > NUM_CU && T <= NUM_CU * 3 / 2)) return -1;
  return vecs <= 1024 * 16 ? 4 : 5;
}

template <typename T, int THREADS, int NV>
bm_status launch_rows(int n, int per_cu, const T* logits, int ld, const int32_t* labels, const float* weight, int V, float* loss,
                      T* dlogits, int ld_d, hipStream_t st) {
  const bool one_each = n <= NUM_CU * per_cu;
  int log_grid = -1;
  if (!one_each)
    for (log_grid = 0; (1 << log_grid) < NUM_CU * per_cu;) ++log_grid;
  hipLaunchKernelGGL((row_kernel<T, THREADS, NV>), dim3(one_each ? n : 1 << log_grid), dim3(THREADS), 0, st, logits, (long)ld, labels,
                     weight, V, n, log_grid, loss, dlogits, (long)ld_d);
  BM_CHECK_LAUNCH("cross entropy rows");
  return BM_OK;
}

template <typename T>
bm_status run_rows(int plan, int n, int V, const T* logits, int ld, const int32_t* labels, const float* weight, float* loss,
                   T* dlogits, int ld_d, hipStream_t st) {
  const int per = ROW_PLANS[plan].per_cu;
  switch (plan) {
    case 0: return launch_rows<T, 64, 4>(n, per, logits, ld, labels, weight, V, loss, dlogits, ld_d, st);
    case 1: return launch_rows<T, 256, 4>(n, per, logits, ld, labels, weight, V, loss, dlogits, ld_d, st);
    case 2: return launch_rows<T, 256, 16>(n, per, logits, ld, labels, weight, V, loss, dlogits, ld_d, st);
    case 3: return launch_rows<T, 512, 16>(n, per, logits, ld, labels, weight, V, loss, dlogits, ld_d, st);
    case 4: return launch_rows<T, 1024, 16>(n, per, logits, ld, labels, weight, V, loss, dlogits, ld_d, st);
    case 6: return launch_rows<T, 1024, 4>(n, per, logits, ld, labels, weight, V, loss, dlogits, ld_d, st);
    case 7: return launch_rows<T, 1024, 8>(n, per, logits, ld, labels, weight, V, loss, dlogits, ld_d, st);
    default: return launch_rows<T, 1024, 20>(n, per, logits, ld, labels, weight, V, loss, dlogits, ld_d, st);
  }
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
  return dtype == BM_DTYPE_BF16 ? run<bf16_t>(dtype, T, V, logits, ld, labels, weight, loss, dlogits, ld_d, w, st)
                                : run<float>(dtype, T, V, logits, ld, labels, weight, loss, dlogits, ld_d, w, st);
}
