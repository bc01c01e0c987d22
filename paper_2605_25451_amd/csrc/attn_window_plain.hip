// Attention with a sliding window and first tokens in fp32 arithmetic (fp32 storage, and bf16 at head sizes 8, 16 and 32): forward and
// gradient on v_mfma_f32_16x16x4_f32.
//
// A workgroup owns 16 queries of a head (o, dq) or 16 keys of a kv head (dk, dv), in columns: S^T = K Q^T, O^T = V^T P^T; its four
// wavefronts take every fourth tile of 16 rows of the other side and meet in LDS at the end, in a fixed order.
// The order of a contraction is free, so a lane reads whole runs of a row:
//   operands along the head: lane (g = l / 16, c = l % 16) holds elements g dh/4 .. + dh/4 of row c, one for each of dh/4 MFMAs
//   operands along the other side's rows: row g * 4 + i, elements c n .. + n (n = dh/16, rounded up) for MFMA i
//   accumulators: element r of a lane is row g * 4 + r, which is where the next product wants its i = r
// so probabilities go from one product to the next in their registers, and nothing passes through LDS before the end.
// Bound by the latency of its loads and dependent MFMAs on short documents, by L2 on long ones (a wavefront's 16 rows are 8 flop a byte: 16 / 16
// heads of 64, 2 documents in 1500 tokens, 43 us, 32 / 8 of 128 165 us, 64 TFLOP/s; gradients 153 and 746).  Against a lane for every eighth of a
// row, products in the vector unit: 700 tokens, window 100, 4 heads of 64, 26.7 -> 10.7 us; gradients of 592 tokens, 12 heads of 64, 183 -> 38,
// of 127 tokens, 32 heads of 128, 305 -> 30.
#include "attn_window.h"

#include <algorithm>

namespace bm {

namespace {

using f32x4 = __attribute__((__vector_size__(4 * sizeof(float)))) float;

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr int ROWS = 16;                                   // of a tile, on either side

struct PlainArgs {
  const void *q, *k, *v, *d_o;
  void *o, *dq, *dk, *dv;
  float *lse_out;
  const float *lse, *delta;
  const int32_t *cu, *cuk;
  int ld, ldk, ldo, ldd, ldd_kv, S, Ttot, Hq, Hkv, kv_wgs;
  float scale;
  LocalMask w;
};

constexpr int low_bit(int n) { return n & -n; }
// N elements that start a multiple of N from a 16-byte boundary
template <int N, typename T>
__device__ inline void load_run(const T* p, float (&x)[N]) {
  constexpr int A = low_bit(N * (int)sizeof(T)), BYTES = A < 16 ? A : 16, E = BYTES / (int)sizeof(T);
  struct alignas(BYTES) Part { T v[E]; };
#pragma unroll
  for (int i = 0; i < N; i += E) {
    const Part t = *reinterpret_cast<const Part*>(p + i);
#pragma unroll
    for (int e = 0; e < E; ++e) x[i + e] = Elt<T>::to_f(t.v[e]);
  }
}
template <int DH> constexpr int cols_of() { return (DH + 15) / 16; }
// this lane's elements c n .. + n of a row; past the row's end (head sizes 8 and 72) its last ones, whose results are left out
template <int DH, typename T>
__device__ inline void load_cols(const T* row, int c, float (&x)[cols_of<DH>()]) {
  constexpr int N = cols_of<DH>();
  if constexpr (DH % 16 == 0) {
    load_run<N>(row + c * N, x);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = Elt<T>::to_f(row[min(c * N + j, DH - 1)]);
  }
}
template <int DH>
__device__ inline f32x4 product(const float (&a)[DH / 4], const float (&b)[DH / 4]) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < DH / 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], s, 0, 0, 0);
  return s;
}
__device__ inline float groups_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}
__device__ inline float groups_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
// what the wavefronts have summed of a tile: [wavefront][column][element of the head]
template <int DH> struct Sums { float x[4][ROWS][cols_of<DH>() * 16 + 4]; };
template <int DH>
__device__ inline void leave(Sums<DH>& s, int wave, int g, int c, const f32x4 (&acc)[cols_of<DH>()]) {
  constexpr int N = cols_of<DH>();
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int j = 0; j < N; ++j) s.x[wave][c][(g * 4 + r) * N + j] = acc[j][r];
}

template <typename T, int DH>
__global__ __launch_bounds__(256) void window_plain_fwd_kernel(PlainArgs a) {
  constexpr int N = cols_of<DH>();
  __shared__ Sums<DH> sums;
  __shared__ float stats[4][ROWS][2];
  const int hq = blockIdx.x % a.Hq, hk = hq / (a.Hq / a.Hkv);
  int seq, qt, nqt;
  if (!find_tile_by_lanes(a.cu, a.cu + 1, a.S, ROWS, blockIdx.x / a.Hq, &seq, &qt, &nqt)) return;
  const int lo = a.cu[seq], L = a.cu[seq + 1] - lo, lok = a.cuk[seq], Lk = a.w.key_end[seq] - lok, off = Lk - L, q0 = qt * ROWS;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int at = off + q0 + c, begin = window_begin(a.w, off + q0);
  const KeyWalk<ROWS> walk(a.w, off, q0, ROWS, Lk);
  const T* kb = (const T*)a.k + (size_t)lok * a.ldk + hk * DH;
  const T* vb = (const T*)a.v + (size_t)lok * a.ldk + hk * DH;
  auto row_of = [&](int key) { return (size_t)min(seen_row(a.w, begin, key), Lk - 1) * a.ldk; };
  float qf[DH / 4];
  load_run<DH / 4>((const T*)a.q + (size_t)(lo + min(q0 + c, L - 1)) * a.ld + hq * DH + g * (DH / 4), qf);
#pragma unroll
  for (int i = 0; i < DH / 4; ++i) qf[i] *= a.scale * LOG2E;
  f32x4 acc[N] = {};
  float m = NO_MAX, l = 0.f, kf[DH / 4];
  auto fetch = [&](int t) {
    if (t < walk.n) load_run<DH / 4>(kb + row_of(walk.tile(t) * ROWS + c) + g * (DH / 4), kf);
  };
  fetch(wave);
  for (int t = wave; t < walk.n; t += 4) {
    const int key0 = walk.tile(t) * ROWS;
    float vc[4][N];
#pragma unroll
    for (int i = 0; i < 4; ++i) load_cols<DH>(vb + row_of(key0 + g * 4 + i), c, vc[i]);
    f32x4 s = product<DH>(kf, qf);
    fetch(t + 4);
    const bool masked = key0 + ROWS - 1 > off + q0 || (off + q0 + ROWS - 1 - key0 >= a.w.window && key0 + ROWS > a.w.sinks);
    if (masked)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (hidden(a.w, key0 + g * 4 + r, at)) s[r] = -INFINITY;
    const float mn = fmaxf(m, groups_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])))), corr = exp2f(m - mn);
    m = mn;
    l *= corr;
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] *= corr;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = exp2f(s[i] - mn);
      l += p;
#pragma unroll
      for (int j = 0; j < N; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vc[i][j], p, acc[j], 0, 0, 0);
    }
  }
  l = groups_sum(l);
  leave<DH>(sums, wave, g, c, acc);
  if (g == 0) { stats[wave][c][0] = m; stats[wave][c][1] = l; }
  __syncthreads();
  for (int e = threadIdx.x; e < min(ROWS, L - q0) * DH; e += 256) {
    const int r = e / DH, d = e % DH;
    float top = NO_MAX;
#pragma unroll
    for (int x = 0; x < 4; ++x) top = fmaxf(top, stats[x][r][0]);
    float sum = 0.f, val = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float f = exp2f(stats[x][r][0] - top);
      sum = fmaf(f, stats[x][r][1], sum);
      val = fmaf(f, sums.x[x][r][d], val);
    }
    ((T*)a.o)[(size_t)(lo + q0 + r) * a.ldo + hq * DH + d] = Elt<T>::from_f(val / sum);
    if (d == 0) a.lse_out[(size_t)hq * a.Ttot + lo + q0 + r] = (top + log2f(sum)) * LN2;
  }
}

// delta = rowsum(dO o): 16 lanes for each token and head
template <typename T>
__global__ __launch_bounds__(256) void window_plain_delta_kernel(const T* __restrict__ o, const T* __restrict__ d_o, int ldo, int dh, float* __restrict__ delta,
                                                                 int Ttot, int Hq) {
  const long row = (long)blockIdx.x * 16 + threadIdx.x / 16;
  const bool live = row < (long)Ttot * Hq;
  const int t = live ? (int)(row / Hq) : 0, h = live ? (int)(row % Hq) : 0;
  const size_t at = (size_t)t * ldo + h * dh;
  float s = 0.f;
  for (int i = threadIdx.x % 16; i < dh; i += 16) s = fmaf(Elt<T>::to_f(o[at + i]), Elt<T>::to_f(d_o[at + i]), s);
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) s += __shfl_xor(s, d, 64);
  if (live && threadIdx.x % 16 == 0) delta[(size_t)h * Ttot + t] = s;
}

// the wavefronts' sums of a tile, times f, in bf16 or fp32
template <typename T, int DH>
__device__ inline void write_sums(Sums<DH>& sums, int wave, int g, int c, const f32x4 (&acc)[cols_of<DH>()], float f, T* out, int ld, int rows) {
  leave<DH>(sums, wave, g, c, acc);
  __syncthreads();
  for (int e = threadIdx.x; e < rows * DH; e += 256) {
    const int r = e / DH, d = e % DH;
    out[(size_t)r * ld + d] = Elt<T>::from_f((((sums.x[0][r][d] + sums.x[1][r][d]) + sums.x[2][r][d]) + sums.x[3][r][d]) * f);
  }
}

// dk and dv of 16 keys: the q heads of the group and the tiles of queries that see one of the keys
template <typename T, int DH>
__device__ inline void plain_dkdv(const PlainArgs& a, Sums<DH>& sums, int block) {
  constexpr int N = cols_of<DH>();
  const int hk = block % a.Hkv, group = a.Hq / a.Hkv;
  int seq, kt, nkt;
  if (!find_tile_by_lanes(a.cuk, a.w.key_end, a.S, ROWS, block / a.Hkv, &seq, &kt, &nkt)) return;
  kt = nkt - 1 - kt;                                       // the first tokens' tiles run longest
  const int lo = a.cu[seq], L = a.cu[seq + 1] - lo, lok = a.cuk[seq], Lk = a.w.key_end[seq] - lok, off = Lk - L, kb0 = kt * ROWS;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int key = kb0 + c;
  const int qlo = max(0, kb0 - off), qhi = kb0 < a.w.sinks ? L : min(L, kb0 + ROWS - 1 - off + a.w.window);
  const int nq = qhi > qlo ? (qhi - qlo + ROWS - 1) / ROWS : 0;
  float kf[DH / 4], vf[DH / 4];
  {
    const size_t at = (size_t)(lok + min(key, Lk - 1)) * a.ldk + hk * DH + g * (DH / 4);
    load_run<DH / 4>((const T*)a.k + at, kf);
    load_run<DH / 4>((const T*)a.v + at, vf);
#pragma unroll
    for (int i = 0; i < DH / 4; ++i) kf[i] *= a.scale * LOG2E;
  }
  f32x4 dk[N] = {}, dv[N] = {};
  for (int it = wave; it < nq * group; it += 4) {
    const int hq = hk * group + it / nq, q0 = qlo + it % nq * ROWS;
    const T* qb = (const T*)a.q + (size_t)lo * a.ld + hq * DH;
    const T* db = (const T*)a.d_o + (size_t)lo * a.ldo + hq * DH;
    float qa[DH / 4], da[DH / 4], lse[4], delta[4], qc[4][N], dc[4][N];
    const int row = min(q0 + c, L - 1);
    load_run<DH / 4>(qb + (size_t)row * a.ld + g * (DH / 4), qa);
    load_run<DH / 4>(db + (size_t)row * a.ldo + g * (DH / 4), da);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = min(q0 + g * 4 + i, L - 1);
      lse[i] = a.lse[(size_t)hq * a.Ttot + lo + r] * LOG2E;
      delta[i] = a.delta[(size_t)hq * a.Ttot + lo + r];
      load_cols<DH>(qb + (size_t)r * a.ld, c, qc[i]);
      load_cols<DH>(db + (size_t)r * a.ldo, c, dc[i]);
    }
    const f32x4 s = product<DH>(qa, kf), dp = product<DH>(da, vf);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int qi = q0 + g * 4 + i;
      const bool seen = qi < qhi && key < Lk && !hidden(a.w, key, off + qi);
      const float p = seen ? exp2f(s[i] - lse[i]) : 0.f, ds = p * (dp[i] - delta[i]);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        dv[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(dc[i][j], p, dv[j], 0, 0, 0);
        dk[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(qc[i][j], ds, dk[j], 0, 0, 0);
      }
    }
  }
  const size_t out = (size_t)(lok + kb0) * a.ldd_kv + hk * DH;
  const int rows = min(ROWS, Lk - kb0);
  write_sums<T, DH>(sums, wave, g, c, dv, 1.0f, (T*)a.dv + out, a.ldd_kv, rows);
  __syncthreads();
  write_sums<T, DH>(sums, wave, g, c, dk, a.scale, (T*)a.dk + out, a.ldd_kv, rows);
}

template <typename T, int DH>
__device__ inline void plain_dq(const PlainArgs& a, Sums<DH>& sums, int block) {
  constexpr int N = cols_of<DH>();
  const int hq = block % a.Hq, hk = hq / (a.Hq / a.Hkv);
  int seq, qt, nqt;
  if (!find_tile_by_lanes(a.cu, a.cu + 1, a.S, ROWS, block / a.Hq, &seq, &qt, &nqt)) return;
  const int lo = a.cu[seq], L = a.cu[seq + 1] - lo, lok = a.cuk[seq], Lk = a.w.key_end[seq] - lok, off = Lk - L, q0 = qt * ROWS;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int at = off + q0 + c;
  const KeyWalk<ROWS> walk(a.w, off, q0, ROWS, Lk);
  const T* kb = (const T*)a.k + (size_t)lok * a.ldk + hk * DH;
  const T* vb = (const T*)a.v + (size_t)lok * a.ldk + hk * DH;
  float qf[DH / 4], df[DH / 4];
  const int row = lo + min(q0 + c, L - 1);
  load_run<DH / 4>((const T*)a.q + (size_t)row * a.ld + hq * DH + g * (DH / 4), qf);
  load_run<DH / 4>((const T*)a.d_o + (size_t)row * a.ldo + hq * DH + g * (DH / 4), df);
  const float lse = a.lse[(size_t)hq * a.Ttot + row] * LOG2E, delta = a.delta[(size_t)hq * a.Ttot + row];
#pragma unroll
  for (int i = 0; i < DH / 4; ++i) qf[i] *= a.scale * LOG2E;
  f32x4 dq[N] = {};
  for (int t = wave; t < walk.n; t += 4) {
    const int key0 = walk.tile(t) * ROWS;
    float kf[DH / 4], vf[DH / 4], kc[4][N];
    const size_t from = (size_t)min(key0 + c, Lk - 1) * a.ldk + g * (DH / 4);
    load_run<DH / 4>(kb + from, kf);
    load_run<DH / 4>(vb + from, vf);
#pragma unroll
    for (int i = 0; i < 4; ++i) load_cols<DH>(kb + (size_t)min(key0 + g * 4 + i, Lk - 1) * a.ldk, c, kc[i]);
    const f32x4 s = product<DH>(kf, qf), dp = product<DH>(vf, df);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = hidden(a.w, key0 + g * 4 + i, at) ? 0.f : exp2f(s[i] - lse), ds = p * (dp[i] - delta);
#pragma unroll
      for (int j = 0; j < N; ++j) dq[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(kc[i][j], ds, dq[j], 0, 0, 0);
    }
  }
  write_sums<T, DH>(sums, wave, g, c, dq, a.scale, (T*)a.dq + (size_t)(lo + q0) * a.ldd + hq * DH, a.ldd, min(ROWS, L - q0));
}

template <typename T, int DH>
__global__ __launch_bounds__(256) void window_plain_bwd_kernel(PlainArgs a) {
  __shared__ Sums<DH> sums;
  if ((int)blockIdx.x < a.kv_wgs) plain_dkdv<T, DH>(a, sums, blockIdx.x);
  else plain_dq<T, DH>(a, sums, blockIdx.x - a.kv_wgs);
}

long tiles_of(const int32_t* begin, const int32_t* end, int S) {
  long n = 0;
  for (int s = 0; s < S; ++s) n += cdiv(end[s] - begin[s], ROWS);
  return n;
}

PlainArgs plain_args(const AttnArgs& a) {
  PlainArgs p{};
  p.q = a.q; p.k = a.k; p.v = a.v;
  p.cu = a.cu_dev; p.cuk = a.kv_cu_dev();
  p.ld = a.ld_qkv; p.ldk = a.kv_ld(); p.ldo = a.Hq * a.dh;
  p.S = a.S; p.Ttot = a.T; p.Hq = a.Hq; p.Hkv = a.Hkv;
  p.scale = 1.0f / sqrtf((float)a.dh);
  p.w = a.local;
  return p;
}

// bf16 comes here with head sizes 8, 16 and 32 only
#define BM_PLAIN_SWITCH(KERNEL)                                              \
  if (a.dtype == BM_DTYPE_BF16) {                                            \
    switch (a.dh) {                                                          \
      case 8: go(KERNEL<bf16_t, 8>); break;                                  \
      case 16: go(KERNEL<bf16_t, 16>); break;                                \
      default: go(KERNEL<bf16_t, 32>);                                       \
    }                                                                        \
  } else {                                                                   \
    switch (a.dh) {                                                          \
      case 8: go(KERNEL<float, 8>); break;                                   \
      case 16: go(KERNEL<float, 16>); break;                                 \
      case 32: go(KERNEL<float, 32>); break;                                 \
      case 64: go(KERNEL<float, 64>); break;                                 \
      case 72: go(KERNEL<float, 72>); break;                                 \
      default: go(KERNEL<float, 128>);                                       \
    }                                                                        \
  }

}  // namespace

bm_status window_forward_plain(const AttnArgs& a, void* o, float* lse, hipStream_t st) {
  PlainArgs p = plain_args(a);
  p.o = o; p.lse_out = lse;
  const long wgs = tiles_of(a.cu_host, a.cu_host + 1, a.S) * a.Hq;
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), 0, st, p); };
  BM_PLAIN_SWITCH(window_plain_fwd_kernel)
  BM_CHECK_LAUNCH("window_plain_fwd");
  return BM_OK;
}

bm_status window_backward_plain(const AttnArgs& a, const void* o, const void* d_o, const float* lse, void* dq, void* dk, void* dv, int ld_dq,
                                float* delta, hipStream_t st) {
  PlainArgs p = plain_args(a);
  p.d_o = d_o; p.lse = lse; p.delta = delta;
  p.dq = dq; p.dk = dk; p.dv = dv; p.ldd = ld_dq; p.ldd_kv = a.ld_dkv;
  const long rows = (long)a.T * a.Hq;
  if (rows > 0) {
    const dim3 grid(cdiv(rows, 16)), block(256);
    if (a.dtype == BM_DTYPE_BF16)
      hipLaunchKernelGGL(window_plain_delta_kernel<bf16_t>, grid, block, 0, st, (const bf16_t*)o, (const bf16_t*)d_o, p.ldo, a.dh, delta, a.T, a.Hq);
    else
      hipLaunchKernelGGL(window_plain_delta_kernel<float>, grid, block, 0, st, (const float*)o, (const float*)d_o, p.ldo, a.dh, delta, a.T, a.Hq);
  }
  p.kv_wgs = (int)(tiles_of(a.kv_cu_host(), a.key_end_host, a.S) * a.Hkv);
  const long wgs = p.kv_wgs + tiles_of(a.cu_host, a.cu_host + 1, a.S) * a.Hq;
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), 0, st, p); };
  if (wgs > 0) {
    BM_PLAIN_SWITCH(window_plain_bwd_kernel)
  }
  BM_CHECK_LAUNCH("window_plain_bwd");
  return BM_OK;
}

}  // namespace bm
