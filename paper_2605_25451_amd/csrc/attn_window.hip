// Attention with a sliding window and first tokens that stay visible: entry points, argument checks, the choice between
// matrix-core kernels and those in plain fp32 arithmetic, and few queries in the latter.
#include "attn_window.h"
#include "../../include/bigmac_window_attention.h"

#include <algorithm>

namespace bm {

size_t window_backward_mfma_scratch_bytes(int window, int sinks, int Hq, int Hkv, int dh, int S, int Tq, int Tk);
bm_status window_forward_mfma(const AttnArgs& a, void* o, float* lse, hipStream_t st);
bm_status window_forward_plain(const AttnArgs& a, void* o, float* lse, hipStream_t st);
bm_status window_backward_plain(const AttnArgs& a, const void* o, const void* d_o, const float* lse, void* dq, void* dk, void* dv, int ld_dq,
                                float* delta, hipStream_t st);
bm_status window_tokens_mfma(const AttnArgs& a, const TokenSplit& split, void* o, float* lse, hipStream_t st);
bm_status window_backward_mfma(const AttnArgs& a, const void* o, const void* d_o, const float* lse, void* dq, void* dk,
                               void* dv, int ld_dq, void* scratch, hipStream_t st);
void window_backward_mfma_plan(const AttnArgs& a, int32_t* out);

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

template <int P> __device__ inline float lanes_sum(float v) {      // over the lanes P, 2 P, ... apart
#pragma unroll
  for (int off = P; off < 64; off <<= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// Few queries in plain arithmetic (fp32, small heads): a workgroup takes a part of the keys of one sequence and kv head and RB of
// its rows (token by token, head by head of the group), a wavefront 64 keys at a time.
//   scores: eight lanes share a key, so that they read 128 bytes of its row at once; their sums meet in the vector unit
//   values: the lanes of a row hold 16 bytes of it each, the weights come back from LDS
// Bound by reading K and V up to four rows.
constexpr int RB = 4;
template <bool STREAM, typename T>
__device__ inline void read16(const T* p, float (&x)[Elt<T>::VEC]) {
  using Raw = unsigned int __attribute__((ext_vector_type(4)));
  struct alignas(16) Run { T v[Elt<T>::VEC]; };
  const Raw* from = reinterpret_cast<const Raw*>(p);
  const Run run = __builtin_bit_cast(Run, STREAM ? __builtin_nontemporal_load(from) : *from);
#pragma unroll
  for (int e = 0; e < Elt<T>::VEC; ++e) x[e] = Elt<T>::to_f(run.v[e]);
}
template <typename T, int DH, bool STREAM>
__global__ __launch_bounds__(256) void window_token_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v, int ld, int ldk, const int32_t* __restrict__ cu,
    const int32_t* __restrict__ cuk, int S, T* __restrict__ o, int ldo, float* __restrict__ lse, int Ttot, int Hkv, int group,
    float scale_log2, LocalMask w, TokenSplit split) {
  constexpr int VEC = Elt<T>::VEC, CH = DH / VEC, CL = (CH + 7) / 8;      // chunks of a row, of a lane
  constexpr int LV = CH <= 1 ? 1 : CH <= 2 ? 2 : CH <= 4 ? 4 : CH <= 8 ? 8 : CH <= 16 ? 16 : 32;   // lanes of a row of values
  constexpr int KV = 64 / LV;                                             // its rows at a time
  __shared__ float weight[4][64][RB];
  __shared__ float sums[4][RB][DH], stats[4][RB][2];
  int hk;
  const int slot = token_slot(split, Hkv, blockIdx.x, &hk);
  TokenPart where;
  if (!find_token_part(split, S, slot, &where)) return;
  const int seq = where.seq, part = where.part, nparts = where.parts;
  const int lo = cu[seq], L = cu[seq + 1] - lo, lok = cuk[seq], Lk = w.key_end[seq] - lok, off = Lk - L;
  const int rows = L * group, r0 = blockIdx.y * RB;
  if (r0 >= rows) return;
  const KeyWalk<TOKEN_KEYS> walk(w, off, 0, L, Lk);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (walk.n + nparts - 1) / nparts, first = part * per, last = min(walk.n, first + per);
  const int begin = window_begin(w, off);
  const int kg = lane >> 3, j = lane & 7, vg = lane / LV, vc = lane % LV;
  float qr[RB][CL][VEC];
  int at[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const int row = min(r0 + r, rows - 1);
    at[r] = off + row / group;
    const T* p = q + (size_t)(lo + row / group) * ld + (hk * group + row % group) * DH;
#pragma unroll
    for (int i = 0; i < CL; ++i) {
      load16(p + min(j + 8 * i, CH - 1) * VEC, qr[r][i]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) qr[r][i][e] = j + 8 * i < CH ? qr[r][i][e] * scale_log2 : 0.f;
    }
  }
  float m[RB], l[RB], acc[RB][VEC];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    m[r] = NO_MAX; l[r] = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[r][e] = 0.f;
  }
  const T* kb = k + (size_t)lok * ldk + hk * DH;
  const T* vb = v + (size_t)lok * ldk + hk * DH;
  // 64 keys: two tiles that may lie apart (first tokens and window); past the part's last one nothing is visible
  for (int t = first + wave * 2; t < last; t += 8) {
    const int ka = walk.tile(t) * TOKEN_KEYS, kn = t + 1 < last ? walk.tile(t + 1) * TOKEN_KEYS : Lk;
    auto key_of = [&](int i) { return i < TOKEN_KEYS ? ka + i : kn + i - TOKEN_KEYS; };
    float sc[RB];
#pragma unroll
    for (int i = 0; i < 8; ++i) {                          // keys i * 8 + kg; lane j keeps those of i == j
      const T* row = kb + (size_t)min(seen_row(w, begin, key_of(i * 8 + kg)), Lk - 1) * ldk;
      float d[RB];
#pragma unroll
      for (int r = 0; r < RB; ++r) d[r] = 0.f;
#pragma unroll
      for (int n = 0; n < CL; ++n) {
        float x[VEC];
        read16<STREAM>(row + min(j + 8 * n, CH - 1) * VEC, x);
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
          for (int e = 0; e < VEC; ++e) d[r] = fmaf(qr[r][n][e], x[e], d[r]);
      }
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        // the eight lanes: neighbours, pairs, then the two halves of eight
        d[r] += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(d[r]), 0xB1, 0xf, 0xf, true));
        d[r] += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(d[r]), 0x4E, 0xf, 0xf, true));
        d[r] += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(d[r]), 0x141, 0xf, 0xf, true));
        sc[r] = i == j ? d[r] : sc[r];
      }
    }
    const int key = key_of(j * 8 + kg);
    float p[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const float x = key >= Lk || hidden(w, key, at[r]) ? -INFINITY : sc[r];
      float mx = x;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d, 64));
      const float mn = fmaxf(m[r], mx), corr = exp2f(m[r] - mn);
      m[r] = mn;
      p[r] = exp2f(x - mn);
      l[r] = l[r] * corr + p[r];
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[r][e] *= corr;
    }
    *reinterpret_cast<float4*>(weight[wave][j * 8 + kg]) = float4{p[0], p[1], p[2], p[3]};
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (a wavefront's own rows: no barrier)
    __builtin_amdgcn_wave_barrier();
#pragma unroll 8
    for (int i = 0; i < 64 / KV; ++i) {
      const int n = i * KV + vg;
      float x[VEC];
      read16<STREAM>(vb + (size_t)min(seen_row(w, begin, key_of(n)), Lk - 1) * ldk + min(vc, CH - 1) * VEC, x);
      const float4 f = *reinterpret_cast<const float4*>(weight[wave][n]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        acc[0][e] = fmaf(f.x, x[e], acc[0][e]);
        acc[1][e] = fmaf(f.y, x[e], acc[1][e]);
        acc[2][e] = fmaf(f.z, x[e], acc[2][e]);
        acc[3][e] = fmaf(f.w, x[e], acc[3][e]);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    l[r] = lanes_sum<1>(l[r]);
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[r][e] = lanes_sum<LV>(acc[r][e]);
    if (vg == 0 && vc < CH)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sums[wave][r][vc * VEC + e] = acc[r][e];
    if (lane == 0) { stats[wave][r][0] = m[r]; stats[wave][r][1] = l[r]; }
  }
  __syncthreads();
  for (int e = tid; e < min(RB, rows - r0) * DH; e += 256) {
    const int r = e / DH, c = e % DH, row = r0 + r;
    float top = NO_MAX;
#pragma unroll
    for (int x = 0; x < 4; ++x) top = fmaxf(top, stats[x][r][0]);
    float sum = 0.f, val = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float f = exp2f(stats[x][r][0] - top);
      sum = fmaf(f, stats[x][r][1], sum);
      val = fmaf(f, sums[x][r][c], val);
    }
    const int t = lo + row / group, h = hk * group + row % group;
    if (nparts == 1) {
      o[(size_t)t * ldo + h * DH + c] = Elt<T>::from_f(val / sum);
      if (c == 0) lse[(size_t)h * Ttot + t] = (top + log2f(sum)) * LN2;
    } else {
      const size_t at = ((size_t)where.place * Hkv + hk) * split.rows + row;
      split.sums[at * DH + c] = val;
      if (c == 0) {
        split.stats[at * 2] = top;
        split.stats[at * 2 + 1] = sum;
      }
    }
  }
}

// Where the parts of more sequences than a table in the arguments holds begin; a workgroup for 256 sequences, which sums the
// parts of all those in front of them for itself.
__global__ __launch_bounds__(256) void window_map_kernel(const int32_t* __restrict__ cu, const int32_t* __restrict__ cuk, int S,
                                                         LocalMask w, TokenSplit t) {
  __shared__ int sums[3][4], front[3][4];
  const int tid = threadIdx.x, wave = tid >> 6, s0 = blockIdx.x * 256, s = s0 + tid;
  auto parts = [&](int i) { return i < S ? t.count(w, cu[i + 1] - cu[i], w.key_end[i] - cuk[i]) : 0; };
  // parts, places and split sequences: in front of this workgroup's, then up to this thread's
  int before[3] = {0, 0, 0};
#pragma unroll 4
  for (int i = tid; i < s0; i += 256) {
    const int n = parts(i);
    before[0] += n;
    before[1] += n > 1 ? n : 0;
    before[2] += n > 1;
  }
  const int mine = parts(s), own[3] = {mine, mine > 1 ? mine : 0, mine > 1};
  int at[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int upto = scan_lanes(own[k]);
    at[k] = upto - own[k];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) before[k] += __shfl_xor(before[k], d, 64);
    if ((tid & 63) == 63) { sums[k][wave] = upto; front[k][wave] = before[k]; }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k)
    for (int x = 0; x < 4; ++x) at[k] += front[k][x] + (x < wave ? sums[k][x] : 0);
  if (s >= S) return;
  t.map[s] = at[0];
  if (s == S - 1) t.map[S] = at[0] + mine;
  t.map[S + 1 + s] = at[1];
  if (mine > 1) t.map[2 * S + 1 + at[2]] = s;
  for (int i = 0; i < mine; ++i) t.map[3 * S + 1 + at[0] + i] = s;
}

// o and lse from the parts of a sequence: 32 threads share a row, four columns each, and take every eighth part in order; the eight are
// joined in order.  grid: x sequences of more than one part, y kv heads, z rows.
template <typename T>
__global__ __launch_bounds__(256) void window_join_kernel(const int32_t* __restrict__ cu, int S, T* __restrict__ o, int ldo,
                                                          float* __restrict__ lse, int Ttot, int Hkv, int group, int dh, TokenSplit split) {
  __shared__ float tops[8], sums[8];
  __shared__ float4 vals[8][32];
  const int hk = blockIdx.y, row = blockIdx.z;
  const TokenPart p = split_sequence(split, S, blockIdx.x);
  const int lo = cu[p.seq], rows = (cu[p.seq + 1] - lo) * group, n = p.parts;
  if (row >= rows) return;
  const int c = threadIdx.x % 32, eighth = threadIdx.x / 32, col = min(c * 4, dh - 4);
  const size_t step = (size_t)Hkv * split.rows, at = ((size_t)p.place * Hkv + hk) * split.rows + row;
  float top = NO_MAX, sum = 0.f;
  float4 val = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = eighth; i < n; i += 8) {
    const float2 s = *reinterpret_cast<const float2*>(split.stats + (at + i * step) * 2);
    const float4 x = *reinterpret_cast<const float4*>(split.sums + (at + i * step) * dh + col);
    const float m = fmaxf(top, s.x), old = exp2f(top - m), f = exp2f(s.x - m);
    top = m;
    sum = sum * old + f * s.y;
    val.x = val.x * old + f * x.x;
    val.y = val.y * old + f * x.y;
    val.z = val.z * old + f * x.z;
    val.w = val.w * old + f * x.w;
  }
  if (c == 0) { tops[eighth] = top; sums[eighth] = sum; }
  vals[eighth][c] = val;
  __syncthreads();
  if (eighth > 0 || c * 4 >= dh) return;
  top = NO_MAX;
#pragma unroll
  for (int x = 0; x < 8; ++x) top = fmaxf(top, tops[x]);
  sum = 0.f;
  val = float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int x = 0; x < 8; ++x) {
    const float f = exp2f(tops[x] - top);
    const float4 y = vals[x][c];
    sum = fmaf(f, sums[x], sum);
    val.x = fmaf(f, y.x, val.x);
    val.y = fmaf(f, y.y, val.y);
    val.z = fmaf(f, y.z, val.z);
    val.w = fmaf(f, y.w, val.w);
  }
  const int t = lo + row / group, h = hk * group + row % group;
  T* out = o + (size_t)t * ldo + h * dh + c * 4;
  out[0] = Elt<T>::from_f(val.x / sum);
  out[1] = Elt<T>::from_f(val.y / sum);
  out[2] = Elt<T>::from_f(val.z / sum);
  out[3] = Elt<T>::from_f(val.w / sum);
  if (c == 0) lse[(size_t)h * Ttot + t] = (top + log2f(sum)) * LN2;
}

template <typename T, int DH>
void token_launch(const AttnArgs& a, const TokenSplit& split, void* o, float* lse, hipStream_t st) {
  auto kern = split.stream ? window_token_kernel<T, DH, true> : window_token_kernel<T, DH, false>;
  hipLaunchKernelGGL(kern, dim3(token_grid(split, a.Hkv), cdiv(split.rows, RB)), dim3(256), 0, st, (const T*)a.q, (const T*)a.k,
                     (const T*)a.v, a.ld_qkv, a.kv_ld(), a.cu_dev, a.kv_cu_dev(), a.S, (T*)o, a.Hq * a.dh, lse, a.T,
                     a.Hkv, a.Hq / a.Hkv, LOG2E / sqrtf((float)a.dh), a.local, split);
}

bool mfma_head(int dtype, int dh) { return dtype == BM_DTYPE_BF16 && (dh == 64 || dh == 72 || dh == 128); }

// Workgroups that the parts of few queries come to, at most next to one per sequence and kv head, and tiles that a part may always have:
// twice as many where the sequences alone fill the chip, so that fewer are split.  us (32 / 8 heads of 128, two workgroups to a CU), 1024 -> 2048
// workgroups: 64 sequences of up to 4096 visible keys 175 -> 172, 256 of 1024 174 -> 193, 16 of 8192 102 both.  4 -> 8 -> 16 tiles: one sequence of
// 8192 18.6 -> 15.7 -> 15.7, 4 of 4096 26.4 -> 24.0 -> 25.2, 55 of 300 20.8 -> 18.1 -> 12.7, 59 of 300, 16 heads of 64, 20.4 -> 19.4 -> 14.9.
constexpr int TOKEN_WGS = 1024, TOKEN_TILES = 8, NUM_CU = 256;
// A sequence of more than one part has at most twice as many as its tiles come to, TOKEN_WGS in all.
constexpr size_t TOKEN_PLACES = 2 * TOKEN_WGS;
// rows x heads of a group that the parts have room for, for any lengths of Tq queries
int token_rows(int Hq, int Hkv, int Tq) {
  const long group = Hq / Hkv;
  return group > TOKEN_ROWS ? 0 : (int)std::min<long>(Tq * group, TOKEN_ROWS);
}
size_t token_map_ints(int S) { return S > TOKEN_TABLE ? 4 * (size_t)S + 1 + TOKEN_WGS : 0; }

bool few_queries(const AttnArgs& a) { return a.max_seqlen * (long)(a.Hq / a.Hkv) <= TOKEN_ROWS; }

// Has every one of the Tk key rows one sequence at most?  Lists that are not in order are sorted, us: 256 sequences 3, 1000 16, 4000 220, which their kernels (151,
// 467, 522) cover; longer ones count as shared.
constexpr int SORTED_SEQS = 4096;
bool owned_rows(const int32_t* begin, const int32_t* end, int S, int Tk) {
  long rows = 0;
  bool in_order = true;
  for (int s = 0, last = 0; s < S; ++s) {
    if (end[s] == begin[s]) continue;
    rows += end[s] - begin[s];
    in_order = in_order && begin[s] >= last;
    last = end[s];
  }
  if (in_order || rows > Tk || S > SORTED_SEQS) return in_order;
  uint64_t spans[SORTED_SEQS];
  int n = 0;
  for (int s = 0; s < S; ++s)
    if (end[s] > begin[s]) spans[n++] = (uint64_t)begin[s] << 32 | (uint32_t)end[s];
  std::sort(spans, spans + n);
  for (int i = 1; i < n; ++i)
    if ((spans[i] >> 32) < (uint32_t)spans[i - 1]) return false;
  return true;
}

struct TokenPlan { TokenSplit split; long places; int joins; };    // joins: sequences of more than one part
TokenPlan token_plan(const AttnArgs& a) {
  TokenSplit t{};
  const int32_t *cq = a.cu_host, *kb = a.cu_k_host, *ke = a.key_end_host;
  long tiles = 0, whole = 0;
  t.per = 1;
  for (int s = 0; s < a.S; ++s) {
    const int n = t.count(a.local, cq[s + 1] - cq[s], ke[s] - kb[s]);
    tiles += n;
    whole += n > 0;
  }
  t.per = std::max(whole * a.Hkv >= NUM_CU ? 2 * TOKEN_TILES : TOKEN_TILES, cdiv(tiles * a.Hkv, TOKEN_WGS));
  t.rows = a.max_seqlen * (a.Hq / a.Hkv);
  long parts = 0, places = 0;
  int joins = 0;
  t.n = a.S <= TOKEN_TABLE ? a.S : 0;
  for (int s = 0; s < a.S; ++s) {
    const int n = t.count(a.local, cq[s + 1] - cq[s], ke[s] - kb[s]);
    if (s < TOKEN_TABLE) t.parts[s] = (uint16_t)n;           // below 2^16: about TOKEN_WGS at most
    parts += n;
    places += n > 1 ? n : 0;
    joins += n > 1;
  }
  t.wgs = (int)(parts * a.Hkv);
  // Keys and values past the caches, where they are more than the L2s hold and read by one workgroup each.  us, through them -> past: 64 sequences of up to 4096
  // (883 MB) 171 -> 153, 256 of 1024 172 -> 151, 1000 of 1024 518 -> 467, 4 of 4096 (67 MB) 22.2 -> 21.4; but 55 of 300 (39 MB) 12.6 -> 13.1, 59 of 300, 16 heads
  // of 64 (43 MB) 14.9 -> 15.2; fp32, 16 of 2000 46 -> 42.  Sequences that share rows find them in the caches: 256 that share 2048 keys 106 -> 222, 16
  // prompts of 4096 with 4 answers each 69 -> 107, 8 that share 32768 67 -> 121.
  t.stream = (mfma_head(a.dtype, a.dh) || t.rows <= RB) && (double)tiles * TOKEN_KEYS * a.Hkv * a.dh * 2 * elt_size(a.dtype) > 60e6 &&
             owned_rows(kb, ke, a.S, a.Tk);
  // The kv heads of a part on one XCD, where a row of a head is no whole cache lines or the chip is full many times: us, 20 sequences of 2000, 16
  // heads of 72, 44.5 -> 35.9; 1000 of 1024, 8 kv heads of 128, 541 -> 517, 256 174 -> 172.5; but one of 8192 13.8 -> 14.5, 16 101 -> 104.
  t.same_xcd = a.dh * elt_size(a.dtype) % 128 != 0 || t.wgs >= 8 * NUM_CU;
  return TokenPlan{t, places, joins};
}

bm_status window_tokens(const AttnArgs& a, void* scratch, void* o, float* lse, hipStream_t st) {
  const TokenPlan plan = token_plan(a);
  TokenSplit t = plan.split;
  t.sums = (float*)scratch;
  t.stats = t.sums + (size_t)plan.places * a.Hkv * t.rows * a.dh;
  t.map = (int32_t*)(t.stats + (size_t)plan.places * a.Hkv * t.rows * 2);
  if (!t.n) {
    hipLaunchKernelGGL(window_map_kernel, dim3(cdiv(a.S, 256)), dim3(256), 0, st, a.cu_dev, a.kv_cu_dev(), a.S, a.local, t);
    BM_CHECK_LAUNCH("window_map");
  }
  if (mfma_head(a.dtype, a.dh)) {
    BM_RETURN_IF(window_tokens_mfma(a, t, o, lse, st));
  } else {
#define BM_HEAD(TT)                                              \
  switch (a.dh) {                                                \
    case 8: token_launch<TT, 8>(a, t, o, lse, st); break;        \
    case 16: token_launch<TT, 16>(a, t, o, lse, st); break;      \
    default: token_launch<TT, 32>(a, t, o, lse, st);             \
  }
    if (a.dtype == BM_DTYPE_BF16) {
      BM_HEAD(bf16_t)
    } else if (a.dh == 64) {
      token_launch<float, 64>(a, t, o, lse, st);
    } else if (a.dh == 72) {
      token_launch<float, 72>(a, t, o, lse, st);
    } else if (a.dh == 128) {
      token_launch<float, 128>(a, t, o, lse, st);
    } else {
      BM_HEAD(float)
    }
#undef BM_HEAD
    BM_CHECK_LAUNCH("window_token");
  }
  if (plan.joins > 0) {
    const dim3 grid(plan.joins, a.Hkv, t.rows), block(256);
#define BM_L(TT)                                                                                                           \
  hipLaunchKernelGGL(window_join_kernel<TT>, grid, block, 0, st, a.cu_dev, a.S, (TT*)o, a.Hq * a.dh, lse, a.T, a.Hkv, a.Hq / a.Hkv, \
                     a.dh, t)
    if (a.dtype == BM_DTYPE_BF16) BM_L(bf16_t); else BM_L(float);
#undef BM_L
    BM_CHECK_LAUNCH("window_join");
  }
  return BM_OK;
}

constexpr int MAX_ROWS = 1 << 26;        // offsets of rows stay far from 2^31

constexpr int MAX_LD = 1 << 24;          // offsets in a tile of 128 rows stay below 2^32 bytes

bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

bm_status check_sizes(int dtype, int window, int sinks, int Hq, int Hkv, int dh, int S) {
  BM_ARG_CHECK(dtype == BM_DTYPE_BF16 || dtype == BM_DTYPE_FP32, "window attention: dtype %d", dtype);
  BM_ARG_CHECK(window >= 1, "window attention: window %d", window);
  BM_ARG_CHECK(sinks >= 0 && sinks <= BM_WINDOW_MAX_SINKS, "window attention: %d first tokens (0..%d)", sinks, BM_WINDOW_MAX_SINKS);
  BM_ARG_CHECK(Hq > 0 && Hkv > 0 && Hq % Hkv == 0 && Hq < (1 << 16), "window attention: heads %d/%d", Hq, Hkv);
  BM_ARG_CHECK(S >= 1 && S < (1 << 16), "window attention: %d sequences", S);
  switch (dh) {
    case 8: case 16: case 32: case 64: case 72: case 128: return BM_OK;
    default: set_error("window attention: head_dim %d unsupported (8,16,32,64,72,128)", dh); return BM_ERR_UNSUPPORTED;
  }
}

// unmasked (query, key) pairs of a head
double pairs_of(int Lq, int Lk, int window, int sinks) {
  // keys of the window: query at p sees min(p + 1, window)
  auto upto = [](double n, double w) { return n <= w ? n * (n + 1) / 2 : w * (w + 1) / 2 + (n - w) * w; };
  double n = upto(Lk, window) - upto(Lk - Lq, window);
  if (sinks > 0)
    n += upto(std::max(0, Lk - window), sinks) - upto(std::max(0, Lk - Lq - window), sinks);
  return n;
}

struct Sequences {
  const int32_t *cu_q_dev, *cu_q_host, *k_begin_dev, *k_end_dev, *k_begin_host, *k_end_host;
};

bm_status check_args(int dtype, int window, int sinks, int Hq, int Hkv, int dh, int ld_q, int ld_kv, const Sequences& c, int S,
                     AttnArgs* a, double* pairs) {
  BM_RETURN_IF(check_sizes(dtype, window, sinks, Hq, Hkv, dh, S));
  const int vec = dtype == BM_DTYPE_BF16 ? 8 : 4;
  BM_ARG_CHECK(ld_q >= (long)Hq * dh && ld_q % vec == 0 && ld_q < MAX_LD, "window attention: query row stride %d", ld_q);
  BM_ARG_CHECK(ld_kv >= (long)Hkv * dh && ld_kv % vec == 0 && ld_kv < MAX_LD, "window attention: key/value row stride %d", ld_kv);
  BM_ARG_CHECK(c.cu_q_dev && c.cu_q_host, "window attention: NULL offsets");
  const bool own = c.k_begin_dev || c.k_end_dev || c.k_begin_host || c.k_end_host;
  BM_ARG_CHECK(!own || (c.k_begin_dev && c.k_end_dev && c.k_begin_host && c.k_end_host),
               "window attention: key offsets are all given or all NULL");
  const int32_t *kb = own ? c.k_begin_host : c.cu_q_host, *ke = own ? c.k_end_host : c.cu_q_host + 1;
  BM_ARG_CHECK(c.cu_q_host[0] == 0, "window attention: query offsets must start at 0");
  int max_q = 0, max_k = 0, rows = 0;
  for (int s = 0; s < S; ++s) {
    BM_ARG_CHECK(c.cu_q_host[s + 1] >= c.cu_q_host[s] && c.cu_q_host[s + 1] <= MAX_ROWS, "window attention: query offsets of sequence %d", s);
    BM_ARG_CHECK(kb[s] >= 0 && ke[s] >= kb[s] && ke[s] <= MAX_ROWS, "window attention: key offsets of sequence %d", s);
    const int lq = c.cu_q_host[s + 1] - c.cu_q_host[s], lk = ke[s] - kb[s];
    BM_ARG_CHECK(lq <= lk, "window attention: sequence %d has %d queries and %d keys", s, lq, lk);
    max_q = std::max(max_q, lq);
    max_k = std::max(max_k, lk);
    rows = std::max(rows, ke[s]);
    *pairs += pairs_of(lq, lk, window, sinks);
  }
  // grids stay below 2^32 threads, but for the gradients' at head size 128, which look at theirs before they launch anything
  BM_ARG_CHECK((long)c.cu_q_host[S] * Hq < (1L << 26) && (long)rows * Hkv < (1L << 26) && (long)S * Hq < (1L << 22),
               "window attention: %d sequences, %d queries of %d heads and %d keys of %d (rows x heads below 2^26, sequences x heads below 2^22)",
               S, c.cu_q_host[S], Hq, rows, Hkv);
  a->dtype = dtype; a->causal = 1; a->Hq = Hq; a->Hkv = Hkv; a->dh = dh;
  a->ld_qkv = ld_q; a->cu_dev = c.cu_q_dev; a->cu_host = c.cu_q_host; a->S = S; a->T = c.cu_q_host[S]; a->max_seqlen = max_q;
  a->cu_k_dev = own ? c.k_begin_dev : c.cu_q_dev; a->cu_k_host = kb; a->Tk = rows; a->ld_kv = ld_kv; a->max_klen = max_k;
  a->local = LocalMask{std::min(window, MAX_ROWS), sinks, own ? c.k_end_dev : c.cu_q_dev + 1};
  a->key_end_host = ke;
  return BM_OK;
}

// Do rows of `heads` heads at p and at x share an element?  Equal strides: their columns may lie side by side.
bool share(const void* p, int rows_p, long ld_p, long width_p, const void* x, int rows_x, long ld_x, long width_x, int size) {
  if (rows_p == 0 || rows_x == 0) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(x);
  const uintptr_t a_end = a + ((rows_p - 1) * ld_p + width_p) * size, b_end = b + ((rows_x - 1) * ld_x + width_x) * size;
  if (a >= b_end || b >= a_end) return false;
  if (ld_p != ld_x) return true;
  const uintptr_t row = (uintptr_t)ld_p * size, ahead = a >= b ? (a - b) % row : (row - (b - a) % row) % row;   // of a's columns against b's
  return ahead < (uintptr_t)width_x * size || row - ahead < (uintptr_t)width_p * size;
}

bm_status check_scratch(const void* scratch, size_t bytes, size_t need) {
  BM_ARG_CHECK(al16(scratch), "window attention: misaligned scratch");
  if (need > 0 && (!scratch || bytes < need)) {
    set_error("window attention: scratch of %zu bytes, %zu needed", scratch ? bytes : (size_t)0, need);
    return BM_ERR_WORKSPACE_TOO_SMALL;
  }
  return BM_OK;
}

}  // namespace

}  // namespace bm

using namespace bm;

extern "C" size_t bm_window_attention_scratch_bytes(int32_t dtype, int32_t window, int32_t sinks, int32_t Hq, int32_t Hkv,
                                                    int32_t dh, int32_t S, int32_t Tq, int32_t Tk) {
  if (check_sizes(dtype, window, sinks, Hq, Hkv, dh, S) != BM_OK || Tq < 0 || Tk < 0 || Tq > MAX_ROWS || Tk > MAX_ROWS) return 0;
  const size_t rows = (size_t)token_rows(Hq, Hkv, Tq);
  return rows ? align_up((TOKEN_PLACES * rows * (dh + 2) + token_map_ints(S)) * sizeof(float), 256) : 0;
}

extern "C" bm_status bm_window_attention_forward(int32_t dtype, int32_t window, int32_t sinks, int32_t Hq, int32_t Hkv,
                                                 int32_t dh, const void* q, int32_t ld_q, const void* k, const void* v,
                                                 int32_t ld_kv, const int32_t* cu_q_dev, const int32_t* cu_q_host,
                                                 const int32_t* k_begin_dev, const int32_t* k_end_dev,
                                                 const int32_t* k_begin_host, const int32_t* k_end_host, int32_t S, void* o,
                                                 float* lse, void* scratch, size_t scratch_bytes, void* hip_stream) {
  AttnArgs a{};
  double pairs = 0;
  const Sequences c{cu_q_dev, cu_q_host, k_begin_dev, k_end_dev, k_begin_host, k_end_host};
  BM_RETURN_IF(check_args(dtype, window, sinks, Hq, Hkv, dh, ld_q, ld_kv, c, S, &a, &pairs));
  if (a.T == 0) return BM_OK;
  BM_ARG_CHECK(q && k && v && o && lse, "window attention: NULL pointer");
  BM_ARG_CHECK(al16(q) && al16(k) && al16(v) && al16(o) && al16(lse), "window attention: misaligned pointer");
  BM_RETURN_IF(check_scratch(scratch, scratch_bytes,
                             bm_window_attention_scratch_bytes(dtype, window, sinks, Hq, Hkv, dh, S, a.T, a.Tk)));
  a.q = q; a.k = k; a.v = v;
  hipStream_t st = (hipStream_t)hip_stream;
  ProfScope prof(PROF_ATTN_FWD, 4.0 * dh * Hq * pairs, st);
  if (few_queries(a)) return window_tokens(a, scratch, o, lse, st);
  if (mfma_head(dtype, dh)) return window_forward_mfma(a, o, lse, st);
  return window_forward_plain(a, o, lse, st);
}

extern "C" size_t bm_window_attention_backward_scratch_bytes(int32_t dtype, int32_t window, int32_t sinks, int32_t Hq,
                                                             int32_t Hkv, int32_t dh, int32_t S, int32_t Tq, int32_t Tk) {
  if (check_sizes(dtype, window, sinks, Hq, Hkv, dh, S) != BM_OK || Tq < 0 || Tk < 0 || Tq > MAX_ROWS || Tk > MAX_ROWS) return 0;
  const size_t generic = align_up((size_t)Hq * Tq * sizeof(float), 256);   // delta
  return mfma_head(dtype, dh) ? window_backward_mfma_scratch_bytes(window, sinks, Hq, Hkv, dh, S, Tq, Tk) : generic;
}

extern "C" bm_status bm_window_attention_backward(int32_t dtype, int32_t window, int32_t sinks, int32_t Hq, int32_t Hkv,
                                                  int32_t dh, const void* q, int32_t ld_q, const void* k, const void* v,
                                                  int32_t ld_kv, const void* o, const void* d_o, const float* lse,
                                                  const int32_t* cu_q_dev, const int32_t* cu_q_host,
                                                  const int32_t* k_begin_dev, const int32_t* k_end_dev,
                                                  const int32_t* k_begin_host, const int32_t* k_end_host, int32_t S, void* dq,
                                                  int32_t ld_dq, void* dk, void* dv, int32_t ld_dkv, void* scratch,
                                                  size_t scratch_bytes, void* hip_stream) {
  AttnArgs a{};
  double pairs = 0;
  const Sequences c{cu_q_dev, cu_q_host, k_begin_dev, k_end_dev, k_begin_host, k_end_host};
  BM_RETURN_IF(check_args(dtype, window, sinks, Hq, Hkv, dh, ld_q, ld_kv, c, S, &a, &pairs));
  if (a.Tk == 0) return BM_OK;
  const int vec = dtype == BM_DTYPE_BF16 ? 8 : 4;
  BM_ARG_CHECK(ld_dq >= (long)Hq * dh && ld_dq % vec == 0, "window attention: dq row stride %d", ld_dq);
  BM_ARG_CHECK(ld_dkv >= (long)Hkv * dh && ld_dkv % vec == 0, "window attention: dk/dv row stride %d", ld_dkv);
  BM_ARG_CHECK(k && v && dk && dv && (a.T == 0 || (q && o && d_o && lse && dq)), "window attention: NULL pointer");
  BM_ARG_CHECK(al16(q) && al16(k) && al16(v) && al16(o) && al16(d_o) && al16(lse) && al16(dq) && al16(dk) && al16(dv),
               "window attention: misaligned pointer");
  // every key row has one owner, and no tile may read what another one has overwritten
  for (int s = 1, end = a.key_end_host[0]; s < S; ++s) {
    if (a.key_end_host[s] == a.cu_k_host[s]) continue;
    BM_ARG_CHECK(a.cu_k_host[s] >= end, "window attention: keys of sequence %d do not lie behind those in front of it", s);
    end = a.key_end_host[s];
  }
  const int size = dtype == BM_DTYPE_BF16 ? 2 : 4;
  const long wq = (long)Hq * dh, wk = (long)Hkv * dh;
  const struct { const void* p; int rows; long ld, width; } in[] = {{q, a.T, ld_q, wq}, {o, a.T, wq, wq}, {d_o, a.T, wq, wq}, {k, a.Tk, ld_kv, wk},
                                                                    {v, a.Tk, ld_kv, wk}},
      out[] = {{dq, a.T, ld_dq, wq}, {dk, a.Tk, ld_dkv, wk}, {dv, a.Tk, ld_dkv, wk}};
  for (const auto& x : in)
    for (const auto& y : out)
      BM_ARG_CHECK(!share(x.p, x.rows, x.ld, x.width, y.p, y.rows, y.ld, y.width, size), "window attention: a gradient lies over an input");
  BM_RETURN_IF(check_scratch(scratch, scratch_bytes,
                             bm_window_attention_backward_scratch_bytes(dtype, window, sinks, Hq, Hkv, dh, S, a.T, a.Tk)));
  a.q = q; a.k = k; a.v = v; a.ld_dkv = ld_dkv;
  hipStream_t st = (hipStream_t)hip_stream;
  ProfScope prof(PROF_ATTN_BWD, 10.0 * dh * Hq * pairs, st);
  if (mfma_head(dtype, dh)) return window_backward_mfma(a, o, d_o, lse, dq, dk, dv, ld_dq, scratch, st);
  return window_backward_plain(a, o, d_o, lse, dq, dk, dv, ld_dq, (float*)scratch, st);
}

extern "C" bm_status bm_probe_window_plan(int32_t dtype, int32_t window, int32_t sinks, int32_t Hq, int32_t Hkv, int32_t dh,
                                          const int32_t* cu_q_host, const int32_t* k_begin_host, const int32_t* k_end_host, int32_t S,
                                          int32_t* forward, int32_t* backward) {
  BM_ARG_CHECK(forward && backward, "window plan: NULL pointer");
  AttnArgs a{};
  double pairs = 0;
  // (the device's copies are not looked at)
  const Sequences c{cu_q_host, cu_q_host, k_begin_host, k_end_host, k_begin_host, k_end_host};
  BM_RETURN_IF(check_args(dtype, window, sinks, Hq, Hkv, dh, Hq * dh, Hkv * dh, c, S, &a, &pairs));
  for (int i = 0; i < 4; ++i) forward[i] = backward[i] = 0;
  forward[0] = few_queries(a) ? 2 : mfma_head(dtype, dh) ? 1 : 0;
  if (forward[0] == 2) {
    const TokenSplit t = token_plan(a).split;
    forward[1] = t.wgs;
    forward[2] = t.stream;
    forward[3] = t.same_xcd;
  }
  if (mfma_head(dtype, dh)) window_backward_mfma_plan(a, backward);
  return BM_OK;
}
