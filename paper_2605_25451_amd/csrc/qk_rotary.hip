// Rotation of queries and keys over several position axes, alone or with the RMS norm of every head in the
// same pass, and the gradients of both.
//
//   n = x r, r = 1 / sqrt(mean(x^2) + eps), y = n g, z = R y       R turns the pairs (i, i + dh/2)
//   d = R^T dz,  dg += sum over tokens and heads of d n,  e = d g,  dx = r (e - n mean(e n))
//
// A group of lanes owns one token and walks heads; a lane keeps VEC pairs, so that cosines and sines are
// formed once per token and walk, in fp64 up to the fraction of a turn.  Bound by memory: every row is read and
// written once, at 4.6 TB/s forward and in the gradient (8192 tokens of 32 + 8 heads of 128, 37 and 55 us; a copy 4.9).
#include "common.h"
#include "../../include/bigmac_window_attention.h"

#include <algorithm>
#include <cmath>

namespace bm {

namespace {

constexpr int MAX_HALF = 128;

struct Rotation {
  double turns[MAX_HALF];               // of a pair, per unit of position
  int end[BM_ROTARY_MAX_AXES];          // axis a: pairs end[a-1] .. end[a]-1
  int axes;
};

struct RotaryArgs {
  const void *x[2];                     // queries and keys before norm and rotation
  const void *in[2];                    // what is turned: x itself (forward) or the gradients (backward)
  void *out[2];
  const void *gain[2];
  const int32_t* positions;
  float* part[2];                       // backward with norm: [workgroups of the side][dh] of gain gradients
  int ld_x, ld_in, ld_out, T, dh, heads[2], per[2], groups_q;   // heads of a side, heads per walk, walks over the query heads
  float eps;
};

template <typename T, int VEC> struct alignas(sizeof(T) * VEC) Pack { T v[VEC]; };

template <int N> using Bytes = unsigned int __attribute__((ext_vector_type(N / 4)));
template <int VEC, bool NT = false, typename T>
__device__ inline void load_vec(const T* p, float (&out)[VEC]) {
  using B = Bytes<sizeof(T) * VEC>;
  const B raw = NT ? __builtin_nontemporal_load(reinterpret_cast<const B*>(p)) : *reinterpret_cast<const B*>(p);
  const Pack<T, VEC> t = __builtin_bit_cast(Pack<T, VEC>, raw);
#pragma unroll
  for (int e = 0; e < VEC; ++e) out[e] = Elt<T>::to_f(t.v[e]);
}
template <int VEC, bool NT = false, typename T>
__device__ inline void store_vec(T* p, const float (&in)[VEC]) {
  Pack<T, VEC> t;
#pragma unroll
  for (int e = 0; e < VEC; ++e) t.v[e] = Elt<T>::from_f(in[e]);
  using B = Bytes<sizeof(T) * VEC>;
  if (NT) __builtin_nontemporal_store(__builtin_bit_cast(B, t), reinterpret_cast<B*>(p));
  else *reinterpret_cast<Pack<T, VEC>*>(p) = t;
}

// cosine and sine of a lane's pairs; the fraction of a turn in fp64
template <int VEC>
__device__ inline void cos_sin(const Rotation& r, const int32_t* __restrict__ positions, int T, int t, int i0, float sign,
                               float (&cs)[VEC], float (&sn)[VEC]) {
  int p[BM_ROTARY_MAX_AXES];
#pragma unroll
  for (int a = 0; a < BM_ROTARY_MAX_AXES; ++a) p[a] = positions[(size_t)min(a, r.axes - 1) * T + t];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const int i = i0 + e;
    const int pos = i < r.end[0] ? p[0] : i < r.end[1] ? p[1] : i < r.end[2] ? p[2] : p[3];
    const double a = (double)pos * r.turns[i];
    float s, c;
    sincospif(2.0f * (float)(a - rint(a)), &s, &c);
    cs[e] = c;
    sn[e] = sign * s;
  }
}

template <int LP> __device__ inline float lanes_sum(float v) {
#pragma unroll
  for (int off = 1; off < LP; off <<= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// LP lanes own a token (a power of two with the norm, whose sums go over them; otherwise just as many as there are
// chunks, LP = 0).  grid: x walks tokens, y the heads of a walk, queries first.
template <typename T, int VEC, int LP, bool NT>
__global__ __launch_bounds__(256) void qk_rotary_fwd_kernel(RotaryArgs a, Rotation rot, float sign) {
  constexpr bool NORM = LP > 0;
  constexpr int U = 4;                                     // heads in flight
  const int half = a.dh >> 1, chunks = half / VEC, lanes = NORM ? LP : chunks;
  const long gid = (long)blockIdx.x * 256 + threadIdx.x;
  const long tok = gid / lanes;
  const int c = (int)(gid - tok * lanes);
  const bool live = tok < a.T && c < chunks;
  const int t = (int)min(tok, (long)a.T - 1), i0 = min(c, chunks - 1) * VEC;
  const int side = (int)blockIdx.y < a.groups_q ? 0 : 1;
  const int first = ((int)blockIdx.y - (side ? a.groups_q : 0)) * a.per[side], last = min(a.heads[side], first + a.per[side]);
  float cs[VEC], sn[VEC], ga[VEC], gb[VEC];
  cos_sin<VEC>(rot, a.positions, a.T, t, i0, sign, cs, sn);
  if (NORM) {
    load_vec<VEC>((const T*)a.gain[side] + i0, ga);
    load_vec<VEC>((const T*)a.gain[side] + half + i0, gb);
  }
  const T* in = (const T*)a.in[side] + (size_t)t * a.ld_in + i0;
  T* out = (T*)a.out[side] + (size_t)t * a.ld_out + i0;
  for (int h0 = first; h0 < last; h0 += U) {
    float x[U][VEC], y[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const T* p = in + (size_t)min(h0 + u, last - 1) * a.dh;
      load_vec<VEC, NT>(p, x[u]);
      load_vec<VEC, NT>(p + half, y[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (NORM) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) ss += x[u][e] * x[u][e] + y[u][e] * y[u][e];
        ss = lanes_sum<LP>(c < chunks ? ss : 0.f);
        const float r = rsqrtf(ss / (float)a.dh + a.eps);
#pragma unroll
        for (int e = 0; e < VEC; ++e) { x[u][e] *= r * ga[e]; y[u][e] *= r * gb[e]; }
      }
      float p[VEC], q[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        p[e] = x[u][e] * cs[e] - y[u][e] * sn[e];
        q[e] = y[u][e] * cs[e] + x[u][e] * sn[e];
      }
      if (live && h0 + u < last) {
        T* o = out + (size_t)(h0 + u) * a.dh;
        store_vec<VEC, NT>(o, p);
        store_vec<VEC, NT>(o + half, q);
      }
    }
  }
}

// gradient with the norm: a workgroup walks tokens and leaves one row of gain gradients
template <typename T, int VEC, int LP, bool NT>
__global__ __launch_bounds__(256) void qk_rotary_norm_bwd_kernel(RotaryArgs a, Rotation rot) {
  constexpr int GROUPS = 256 / LP, U = 2;
  __shared__ float sums[GROUPS][2 * LP * VEC + 1];
  const int half = a.dh >> 1, chunks = half / VEC;
  const int c = threadIdx.x % LP, grp = threadIdx.x / LP;
  const int i0 = min(c, chunks - 1) * VEC;
  const int side = (int)blockIdx.y < a.groups_q ? 0 : 1;
  const int walk = (int)blockIdx.y - (side ? a.groups_q : 0);
  const int first = walk * a.per[side], last = min(a.heads[side], first + a.per[side]);
  float ga[VEC], gb[VEC], da[VEC], db[VEC];
  load_vec<VEC>((const T*)a.gain[side] + i0, ga);
  load_vec<VEC>((const T*)a.gain[side] + half + i0, gb);
#pragma unroll
  for (int e = 0; e < VEC; ++e) { da[e] = 0.f; db[e] = 0.f; }
  const float inv = 1.0f / (float)a.dh;
  // (every lane of a wavefront makes the same number of trips: the sums go over lanes)
  for (long base = (long)blockIdx.x * GROUPS; base < a.T; base += (long)gridDim.x * GROUPS) {
    const long tok = base + grp;
    const bool live = tok < a.T && c < chunks;
    const int t = (int)min(tok, (long)a.T - 1);
    float cs[VEC], sn[VEC];
    cos_sin<VEC>(rot, a.positions, a.T, t, i0, -1.f, cs, sn);
    const T* in = (const T*)a.in[side] + (size_t)t * a.ld_in + i0;
    const T* raw = (const T*)a.x[side] + (size_t)t * a.ld_x + i0;
    T* out = (T*)a.out[side] + (size_t)t * a.ld_out + i0;
    for (int h0 = first; h0 < last; h0 += U) {
      float d0[U][VEC], d1[U][VEC], x0[U][VEC], x1[U][VEC];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const size_t at = (size_t)min(h0 + u, last - 1) * a.dh;
        load_vec<VEC, NT>(in + at, d0[u]);
        load_vec<VEC, NT>(in + at + half, d1[u]);
        load_vec<VEC, NT>(raw + at, x0[u]);
        load_vec<VEC, NT>(raw + at + half, x1[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float ss = 0.f, dot = 0.f;
        float p[VEC], q[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          p[e] = d0[u][e] * cs[e] - d1[u][e] * sn[e];
          q[e] = d1[u][e] * cs[e] + d0[u][e] * sn[e];
          ss += x0[u][e] * x0[u][e] + x1[u][e] * x1[u][e];
          dot += p[e] * ga[e] * x0[u][e] + q[e] * gb[e] * x1[u][e];
        }
        ss = lanes_sum<LP>(c < chunks ? ss : 0.f);
        dot = lanes_sum<LP>(c < chunks ? dot : 0.f);
        const float r = rsqrtf(ss * inv + a.eps), k = dot * r * inv;      // k: mean(e n)
        if (live && h0 + u < last) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float n0 = x0[u][e] * r, n1 = x1[u][e] * r;
            da[e] += p[e] * n0;
            db[e] += q[e] * n1;
            p[e] = r * (p[e] * ga[e] - n0 * k);
            q[e] = r * (q[e] * gb[e] - n1 * k);
          }
          T* o = out + (size_t)(h0 + u) * a.dh;
          store_vec<VEC, NT>(o, p);
          store_vec<VEC, NT>(o + half, q);
        }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    sums[grp][c * VEC + e] = da[e];
    sums[grp][LP * VEC + c * VEC + e] = db[e];
  }
  __syncthreads();
  if ((int)threadIdx.x < a.dh) {
    const int i = threadIdx.x, at = i < half ? i : LP * VEC + i - half;
    float s = 0.f;
    for (int g = 0; g < GROUPS; ++g) s += sums[g][at];
    a.part[side][((size_t)walk * gridDim.x + blockIdx.x) * a.dh + i] = s;
  }
}

// Heads of 32, 64 or 128 bytes, whose halves are less than a cache line: a lane holds one 16-byte run of the head, so that the lanes of a head
// read it at once, and gets the other element of each pair from its mirror among them (lane c of the first half and LP - 1 - c hold the
// same pairs).  16351 tokens, 12 + 12 heads of 64, bf16: 27.4 -> 22.7 us, with the norm 27.7 -> 24.7, its gradient 43.7 -> 40.4.
template <int LP>
__device__ inline float mirrored(float v) {
  constexpr int CTRL = LP == 2 ? 0xB1 : LP == 4 ? 0x1B : 0x141;            // swaps in pairs, reversals of four and of eight lanes
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}

template <typename T, int VEC, int LP, bool NORM, bool NT>
__global__ __launch_bounds__(256) void qk_rotary_small_fwd_kernel(RotaryArgs a, Rotation rot, float sign) {
  constexpr int DH = LP * VEC, HALF = DH / 2, U = 8;                       // heads in flight
  const long gid = (long)blockIdx.x * 256 + threadIdx.x;
  const long tok = gid / LP;
  const int c = threadIdx.x % LP, upper = c >= LP / 2, i0 = (upper ? LP - 1 - c : c) * VEC, at = upper * HALF + i0;
  const bool live = tok < a.T;
  const int t = (int)min(tok, (long)a.T - 1);
  const int side = (int)blockIdx.y < a.groups_q ? 0 : 1;
  const int first = ((int)blockIdx.y - (side ? a.groups_q : 0)) * a.per[side], last = min(a.heads[side], first + a.per[side]);
  float cs[VEC], sn[VEC], g[VEC];
  cos_sin<VEC>(rot, a.positions, a.T, t, i0, upper ? sign : -sign, cs, sn);
  if (NORM) load_vec<VEC>((const T*)a.gain[side] + at, g);
  const T* in = (const T*)a.in[side] + (size_t)t * a.ld_in + at;
  T* out = (T*)a.out[side] + (size_t)t * a.ld_out + at;
  for (int h0 = first; h0 < last; h0 += U) {
    float x[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u) load_vec<VEC, NT>(in + (size_t)min(h0 + u, last - 1) * DH, x[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (NORM) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) ss += x[u][e] * x[u][e];
        const float r = rsqrtf(lanes_sum<LP>(ss) / (float)DH + a.eps);
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[u][e] *= r * g[e];
      }
      float z[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) z[e] = x[u][e] * cs[e] + mirrored<LP>(x[u][e]) * sn[e];
      if (live && h0 + u < last) store_vec<VEC, NT>(out + (size_t)(h0 + u) * DH, z);
    }
  }
}

template <typename T, int VEC, int LP, bool NT>
__global__ __launch_bounds__(256) void qk_rotary_small_norm_bwd_kernel(RotaryArgs a, Rotation rot) {
  constexpr int GROUPS = 256 / LP, DH = LP * VEC, HALF = DH / 2, U = 4;
  __shared__ float sums[GROUPS][DH + 1];
  const int c = threadIdx.x % LP, grp = threadIdx.x / LP, upper = c >= LP / 2, i0 = (upper ? LP - 1 - c : c) * VEC, at = upper * HALF + i0;
  const int side = (int)blockIdx.y < a.groups_q ? 0 : 1;
  const int walk = (int)blockIdx.y - (side ? a.groups_q : 0);
  const int first = walk * a.per[side], last = min(a.heads[side], first + a.per[side]);
  float g[VEC], dg[VEC];
  load_vec<VEC>((const T*)a.gain[side] + at, g);
#pragma unroll
  for (int e = 0; e < VEC; ++e) dg[e] = 0.f;
  // (every lane of a wavefront makes the same number of trips: the sums go over lanes)
  for (long base = (long)blockIdx.x * GROUPS; base < a.T; base += (long)gridDim.x * GROUPS) {
    const long tok = base + grp;
    const bool live = tok < a.T;
    const int t = (int)min(tok, (long)a.T - 1);
    float cs[VEC], sn[VEC];
    cos_sin<VEC>(rot, a.positions, a.T, t, i0, upper ? -1.f : 1.f, cs, sn);
    const T* in = (const T*)a.in[side] + (size_t)t * a.ld_in + at;
    const T* raw = (const T*)a.x[side] + (size_t)t * a.ld_x + at;
    T* out = (T*)a.out[side] + (size_t)t * a.ld_out + at;
    for (int h0 = first; h0 < last; h0 += U) {
      float d[U][VEC], x[U][VEC];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const size_t head = (size_t)min(h0 + u, last - 1) * DH;
        load_vec<VEC, NT>(in + head, d[u]);
        load_vec<VEC, NT>(raw + head, x[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float ss = 0.f, dot = 0.f, p[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          p[e] = d[u][e] * cs[e] + mirrored<LP>(d[u][e]) * sn[e];
          ss += x[u][e] * x[u][e];
          dot += p[e] * g[e] * x[u][e];
        }
        ss = lanes_sum<LP>(ss);
        dot = lanes_sum<LP>(dot);
        const float r = rsqrtf(ss * (1.0f / DH) + a.eps), k = dot * r * (1.0f / DH);      // k: mean(e n)
        if (live && h0 + u < last) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float n = x[u][e] * r;
            dg[e] += p[e] * n;
            p[e] = r * (p[e] * g[e] - n * k);
          }
          store_vec<VEC, NT>(out + (size_t)(h0 + u) * DH, p);
        }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sums[grp][at + e] = dg[e];
  __syncthreads();
  if ((int)threadIdx.x < DH) {
    float s = 0.f;
    for (int i = 0; i < GROUPS; ++i) s += sums[i][threadIdx.x];
    a.part[side][((size_t)walk * gridDim.x + blockIdx.x) * DH + threadIdx.x] = s;
  }
}

// Lanes of a token and elements of a lane
struct Lanes { int vec, chunks, pow2; bool small; };      // small: a lane for every 16 bytes of a head; otherwise for 16 (8) bytes of both halves
Lanes lanes_of(const bm_qk_rotary_desc& d) {
  Lanes l;
  const int half = d.head_dim / 2;
  const int bytes = d.head_dim * (int)elt_size(d.dtype);
  l.small = bytes == 32 || bytes == 64 || bytes == 128;
  l.vec = d.dtype == BM_DTYPE_BF16 && (half % 8 == 0 || l.small) ? 8 : 4;
  l.chunks = l.small ? bytes / 16 : half / l.vec;
  l.pow2 = 1;
  while (l.pow2 < l.chunks) l.pow2 *= 2;
  return l;
}

// Walks over the heads of either side: few tokens have their heads dealt to more lanes, each of which forms the angles again.
constexpr long WANTED_LANES = 1L << 18;
constexpr int MAX_WALKS = 1 << 14;       // of a grid's 2^16
void deal_heads(const bm_qk_rotary_desc& d, long lanes, RotaryArgs* a, int* groups) {
  const int H = d.n_q_heads + d.n_kv_heads;
  const int walks = (int)std::min<long>(std::min(H, MAX_WALKS), std::max<long>(1, WANTED_LANES / std::max<long>(lanes, 1)));
  const int per = cdiv(H, walks);
  a->heads[0] = d.n_q_heads;
  a->heads[1] = d.n_kv_heads;
  int n[2];
  for (int s = 0; s < 2; ++s) {
    n[s] = a->heads[s] ? cdiv(a->heads[s], per) : 0;
    a->per[s] = n[s] ? cdiv(a->heads[s], n[s]) : 1;
  }
  a->groups_q = n[0];
  *groups = n[0] + n[1];
}

// workgroups that walk the tokens in the gradient with the norm; each leaves a row per walk of heads
constexpr int BWD_WORKGROUPS = 1024;
struct BwdGrid { int x, y, slots[2]; };
BwdGrid bwd_grid(const bm_qk_rotary_desc& d, int T, RotaryArgs* a) {
  const Lanes l = lanes_of(d);
  BwdGrid g;
  deal_heads(d, (long)T * l.pow2, a, &g.y);
  const int per = 256 / l.pow2;
  // every workgroup makes as many trips (8192 tokens of 32 + 8 heads: 2 or 1 in 204 x 5 workgroups -> 2 in 128 x 5, 67.5 -> 59.4 us)
  const int chunks = cdiv(T, per);
  g.x = cdiv(chunks, cdiv(chunks, std::max(1, BWD_WORKGROUPS / g.y)));
  g.slots[0] = g.x * a->groups_q;
  g.slots[1] = g.x * (g.y - a->groups_q);
  return g;
}

bm_status check(const bm_qk_rotary_desc* d) {
  BM_ARG_CHECK(d, "qk rotary: NULL desc");
  BM_ARG_CHECK(d->dtype == BM_DTYPE_BF16 || d->dtype == BM_DTYPE_FP32, "qk rotary: dtype %d", d->dtype);
  BM_ARG_CHECK(d->n_q_heads >= 0 && d->n_kv_heads >= 0 && d->n_q_heads <= (1 << 16) && d->n_kv_heads <= (1 << 16) &&
               d->n_q_heads + d->n_kv_heads > 0, "qk rotary: heads %d/%d", d->n_q_heads, d->n_kv_heads);
  if (d->head_dim < 8 || d->head_dim > 2 * MAX_HALF || d->head_dim % 8 != 0) {
    set_error("qk rotary: head_dim %d unsupported (a multiple of 8 up to %d)", d->head_dim, 2 * MAX_HALF);
    return BM_ERR_UNSUPPORTED;
  }
  BM_ARG_CHECK(d->n_axes >= 1 && d->n_axes <= BM_ROTARY_MAX_AXES, "qk rotary: %d axes", d->n_axes);
  long sum = 0;
  for (int i = 0; i < d->n_axes; ++i) {
    BM_ARG_CHECK(d->pairs[i] >= 0, "qk rotary: axis %d has %d pairs", i, d->pairs[i]);
    sum += d->pairs[i];
  }
  BM_ARG_CHECK(sum == d->head_dim / 2, "qk rotary: the axes have %ld pairs, a head of %d has %d", sum, d->head_dim, d->head_dim / 2);
  BM_ARG_CHECK((d->own_frequencies == 0 || d->own_frequencies == 1) && (d->norm == 0 || d->norm == 1),
               "qk rotary: own_frequencies %d, norm %d", d->own_frequencies, d->norm);
  BM_ARG_CHECK(d->base > 0.f && std::isfinite(d->base), "qk rotary: base %g", (double)d->base);
  BM_ARG_CHECK(!d->norm || (d->eps >= 0.f && std::isfinite(d->eps)), "qk rotary: eps %g", (double)d->eps);
  return BM_OK;
}

bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// rows of one stride that hold the heads of both sides
bm_status check_rows(const bm_qk_rotary_desc& d, const char* what, const void* q, const void* k, int ld) {
  const int vec = d.dtype == BM_DTYPE_BF16 ? 8 : 4;
  BM_ARG_CHECK((!d.n_q_heads || (q && al16(q))) && (!d.n_kv_heads || (k && al16(k))), "qk rotary: %s NULL or misaligned", what);
  BM_ARG_CHECK(ld >= (long)std::max(d.n_q_heads, d.n_kv_heads) * d.head_dim && ld % vec == 0, "qk rotary: %s rows of %d elements", what, ld);
  return BM_OK;
}

Rotation rotation(const bm_qk_rotary_desc& d) {
  Rotation r{};
  const int half = d.head_dim / 2;
  const double turn = 6.283185307179586476925286766559, log_base = std::log((double)d.base);
  int first = 0;
  double fine[8], fine_step = NAN;                         // base^-(j) by eights and ones: two roundings more
  for (int a = 0; a < BM_ROTARY_MAX_AXES; ++a) {
    const int n = a < d.n_axes ? d.pairs[a] : 0, j0 = d.own_frequencies ? 0 : first;
    const double step = d.own_frequencies ? -log_base / std::max(n, 1) : -log_base / half;
    if (step != fine_step) {
      fine_step = step;
      for (int j = 0; j < 8; ++j) fine[j] = std::exp(step * j);
    }
    for (int j = 0; j < n; j += 8) {
      const double coarse = std::exp(step * (j0 + j)) / turn;
      for (int e = j; e < std::min(n, j + 8); ++e) r.turns[first + e] = coarse * fine[e - j];
    }
    first += n;
    r.end[a] = first;
  }
  r.axes = d.n_axes;
  return r;
}

// Do rows go past the caches?  Accesses of whole 128-byte lines, of more than the L2s hold together (32 MB): 32 + 8 heads of 128, us, through them
// -> past: 8192 tokens with the norm 41.7 -> 37.3, gradient 59.4 -> 54.8; 32768 tokens 146 -> 137, gradient 230 -> 222.  Fewer tokens are
// read again while they are still there (2048: 12.6 -> 13.4); parts of lines are slower (fp32, 16 + 16 heads of 72, 8192 tokens, 41 -> 52).
bool past_caches(const bm_qk_rotary_desc& d, const Lanes& l, int T) {
  const double bytes = (double)T * (d.n_q_heads + d.n_kv_heads) * d.head_dim * elt_size(d.dtype);
  const int run = (l.small ? d.head_dim : d.head_dim / 2) * (int)elt_size(d.dtype);
  return run % 128 == 0 && bytes > 32e6;
}

template <typename T, int VEC, bool NT>
void launch_fwd(const RotaryArgs& a, const Rotation& r, const Lanes& l, bool norm, float sign, int groups, hipStream_t st) {
  const int lanes = norm ? l.pow2 : l.chunks;
  const dim3 grid(cdiv((long)a.T * lanes, 256), groups), block(256);
  if (l.small) {
#define BM_S(LP)                                                                                                        \
  if (norm) hipLaunchKernelGGL((qk_rotary_small_fwd_kernel<T, VEC, LP, true, NT>), grid, block, 0, st, a, r, sign);      \
  else hipLaunchKernelGGL((qk_rotary_small_fwd_kernel<T, VEC, LP, false, NT>), grid, block, 0, st, a, r, sign)
    if constexpr (sizeof(T) * VEC == 16) {
      switch (l.chunks) { case 2: BM_S(2); break; case 4: BM_S(4); break; default: BM_S(8); }
    }
#undef BM_S
    return;
  }
#define BM_L(LP) hipLaunchKernelGGL((qk_rotary_fwd_kernel<T, VEC, LP, NT>), grid, block, 0, st, a, r, sign)
  if (!norm) BM_L(0);
  else switch (l.pow2) {
    case 1: BM_L(1); break; case 2: BM_L(2); break; case 4: BM_L(4); break;
    case 8: BM_L(8); break; case 16: BM_L(16); break; default: BM_L(32);
  }
#undef BM_L
}

template <typename T, int VEC, bool NT>
void launch_bwd(const RotaryArgs& a, const Rotation& r, const Lanes& l, const BwdGrid& g, hipStream_t st) {
  const dim3 grid(g.x, g.y), block(256);
  if (l.small) {
#define BM_S(LP) hipLaunchKernelGGL((qk_rotary_small_norm_bwd_kernel<T, VEC, LP, NT>), grid, block, 0, st, a, r)
    if constexpr (sizeof(T) * VEC == 16) {
      switch (l.chunks) { case 2: BM_S(2); break; case 4: BM_S(4); break; default: BM_S(8); }
    }
#undef BM_S
    return;
  }
#define BM_L(LP) hipLaunchKernelGGL((qk_rotary_norm_bwd_kernel<T, VEC, LP, NT>), grid, block, 0, st, a, r)
  switch (l.pow2) {
    case 1: BM_L(1); break; case 2: BM_L(2); break; case 4: BM_L(4); break;
    case 8: BM_L(8); break; case 16: BM_L(16); break; default: BM_L(32);
  }
#undef BM_L
}

#define BM_DISPATCH(D, L, PAST, FN, ...)                                                            \
  if ((D).dtype == BM_DTYPE_FP32) {                                                                 \
    if (PAST) FN<float, 4, true>(__VA_ARGS__); else FN<float, 4, false>(__VA_ARGS__);               \
  } else if ((L).vec == 8) {                                                                        \
    if (PAST) FN<bf16_t, 8, true>(__VA_ARGS__); else FN<bf16_t, 8, false>(__VA_ARGS__);             \
  } else {                                                                                          \
    FN<bf16_t, 4, false>(__VA_ARGS__);                                                              \
  }

// forward, and the gradient without the norm (sign -1)
bm_status turn(const bm_qk_rotary_desc& d, RotaryArgs a, bool norm, float sign, hipStream_t st) {
  const Lanes l = lanes_of(d);
  int groups;
  deal_heads(d, (long)a.T * (norm ? l.pow2 : l.chunks), &a, &groups);
  const Rotation r = rotation(d);
  const bool past = past_caches(d, l, a.T);
  BM_DISPATCH(d, l, past, launch_fwd, a, r, l, norm, sign, groups, st)
  BM_CHECK_LAUNCH("qk_rotary");
  return BM_OK;
}

constexpr int MAX_TOKENS = 1 << 26;      // a grid of 32 lanes per token stays below 2^31 workitems

}  // namespace

}  // namespace bm

using namespace bm;

extern "C" bm_status bm_qk_rotary_forward(const bm_qk_rotary_desc* d, int32_t T, const void* q, const void* k, int32_t ld,
                                          const int32_t* positions, const void* q_gain, const void* k_gain, void* q_out,
                                          void* k_out, int32_t ld_out, void* hip_stream) {
  BM_RETURN_IF(check(d));
  BM_ARG_CHECK(T >= 0 && T <= MAX_TOKENS, "qk rotary: %d tokens", T);
  if (T == 0) return BM_OK;
  BM_RETURN_IF(check_rows(*d, "input", q, k, ld));
  BM_RETURN_IF(check_rows(*d, "output", q_out, k_out, ld_out));
  BM_ARG_CHECK(positions && al16(positions), "qk rotary: positions NULL or misaligned");
  if (d->norm)
    BM_ARG_CHECK((!d->n_q_heads || (q_gain && al16(q_gain))) && (!d->n_kv_heads || (k_gain && al16(k_gain))),
                 "qk rotary: gain NULL or misaligned");
  else
    BM_ARG_CHECK(!q_gain && !k_gain, "qk rotary: gains without norm");
  BM_ARG_CHECK((q != q_out || !d->n_q_heads || ld == ld_out) && (k != k_out || !d->n_kv_heads || ld == ld_out),
               "qk rotary: in place with another row stride");
  RotaryArgs a{};
  a.in[0] = a.x[0] = q; a.in[1] = a.x[1] = k;
  a.out[0] = q_out; a.out[1] = k_out;
  a.gain[0] = q_gain; a.gain[1] = k_gain;
  a.positions = positions;
  a.ld_x = a.ld_in = ld; a.ld_out = ld_out;
  a.T = T; a.dh = d->head_dim; a.eps = d->eps;
  hipStream_t st = (hipStream_t)hip_stream;
  ProfScope prof(PROF_ELEMENTWISE, 2.0 * T * (d->n_q_heads + d->n_kv_heads) * d->head_dim * elt_size(d->dtype), st);
  return turn(*d, a, d->norm != 0, 1.f, st);
}

extern "C" size_t bm_qk_rotary_backward_scratch_bytes(const bm_qk_rotary_desc* d, int32_t T) {
  if (check(d) != BM_OK || T < 1 || T > MAX_TOKENS || !d->norm) return 0;
  // the same for every T: no grid has more workgroups
  const int slots = std::max(BWD_WORKGROUPS, std::min(d->n_q_heads + d->n_kv_heads, MAX_WALKS) + 1);
  return align_up((size_t)slots * d->head_dim * sizeof(float), 256);
}

extern "C" bm_status bm_qk_rotary_backward(const bm_qk_rotary_desc* d, int32_t T, const void* q, const void* k, int32_t ld,
                                           const int32_t* positions, const void* q_gain, const void* k_gain,
                                           const void* dq_out, const void* dk_out, int32_t ld_dout, void* dq, void* dk,
                                           int32_t ld_dqk, float* dq_gain, float* dk_gain, void* scratch,
                                           size_t scratch_bytes, void* hip_stream) {
  BM_RETURN_IF(check(d));
  BM_ARG_CHECK(T >= 0 && T <= MAX_TOKENS, "qk rotary: %d tokens", T);
  if (T == 0) return BM_OK;
  BM_RETURN_IF(check_rows(*d, "gradient", dq_out, dk_out, ld_dout));
  BM_RETURN_IF(check_rows(*d, "output", dq, dk, ld_dqk));
  BM_ARG_CHECK(positions && al16(positions), "qk rotary: positions NULL or misaligned");
  BM_ARG_CHECK((dq != dq_out || !d->n_q_heads || ld_dqk == ld_dout) && (dk != dk_out || !d->n_kv_heads || ld_dqk == ld_dout),
               "qk rotary: in place with another row stride");
  RotaryArgs a{};
  a.in[0] = dq_out; a.in[1] = dk_out;
  a.out[0] = dq; a.out[1] = dk;
  a.positions = positions;
  a.ld_in = ld_dout; a.ld_out = ld_dqk;
  a.T = T; a.dh = d->head_dim; a.eps = d->eps;
  hipStream_t st = (hipStream_t)hip_stream;
  const double bytes = (d->norm ? 3.0 : 2.0) * T * (d->n_q_heads + d->n_kv_heads) * d->head_dim * elt_size(d->dtype);
  if (!d->norm) {
    BM_ARG_CHECK(!q_gain && !k_gain && !dq_gain && !dk_gain, "qk rotary: gains without norm");
    ProfScope prof(PROF_ELEMENTWISE, bytes, st);
    return turn(*d, a, false, -1.f, st);
  }
  BM_RETURN_IF(check_rows(*d, "input", q, k, ld));
  BM_ARG_CHECK((!d->n_q_heads || (q_gain && al16(q_gain) && dq_gain && al16(dq_gain))) &&
               (!d->n_kv_heads || (k_gain && al16(k_gain) && dk_gain && al16(dk_gain))), "qk rotary: gain NULL or misaligned");
  BM_ARG_CHECK((dq != q || !d->n_q_heads || ld_dqk == ld) && (dk != k || !d->n_kv_heads || ld_dqk == ld),
               "qk rotary: in place with another row stride");
  BM_ARG_CHECK(al16(scratch), "qk rotary: misaligned scratch");
  const size_t need = bm_qk_rotary_backward_scratch_bytes(d, T);
  if (!scratch || scratch_bytes < need) {
    set_error("qk rotary: scratch of %zu bytes, %zu needed", scratch ? scratch_bytes : (size_t)0, need);
    return BM_ERR_WORKSPACE_TOO_SMALL;
  }
  const BwdGrid g = bwd_grid(*d, T, &a);
  a.x[0] = q; a.x[1] = k; a.ld_x = ld;
  a.gain[0] = q_gain; a.gain[1] = k_gain;
  a.part[0] = (float*)scratch;
  a.part[1] = a.part[0] + (size_t)g.slots[0] * a.dh;
  const Lanes l = lanes_of(*d);
  const Rotation r = rotation(*d);
  ProfScope prof(PROF_ELEMENTWISE, bytes, st);
  const bool past = past_caches(*d, l, T);
  BM_DISPATCH(*d, l, past, launch_bwd, a, r, l, g, st)
  BM_CHECK_LAUNCH("qk_rotary_bwd");
  ColumnSums sums;
  if (d->n_q_heads) BM_RETURN_IF(sums.add(a.part[0], g.slots[0], a.dh, a.dh, dq_gain));
  if (d->n_kv_heads) BM_RETURN_IF(sums.add(a.part[1], g.slots[1], a.dh, a.dh, dk_gain));
  return flush_column_sums(&sums, st);
}
