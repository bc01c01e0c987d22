// Entry points of attention with a sliding window and first tokens that stay visible: argument checks, and the choice
// between the matrix-core kernels and those in plain fp32 arithmetic.
#include "common.h"
#include "../../include/bigmac_window_attention.h"

#include <algorithm>

namespace bm {

bool attention_mfma_supported(const AttnArgs& a);
size_t window_backward_mfma_scratch_bytes(int window, int sinks, int Hq, int Hkv, int dh, int S, int Tq, int Tk);
bm_status window_forward_mfma(const AttnArgs& a, void* o, float* lse, hipStream_t st);
bm_status window_backward_mfma(const AttnArgs& a, const void* o, const void* d_o, const float* lse, void* dq, void* dk,
                               void* dv, int ld_dq, void* scratch, hipStream_t st);

namespace {

constexpr int MAX_ROWS = 1 << 28;        // offsets of rows stay far from 2^31

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
  BM_ARG_CHECK(ld_q >= (long)Hq * dh && ld_q % vec == 0, "window attention: query row stride %d", ld_q);
  BM_ARG_CHECK(ld_kv >= (long)Hkv * dh && ld_kv % vec == 0, "window attention: key/value row stride %d", ld_kv);
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
  // grids stay below 2^32 threads
  BM_ARG_CHECK((long)c.cu_q_host[S] * Hq < (1L << 28) && (long)rows * Hkv < (1L << 28),
               "window attention: %d queries of %d heads and %d keys of %d (rows x heads below 2^28)", c.cu_q_host[S], Hq, rows, Hkv);
  a->dtype = dtype; a->causal = 1; a->Hq = Hq; a->Hkv = Hkv; a->dh = dh;
  a->ld_qkv = ld_q; a->cu_dev = c.cu_q_dev; a->cu_host = c.cu_q_host; a->S = S; a->T = c.cu_q_host[S]; a->max_seqlen = max_q;
  a->cu_k_dev = own ? c.k_begin_dev : c.cu_q_dev; a->cu_k_host = kb; a->Tk = rows; a->ld_kv = ld_kv; a->max_klen = max_k;
  a->local = LocalMask{std::min(window, MAX_ROWS), sinks, own ? c.k_end_dev : c.cu_q_dev + 1};
  a->key_end_host = ke;
  return BM_OK;
}

bool mfma_head(int dtype, int dh) { return dtype == BM_DTYPE_BF16 && (dh == 64 || dh == 72 || dh == 128); }

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
  return 0;
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
  if (mfma_head(dtype, dh)) return window_forward_mfma(a, o, lse, st);
  return attention_forward_generic(a, o, lse, st);
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
  BM_RETURN_IF(check_scratch(scratch, scratch_bytes,
                             bm_window_attention_backward_scratch_bytes(dtype, window, sinks, Hq, Hkv, dh, S, a.T, a.Tk)));
  a.q = q; a.k = k; a.v = v; a.ld_dkv = ld_dkv;
  hipStream_t st = (hipStream_t)hip_stream;
  ProfScope prof(PROF_ATTN_BWD, 10.0 * dh * Hq * pairs, st);
  if (mfma_head(dtype, dh)) return window_backward_mfma(a, o, d_o, lse, dq, dk, dv, ld_dq, scratch, st);
  return attention_backward_generic(a, o, d_o, lse, dq, dk, dv, ld_dq, (float*)scratch, st);
}
