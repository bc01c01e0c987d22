// Sliding windows (LocalMask): which key tiles a tile of queries walks, and how few queries are split over their keys.
#pragma once
#include "common.h"

namespace bm {

// The key tiles of FKT rows that a tile of query rows walks -- those of the first tokens, then those from its first query's
// window to its last query.  Queries stand at `off` + their row.
template <int FKT>
struct KeyWalk {
  int sinks, near, n;                // tiles of first tokens in front of the window, the window's first tile, tiles in all
  __host__ __device__ inline KeyWalk(const LocalMask& w, int off, int q0, int rows, int Lk) {
    const int end = off + q0 + rows, kend = Lk < end ? Lk : end, begin = off + q0 - w.window + 1;
    near = (begin > 0 ? begin : 0) / FKT;
    sinks = ((w.sinks < kend ? w.sinks : kend) + FKT - 1) / FKT;
    sinks = sinks < near ? sinks : near;
    n = (kend + FKT - 1) / FKT + sinks - near;
  }
  __host__ __device__ inline int tile(int t) const { return t >= sinks ? t - sinks + near : t; }
};
__device__ inline bool hidden(const LocalMask& w, int key, int at) {
  return key > at || (at - key >= w.window && key >= w.sinks);
}
// the running maximum before the first visible key: finite, so that masked scores (-inf) of a first tile give 0
constexpr float NO_MAX = -3e38f;

// Few queries per sequence: the key tiles of every sequence are cut into parts of `per` tiles, a workgroup for each part and kv
// head.  Parts number from 0 in pack order; a sequence of more than one leaves fp32 sums for window_join_kernel:
// sums [part][kv head][rows][dh] and stats [part][kv head][rows] (maximum in base 2, sum).
constexpr int TOKEN_KEYS = 32;       // keys of a tile
constexpr int TOKEN_ROWS = 32;       // queries x heads of a group, at most
struct TokenSplit {
  int per, rows, wgs;                // rows: of the sequence with most queries
  float *sums, *stats;
  int n;                             // sequences whose parts stand below (0: they are counted on the device)
  uint16_t parts[64];
  __host__ __device__ inline int count(const LocalMask& w, int Lq, int Lk) const {
    return Lq > 0 ? (KeyWalk<TOKEN_KEYS>(w, Lk - Lq, 0, Lq, Lk).n + per - 1) / per : 0;
  }
};
__device__ inline int token_parts(const TokenSplit& t, const LocalMask& w, const int32_t* __restrict__ cu,
                                  const int32_t* __restrict__ cuk, int s) {
  return t.n ? t.parts[s] : t.count(w, cu[s + 1] - cu[s], w.key_end[s] - cuk[s]);
}
__device__ inline bool find_token_part(const TokenSplit& t, const LocalMask& w, const int32_t* __restrict__ cu,
                                       const int32_t* __restrict__ cuk, int S, int id, int* seq, int* part, int* parts) {
  for (int s = 0; s < S; ++s) {
    const int n = token_parts(t, w, cu, cuk, s);
    if (id < n) { *seq = s; *part = id; *parts = n; return true; }
    id -= n;
  }
  return false;
}

}  // namespace bm
