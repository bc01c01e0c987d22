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

// the first key that the window of the queries from `at` on holds
__host__ __device__ inline int window_begin(const LocalMask& w, int at) { return at >= w.window ? at - w.window + 1 : 0; }
// a row to read in place of key j: rows that no query from the one with this `begin` on sees are left alone
__device__ inline int seen_row(const LocalMask& w, int begin, int j) { return j < w.sinks || j > begin ? j : begin; }

// Few queries per sequence: the key tiles of every sequence are cut into about equal parts of at most `per` tiles, a workgroup for each
// part and kv head.  Parts number from 0 in pack order; those of sequences with more than one, which leave fp32 sums for
// window_join_kernel, have places numbered from 0 as well:
// sums [place][kv head][rows][dh] and stats [place][kv head][rows] (maximum in base 2, sum).
constexpr int TOKEN_KEYS = 32;       // keys of a tile
constexpr int TOKEN_ROWS = 32;       // queries x heads of a group, at most
constexpr int TOKEN_TABLE = 64;
struct TokenSplit {
  int per, rows, wgs, same_xcd, stream;       // rows: of the sequence with most queries
  float *sums, *stats;
  int n;                             // sequences whose parts stand below (0: more than the table holds, see map)
  // written by window_map_kernel: [S+1] first part and [S] first place of a sequence, [S] those of more than one part, [parts] the sequence
  int32_t* map;
  uint16_t parts[TOKEN_TABLE];
  __host__ __device__ inline int count(const LocalMask& w, int Lq, int Lk) const {
    return Lq > 0 ? (KeyWalk<TOKEN_KEYS>(w, Lk - Lq, 0, Lq, Lk).n + per - 1) / per : 0;
  }
};
// which part and kv head a workgroup takes (they go round-robin over the 8 XCDs), and how many there are
__device__ inline int token_slot(const TokenSplit& t, int Hkv, int block, int* hk) {
  const int id = t.same_xcd ? block >> 3 : block;
  *hk = id % Hkv;
  return t.same_xcd ? id / Hkv * 8 + (block & 7) : id / Hkv;
}
inline int token_grid(const TokenSplit& t, int Hkv) { return t.same_xcd ? cdiv(t.wgs, 8 * Hkv) * 8 * Hkv : t.wgs; }
struct TokenPart { int seq, part, parts, place; };
// sums of v over the lanes up to this one
__device__ inline int scan_lanes(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int x = __shfl_up(v, d, 64);
    v += lane >= d ? x : 0;
  }
  return v;
}
// the parts of a sequence, of those in front of it and their places, from the table: a lane for each sequence
__device__ inline TokenPart table_entry(int seq, int mine, int upto, int places) {
  const int parts = __builtin_amdgcn_readlane(mine, seq), before = __builtin_amdgcn_readlane(upto, seq) - parts;
  return TokenPart{seq, before, parts, __builtin_amdgcn_readlane(places, seq) - (parts > 1 ? parts : 0)};
}
// part `id` in pack order (wave-uniform)
__device__ inline bool find_token_part(const TokenSplit& t, int S, int id, TokenPart* p) {
  if (t.n) {
    const int lane = threadIdx.x & 63, mine = lane < t.n ? t.parts[lane] : 0;
    const int upto = scan_lanes(mine), places = scan_lanes(mine > 1 ? mine : 0);
    const uint64_t past = __builtin_amdgcn_ballot_w64(id < upto);
    if (past == 0) return false;
    *p = table_entry(__builtin_ctzll(past), mine, upto, places);
  } else {
    if (id >= t.map[S]) return false;
    const int seq = t.map[3 * S + 1 + id], before = t.map[seq];
    *p = TokenPart{seq, before, t.map[seq + 1] - before, t.map[S + 1 + seq]};
  }
  p->part = id - p->part;
  p->place += p->part;
  return true;
}
// the j-th sequence of more than one part, and the place of its first
__device__ inline TokenPart split_sequence(const TokenSplit& t, int S, int j) {
  if (!t.n) {
    const int seq = t.map[2 * S + 1 + j], before = t.map[seq];
    return TokenPart{seq, before, t.map[seq + 1] - before, t.map[S + 1 + seq]};
  }
  const int lane = threadIdx.x & 63, mine = lane < t.n ? t.parts[lane] : 0, many = mine > 1;
  const int nth = scan_lanes(many), upto = scan_lanes(mine), places = scan_lanes(many ? mine : 0);
  return table_entry(__builtin_ctzll(__builtin_amdgcn_ballot_w64(many && nth == j + 1)), mine, upto, places);
}

// Tiles of `rows` rows in front of a sequence, for packs of more sequences than a table holds: 64 sequences at a time, a lane for each.
// Later tiles of a sequence come first.
__device__ inline bool find_tile_by_lanes(const int32_t* __restrict__ begin, const int32_t* __restrict__ end, int S, int rows, int id,
                                          int* seq, int* tile, int* ntiles) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < S; s0 += 64) {
    const int s = min(s0 + lane, S - 1), mine = s0 + lane < S ? (end[s] - begin[s] + rows - 1) / rows : 0;
    const int upto = scan_lanes(mine);
    const uint64_t past = __builtin_amdgcn_ballot_w64(id < upto);
    if (past != 0) {
      const int l = __builtin_ctzll(past), n = __builtin_amdgcn_readlane(mine, l);
      *seq = s0 + l;
      *tile = __builtin_amdgcn_readlane(upto, l) - 1 - id;     // n - 1 - (id - tiles in front)
      *ntiles = n;
      return true;
    }
    id -= __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

}  // namespace bm
