// Variable-length flash attention on the gfx950 matrix cores (bf16 in, fp32
// accumulate, online softmax in base 2), forward and backward.
//
// Packing: a workgroup owns one tile of 128 or 256 rows of ONE sequence and one head, so
// attention is block-diagonal by construction; tiles are enumerated by walking
// cu_seqlens (no padded grid), longest-running tiles first.
//
// Layout trick.  All score matrices are produced TRANSPOSED by the MFMA
// (keys x queries for forward/dQ, queries x keys for dK/dV), so that the
// softmax statistic of a row lives in ONE lane (two lanes for the two 32-lane
// halves) instead of being spread over a wavefront, and the fp32 accumulator
// of one MFMA is -- after conversion to bf16 -- exactly the B operand of the
// next MFMA (P feeds P*V, dS feeds dS*K / dS*Q): probabilities never touch LDS.
// The matching A operands (V^T, K^T, Q^T, dO^T) come from the LDS transpose
// read (ds_read_b64_tr_b16) of tiles stored in their natural [row][dh] form.
// Tiles are XOR-swizzled with a pattern that is conflict-free for both the
// 16-byte row reads and the transpose reads.
//
// Backward is split in two kernels (dK/dV per key tile, dQ per query tile),
// each recomputing P from the saved log-sum-exp: every output element has one
// owner, so there are no floating-point atomics and results are reproducible.
#include "common.h"
#include "attn_window.h"

#include <type_traits>

namespace bm {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// Head sizes: 64 and 128 fit the 32x32x16 MFMA exactly; 72 (the DiT blocks) is run
// with its contraction padded to 80 and its output rows padded to 96 by zero chunks
// that exist only in LDS and registers, never in HBM.
template <int DH>
struct HeadDim {
  static constexpr int KS = (DH + 15) / 16;    // k=16 steps when dh is the contraction index
  static constexpr int NB = (DH + 31) / 32;    // 32-row blocks when dh is an output index
  static constexpr int DHL = NB * 32;          // LDS row width in elements
  static constexpr int VCH = DH / 8;           // 16-byte chunks of a row that hold data
};

// ---- swizzled [rows][DHL] bf16 tile -----------------------------------------
template <int DHL>
__device__ inline int tile_swizzle(int row) {      // chunk c of a row sits in slot c ^ tile_swizzle(row)
  if (DHL == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
  if (DHL == 96) return (row >> 2) & 3;
  const int v = row >> 1;
  return ((v & 1) << 2) | ((v >> 1) & 3);
}
template <int DHL>
__device__ inline int tile_off(int row, int c) {   // element offset of 16-byte chunk c of a row
  return row * DHL + ((c ^ tile_swizzle<DHL>(row)) << 3);
}

// 8 consecutive dh values (chunk c) of a global row as an MFMA operand; zeros past dh
template <int DH>
__device__ inline bf16x8 load_chunk(const bf16_t* row, int c) {
  if (DH % 16 == 0 || c < HeadDim<DH>::VCH) return *reinterpret_cast<const bf16x8*>(row + c * 8);
  bf16x8 z;
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = (bf16_t)0.f;
  return z;
}

// operand fragment, rows of the tile are the MFMA row/col index, dh is the k index:
// lane l -> tile row row0 + l%32, dh = ks*16 + (l/32)*8 .. +7
template <int DH>
__device__ inline bf16x8 frag_rows(const bf16_t* t, int row0, int ks, int lane) {
  return *reinterpret_cast<const bf16x8*>(t + tile_off<DH>(row0 + (lane & 31), ks * 2 + (lane >> 5)));
}

// A operand X^T: MFMA row = dh index col0 + l%32, k index = tile rows, in the
// order the fp32 accumulator of a transposed score block hands them over:
// half h = l/32 supplies tile rows r0+4h..+3 and r0+8+4h..+3.
template <int DH>
__device__ inline bf16x8 frag_cols(const bf16_t* t, int col0, int r0, int lane) {
  const int gi = lane >> 4, s = lane & 15;
  const int col = col0 + (gi & 1) * 16 + (s & 3) * 4;
  const int row = r0 + (gi >> 1) * 4 + (s >> 2);
  const bf16_t* p0 = t + tile_off<DH>(row, col >> 3) + (col & 7);
  const bf16_t* p1 = t + tile_off<DH>(row + 8, col >> 3) + (col & 7);
  s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)p0);
  s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)p1);
  union { struct { s16x4 a, b; } s; bf16x8 v; } u;
  u.s.a = lo; u.s.b = hi;
  return u.v;
}

// max / sum of a value with the one held by the lane 32 away (the two halves of a wavefront own
// the same score column): v_permlane32_swap exchanges the halves in the vector unit, without the
// trip through the LDS crossbar that a lane shuffle takes
__device__ inline float max_with_other_half(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_with_other_half(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// accumulator rows 8t..8t+7 of a 32x32 block -> bf16 B operand of a k=16 step
__device__ inline bf16x8 acc_to_operand(const f32x16& a, int t) {
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (bf16_t)a[t * 8 + e];
  return r;
}

__device__ inline const bf16_t* scalar_ptr(const void* p) {
  const uint64_t b = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const bf16_t*>(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32)) << 32) |
                                         (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b));
}

// ---- global -> LDS: a [ROWS][DH] tile brought in by NT threads -------------------
// 16-byte loads that write LDS directly (no registers, no LDS store
// instructions): lane l of a wavefront fills bytes [16 l, 16 l + 16) of a 1 KiB run of slots, so the
// swizzle is applied on the global side -- the lane that owns slot s of a row fetches chunk
// s ^ tile_swizzle(row).  Padding slots (head sizes that are no multiple of 32) are never written
// by a load: zero() clears them once.  The loads are asynchronous: wait for vmcnt(0), then a
// workgroup barrier, before any wavefront reads the tile.
template <int ROWS, int DH, int NT, bool STREAM = false>
struct TileAsync {
  static constexpr int DHL = HeadDim<DH>::DHL;
  static constexpr int CPR = DHL / 8;
  static constexpr int SLOTS = ROWS * CPR;
  static constexpr int CH = (SLOTS + NT - 1) / NT;    // loads per thread (the last round may be short)
  // UNI: every load of a thread has the same chunk, and rows a fixed distance apart
  static constexpr bool UNI = NT % CPR == 0 && (NT / CPR) % 16 == 0 && SLOTS % NT == 0;
  static constexpr int RSTEP = NT / CPR, NV = UNI ? 1 : CH;
  static_assert(SLOTS % 64 == 0 && NT % 64 == 0, "a tile is a whole number of 1 KiB runs");
  static constexpr bool ALL_LIVE = DHL == DH && SLOTS % NT == 0;   // no padding slot, no short round
  uint32_t goff[NV];    // byte offset of a load from the tile's first row (full tiles)
  int tid_;             // the thread's index among the NT that bring the tile in
  // (row, chunk) of load i; false: it would fill a padding slot or lies past the tile
  __device__ inline bool place(int i, int* row, int* chunk, int tid) const {
    const int id = tid + i * NT;
    *row = id / CPR;
    *chunk = (id % CPR) ^ tile_swizzle<DHL>(*row);
    return ALL_LIVE || (id < SLOTS && *chunk < HeadDim<DH>::VCH);
  }
  __device__ inline void init(int ld, int tid) {
    tid_ = tid;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      int row, c;
      place(i, &row, &c, tid);
      goff[i] = (uint32_t)row * (uint32_t)ld * 2u + (uint32_t)c * 16u;
    }
  }
  // STREAM: past the caches, for data that no other workgroup reads.
  // One 16-byte load per lane straight into LDS.  Written as inline assembly so that the compiler does
  // not see an LDS write in flight: it would otherwise make every LDS read that follows wait for
  // vmcnt(0) and the tile would no longer stream in behind the arithmetic.  The caller orders the
  // reads of a tile after wait_async_tiles() and a barrier.
  static __device__ inline void load16(const void* base, uint32_t voff, uint32_t lds_addr) {
    if constexpr (STREAM)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt"
                   :: "s"(lds_addr), "v"(voff), "s"(base) : "memory", "m0");
    else
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                   :: "s"(lds_addr), "v"(voff), "s"(base) : "memory", "m0");
  }
  // base: first row of the tile (wave-uniform); rows_left: valid rows from there (>= 1), rows beyond
  // them are clamped to the last valid one (their results are masked or unused); wave: wave-uniform
  __device__ inline void issue(const bf16_t* __restrict__ base_in, int ld, int rows_left, bf16_t* t,
                               int wave) const {
    // the base goes into the asm statement as a scalar register pair: say so, wherever the caller's
    // arithmetic left it
    const uint64_t b64 = reinterpret_cast<uint64_t>(base_in);
    const bf16_t* base = reinterpret_cast<const bf16_t*>(
        ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b64 >> 32)) << 32) |
        (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b64));
    rows_left = __builtin_amdgcn_readfirstlane(rows_left);
    const uint32_t dst = (uint32_t)(size_t)(__attribute__((address_space(3))) char*)(t + wave * 512);
    if (rows_left >= ROWS) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        int row, c;
        // (UNI: the distance between a thread's loads goes into the scalar base, not into a register each)
        if (place(i, &row, &c, tid_))
          load16(base + (UNI ? (size_t)(i * RSTEP) * ld : (size_t)0), goff[UNI ? 0 : i], dst + i * NT * 16);
      }
    } else {
      // a cut tile (the last one of a sequence): offsets from scratch, rows clamped.  The thread index
      // passes through an empty asm so that none of this is computed ahead of the loop and kept in
      // registers for the one step that needs it.
      int t_op = tid_;
      asm volatile("" : "+v"(t_op));
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        int row, c;
        if (place(i, &row, &c, t_op))
          load16(base, (uint32_t)min(row, rows_left - 1) * (uint32_t)ld * 2u + (uint32_t)c * 16u, dst + i * NT * 16);
      }
    }
  }
  // the same for the tile of keys from key0 on under a window: rows that no query from the one with this `begin` on sees are not
  // read, but the last of the first tokens or the first row of the window in their place
  __device__ inline void issue(const LocalMask& w, int begin, const bf16_t* __restrict__ keys, int ld, int key0, int Lk, bf16_t* t,
                               int wave) const {
    const int hidden_from = max(key0, w.sinks), instead = key0 < w.sinks ? w.sinks - 1 : begin;
    if (begin <= hidden_from || hidden_from >= key0 + ROWS) return issue(keys + (size_t)key0 * ld, ld, Lk - key0, t, wave);
    const bf16_t* const base = scalar_ptr(keys + (size_t)key0 * ld);
    const uint32_t dst = (uint32_t)(size_t)(__attribute__((address_space(3))) char*)(t + wave * 512);
    int t_op = tid_;
    asm volatile("" : "+v"(t_op));
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      int row, c;
      if (place(i, &row, &c, t_op)) {
        const int j = key0 + row, from = j >= hidden_from && j < begin ? instead : min(j, Lk - 1);
        load16(base, (uint32_t)(from - key0) * (uint32_t)ld * 2u + (uint32_t)c * 16u, dst + i * NT * 16);
      }
    }
  }
  static __device__ inline void zero_padding(bf16_t* t, int tid) {
    if (DHL == DH) return;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int id = tid + i * NT;
      const int r = id / CPR, c = (id % CPR) ^ tile_swizzle<DHL>(r);
      if (id < SLOTS && c >= HeadDim<DH>::VCH) *reinterpret_cast<u32x4*>(t + id * 8) = u32x4{0u, 0u, 0u, 0u};
    }
  }
};
// The tile loads are invisible to the compiler's wait-count bookkeeping, so the wait for them is
// written out as well.  A vmcnt wait that the compiler adds for one of ITS loads would also wait for
// tile loads in flight: settle_compiler_loads() (a wait the bookkeeping does read) goes once in front
// of a loop that streams tiles, after the kernel's ordinary loads, so that none is added inside.
__device__ inline void wait_async_tiles() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ inline void settle_compiler_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); /* vmcnt(0) */ }

// The order in which the tiles of the sequences are handed out: workgroups are dispatched in id
// order, so the sequences whose tiles run longest go first and the short ones fill the tail of the
// launch.  Built on the host from the host copy of the offsets (the same copy that sizes the grid)
// and passed by value in the kernel arguments: nothing to allocate or copy, and a workgroup finds
// its tile from one batch of scalar loads instead of a dependent load per sequence.  Any order
// gives the same results, only the schedule changes.  n == 0: no table (more than 64 sequences),
// the kernel walks the offsets in pack order.
struct SeqOrder {
  int n;                // positions in use, a multiple of 16
  uint32_t w[64];       // position i: sequence index in bits 0..7, its number of tiles above
};

// cu_tiles: offsets of the side that is cut into tiles of `rows` rows; cu_cost: offsets of the side
// a tile loops over (its running time).  sorted = false keeps the pack order: under a causal mask
// a pack has tiles of every length whatever the order, and the long sequences' tiles all running at
// once measured slower (their operands no longer fit the L2 of an XCD together).
// (end: where the sequences end, when rows may lie between them.)
SeqOrder make_seq_order(const int32_t* cu_tiles, const int32_t* cu_cost, int S, int rows, bool sorted, const int32_t* end = nullptr) {
  if (!end) end = cu_tiles + 1;
  SeqOrder o;
  o.n = 0;
  for (int i = 0; i < 64; ++i) o.w[i] = 0;          // unused positions: sequence 0, no tile
  if (S < 1 || S > 64) return o;
  for (int s = 0; s < S; ++s)
    if ((end[s] - cu_tiles[s] + rows - 1) / rows >= (1 << 24)) return o;
  unsigned char idx[64];
  for (int i = 0; i < S; ++i) idx[i] = (unsigned char)i;
  // stable insertion sort by descending length
  for (int i = 1; sorted && i < S; ++i) {
    const unsigned char x = idx[i];
    const int lx = cu_cost[x + 1] - cu_cost[x];
    int j = i;
    while (j > 0 && cu_cost[idx[j - 1] + 1] - cu_cost[idx[j - 1]] < lx) { idx[j] = idx[j - 1]; --j; }
    idx[j] = x;
  }
  o.n = (S + 15) / 16 * 16;
  for (int i = 0; i < S; ++i) {
    const int nt = (end[idx[i]] - cu_tiles[idx[i]] + rows - 1) / rows;
    o.w[i] = ((uint32_t)nt << 8) | idx[i];
  }
  return o;
}

// which (sequence, tile) a linear tile id is; tiles of `rows` rows, later tiles of a
// sequence first (under a causal mask they are the long ones).  Wave-uniform throughout.
__device__ inline bool find_tile(const int32_t* __restrict__ cu, const SeqOrder& ord, int S, int rows, int id,
                                 int* seq, int* tile, int* ntiles) {
  if (ord.n == 0) {
    for (int s = 0; s < S; ++s) {
      const int L = cu[s + 1] - cu[s];
      const int nt = (L + rows - 1) / rows;
      if (id < nt) { *seq = s; *tile = nt - 1 - id; *ntiles = nt; return true; }
      id -= nt;
    }
    return false;
  }
  for (int s0 = 0; s0 < ord.n; s0 += 16) {
    uint32_t e[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) e[j] = ord.w[s0 + j];
    int found = -1, fid = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) {               // branch-free choice among the sixteen
      const int n = (int)(e[j] >> 8);
      const bool here = found < 0 && id < n;
      found = here ? (int)e[j] : found;
      fid = here ? id : fid;
      id -= found < 0 ? n : 0;
    }
    if (found >= 0) {
      const int nt = found >> 8;
      *seq = found & 255; *tile = nt - 1 - fid; *ntiles = nt;
      return true;
    }
  }
  return false;
}

// the same where rows may lie between the sequences, and faster for packs without a table
__device__ inline bool find_tile(const int32_t* __restrict__ begin, const int32_t* __restrict__ end, const SeqOrder& ord, int S,
                                 int rows, int id, int* seq, int* tile, int* ntiles) {
  if (ord.n) return find_tile(begin, ord, S, rows, id, seq, tile, ntiles);
  return find_tile_by_lanes(begin, end, S, rows, id, seq, tile, ntiles);
}

// every tile from the first one on
template <int FKT>
struct AllKeys {
  int n;
  __device__ inline AllKeys(bool causal, int q0, int rows, int Lk) {
    const int kend = causal ? min(Lk, q0 + rows) : Lk;
    n = (kend + FKT - 1) / FKT;
  }
  __device__ inline int tile(int t) const { return t; }
};
// all of the keys key0 .. key0 + n - 1 visible to all of the queries at a .. a + m - 1; none to any of them
__device__ inline bool all_visible(const LocalMask& w, int key0, int n, int a, int m) {
  return key0 + n - 1 <= a && (a + m - 1 - key0 < w.window || key0 + n <= w.sinks);
}
__device__ inline bool none_visible(const LocalMask& w, int key0, int n, int a, int m) {
  return key0 > a + m - 1 || (a - (key0 + n - 1) >= w.window && key0 >= w.sinks);
}
// Scores of NB blocks of 32 keys from key0 on that the query at `ahead` behind key0 + half * 4 does not see become -inf; first_at: the first of the
// wavefront's 32 queries.  Most tiles that need a test need one of the two.
template <int NB>
__device__ inline void hide_scores(const LocalMask& w, int key0, int first_at, int ahead, int half4, f32x16 (&s)[NB]) {
  if (key0 + NB * 32 - 1 > first_at)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[b][r] = b * 32 + (r >> 2) * 8 + (r & 3) > ahead ? -INFINITY : s[b][r];
  if (first_at + 31 - key0 >= w.window && key0 + NB * 32 > w.sinks) {
    const int behind = ahead - w.window, sinks = w.sinks - key0 - half4;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int e = b * 32 + (r >> 2) * 8 + (r & 3);
        s[b][r] = e <= behind && e >= sinks ? -INFINITY : s[b][r];
      }
  }
}
// Linear workgroup id -> (tile id, head).  Heads vary fastest, and since workgroup
// ids go round-robin over the 8 XCDs, head index i lands on XCD i%8: give XCD x
// the consecutive heads x*(H/8).., so every tile of one head -- and the q heads of
// one GQA group -- meet their K/V in the same XCD's L2.
__device__ inline void tile_and_head(int H, int* tile, int* head, int b) {
  const int i = b % H;
  *tile = b / H;
  *head = (H % 8 == 0) ? (i % 8) * (H / 8) + i / 8 : i;
}

// =============================================================================
// forward
// =============================================================================
constexpr int NUM_CU = 256;
constexpr int FQ = 128;   // query rows per workgroup (32 per wavefront)
constexpr int FK = 64;    // keys per step

template <int DH, bool CAUSAL, bool WINDOW>
__global__ __launch_bounds__(256, 2) void fa_fwd_kernel(
    const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v, int ld,
    int ldk, const int32_t* __restrict__ cu, const int32_t* __restrict__ cuk, int S,
    bf16_t* __restrict__ o, int ldo, float* __restrict__ lse, int Ttot, int Hq, int group,
    float scale_log2, SeqOrder ord, LocalMask w) {
  // K and V tiles are double-buffered: tile kt+1 streams into LDS while tile kt is consumed
  constexpr int TILE = FK * HeadDim<DH>::DHL;
  __shared__ __attribute__((aligned(1024))) bf16_t Kbuf[2 * TILE];
  __shared__ __attribute__((aligned(1024))) bf16_t Vbuf[2 * TILE];
  int seq, qt, nqt, tile_id, hq;
  tile_and_head(Hq, &tile_id, &hq, blockIdx.x);
  if (WINDOW ? !find_tile(cu, cu + 1, ord, S, FQ, tile_id, &seq, &qt, &nqt) : !find_tile(cu, ord, S, FQ, tile_id, &seq, &qt, &nqt)) return;
  const int hk = hq / group;
  const int lo = cu[seq], L = cu[seq + 1] - lo;
  // keys and values may be packed on their own (a chunk of a context-parallel partition)
  const int lok = cuk[seq], Lk = (WINDOW ? w.key_end[seq] : cuk[seq + 1]) - lok;
  const int q0 = qt * FQ;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int half = lane >> 5;
  const int qpos = q0 + wave * 32 + (lane & 31);          // this lane's query (column of S^T)
  const int qrow = min(qpos, L - 1);
  if (Lk == 0) {
    // no key in this chunk (workgroup-uniform): zero output, lse = -inf
    if (qpos < L) {
      bf16_t* op = o + (size_t)(lo + qpos) * ldo + hq * DH;
      for (int c = half * (DH / 2); c < (half + 1) * (DH / 2); c += 4) {
        bf16x4 z = {(bf16_t)0.f, (bf16_t)0.f, (bf16_t)0.f, (bf16_t)0.f};
        *reinterpret_cast<bf16x4*>(op + c) = z;
      }
      if (half == 0) lse[(size_t)hq * Ttot + lo + qpos] = -INFINITY;
    }
    return;
  }

  bf16x8 qf[HeadDim<DH>::KS];
  {
    const bf16_t* qp = q + (size_t)(lo + qrow) * ld + hq * DH;
#pragma unroll
    for (int ks = 0; ks < HeadDim<DH>::KS; ++ks) qf[ks] = load_chunk<DH>(qp, ks * 2 + half);
  }
  f32x16 oacc[HeadDim<DH>::NB];
#pragma unroll
  for (int j = 0; j < HeadDim<DH>::NB; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[j][r] = 0.f;
  float m = WINDOW ? NO_MAX : -INFINITY, lsum = 0.f;

  const int off = WINDOW ? Lk - L : 0;
  const auto walk = [&] {
    if constexpr (WINDOW) return KeyWalk<FK>(w, off, q0, FQ, Lk);
    else return AllKeys<FK>(CAUSAL, q0, FQ, Lk);
  }();
  const int nkt = walk.n;
  const bf16_t* kbase = k + (size_t)lok * ldk + hk * DH;
  const bf16_t* vbase = v + (size_t)lok * ldk + hk * DH;
  using Tile = TileAsync<FK, DH, 256>;
  Tile tile;
  tile.init(ldk, tid);
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    Tile::zero_padding(Kbuf + b * TILE, tid);
    Tile::zero_padding(Vbuf + b * TILE, tid);
  }
  const int begin = WINDOW ? window_begin(w, off + q0) : 0;
  auto fetch = [&](const bf16_t* base, int t, bf16_t* dst) {
    if constexpr (WINDOW) tile.issue(w, begin, base, ldk, t * FK, Lk, dst, wave_u);
    else tile.issue(base + (size_t)t * FK * ldk, ldk, Lk - t * FK, dst, wave_u);
  };
  fetch(kbase, walk.tile(0), Kbuf);
  fetch(vbase, walk.tile(0), Vbuf);
  settle_compiler_loads();                 // the Q fragments (and, with them, tile 0)

  // The step comes in two copies, without and with the per-element mask test, each in a loop of
  // its own: the leading key tiles lie wholly inside the sequence (and before the diagonal under a
  // causal mask) and need no test; written as a run-time condition inside the unrolled code, the
  // test becomes compare/select pairs that every step pays for.  Every wavefront runs nkt steps
  // in total (the split may differ between wavefronts; the barrier count per step does not).
  auto step = [&](int kt, auto masked, auto parity) {
    constexpr bool MASKED = decltype(masked)::value;
    constexpr int PAR = decltype(parity)::value;
    const bf16_t* Ks = Kbuf + PAR * TILE;
    const bf16_t* Vs = Vbuf + PAR * TILE;
    // one barrier per step: tile kt has landed for every wavefront, and every wavefront is done
    // with tile kt-1, whose buffer the loads of tile kt+1 overwrite
    wait_async_tiles();
    __syncthreads();
    if (kt + 1 < nkt) {
      fetch(kbase, walk.tile(kt + 1), Kbuf + (1 - PAR) * TILE);
      fetch(vbase, walk.tile(kt + 1), Vbuf + (1 - PAR) * TILE);
    }
    const int key0 = walk.tile(kt) * FK;
    if (WINDOW && MASKED && none_visible(w, key0, FK, off + q0 + wave_u * 32, 32)) return;
    // S^T = K Q^T for both 32-key blocks first: the MFMAs of block 1 run while the
    // softmax arithmetic of block 0 occupies the vector unit, and the P V MFMAs of
    // block 0 run under the softmax of block 1.
    f32x16 sacc[FK / 32];
#pragma unroll
    for (int b = 0; b < FK / 32; ++b) sacc[b] = f32x16{};
    {
      // K fragments are requested from LDS AHEAD MFMAs before their use (a ring of register sets)
      constexpr int KS = HeadDim<DH>::KS, NSTEP = (FK / 32) * KS, AHEAD = 2;
      bf16x8 fk[AHEAD + 1];
#pragma unroll
      for (int n = 0; n < AHEAD && n < NSTEP; ++n) fk[n] = frag_rows<HeadDim<DH>::DHL>(Ks, (n / KS) * 32, n % KS, lane);
#pragma unroll
      for (int n = 0; n < NSTEP; ++n) {
        const int m = n + AHEAD;
        if (m < NSTEP) fk[m % (AHEAD + 1)] = frag_rows<HeadDim<DH>::DHL>(Ks, (m / KS) * 32, m % KS, lane);
        sacc[n / KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[n % (AHEAD + 1)], qf[n % KS], sacc[n / KS], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // mask: keys past the sequence end, and keys after the query under a causal mask
    if constexpr (WINDOW && MASKED) hide_scores<FK / 32>(w, key0, off + q0 + wave_u * 32, off + qpos - key0 - half * 4, half * 4, sacc);
#pragma unroll
    for (int b = 0; b < FK / 32; ++b) {
      float mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (MASKED && !WINDOW) {
          const int key = key0 + b * 32 + (r >> 2) * 8 + half * 4 + (r & 3);
          if (key >= Lk || (CAUSAL && key > qpos)) sacc[b][r] = -INFINITY;
        }
        mx = fmaxf(mx, sacc[b][r]);
      }
      mx = max_with_other_half(mx) * scale_log2;
      // Lazy rescaling: the running maximum only moves (and O, l are only rescaled)
      // when some row's maximum grew by more than 2^8; until then probabilities are
      // taken relative to the older maximum (they stay below 2^8, exact in fp32).
      if (__builtin_amdgcn_ballot_w64(mx > m + 8.0f) != 0) {
        const float m_new = fmaxf(m, mx);
        const float corr = __builtin_amdgcn_exp2f(m - m_new);   // m = -inf at the start: 0
        m = m_new;
        lsum *= corr;
#pragma unroll
        for (int j = 0; j < HeadDim<DH>::NB; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[j][r] *= corr;
      }
      float psum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sacc[b][r], scale_log2, -m));   // masked: exp2(-inf) = 0
        sacc[b][r] = p;
        psum += p;
      }
      lsum += psum;
      const bf16x8 p0 = acc_to_operand(sacc[b], 0), p1 = acc_to_operand(sacc[b], 1);
      // O^T += V^T P^T, the transposed V operands requested one pair of MFMAs ahead
      {
        constexpr int NB = HeadDim<DH>::NB;
        bf16x8 fr[2][2];
        fr[0][0] = frag_cols<HeadDim<DH>::DHL>(Vs, 0, b * 32, lane);
        fr[0][1] = frag_cols<HeadDim<DH>::DHL>(Vs, 0, b * 32 + 16, lane);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          if (j + 1 < NB) {
            fr[(j + 1) & 1][0] = frag_cols<HeadDim<DH>::DHL>(Vs, (j + 1) * 32, b * 32, lane);
            fr[(j + 1) & 1][1] = frag_cols<HeadDim<DH>::DHL>(Vs, (j + 1) * 32, b * 32 + 16, lane);
          }
          oacc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[j & 1][0], p0, oacc[j], 0, 0, 0);
          oacc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[j & 1][1], p1, oacc[j], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  };
  // tiles kt < n_plain need no test: key0 + FK <= Lk, and key0 + FK - 1 <= this wavefront's first query
  int n_plain = Lk / FK;
  if (CAUSAL) n_plain = min(n_plain, (q0 + wave * 32 + 1) / FK);
  n_plain = min(n_plain, nkt);
  using P0 = std::integral_constant<int, 0>;
  using P1 = std::integral_constant<int, 1>;
  for (int kt = 0; kt < nkt; ++kt) {
    const bool plain = WINDOW ? all_visible(w, walk.tile(kt) * FK, FK, off + q0 + wave_u * 32, 32) : kt < n_plain;
    if (kt & 1) { if (plain) step(kt, std::false_type{}, P1{}); else step(kt, std::true_type{}, P1{}); }
    else { if (plain) step(kt, std::false_type{}, P0{}); else step(kt, std::true_type{}, P0{}); }
  }
  lsum = sum_with_other_half(lsum);
  if (qpos < L) {
    const float inv = 1.0f / lsum;
    bf16_t* op = o + (size_t)(lo + qpos) * ldo + hq * DH;
#pragma unroll
    for (int j = 0; j < HeadDim<DH>::NB; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (bf16_t)(oacc[j][g * 4 + e] * inv);
        if (DH % 32 == 0 || j * 32 + g * 8 + half * 4 < DH)
          *reinterpret_cast<bf16x4*>(op + j * 32 + g * 8 + half * 4) = w;
      }
    if (half == 0) lse[(size_t)hq * Ttot + lo + qpos] = (m + log2f(lsum)) * LN2;
  }
}

// ---- tiles whose reads are one lane constant plus an immediate offset (head sizes 64 and 128) ----------
// A run of 512 / DH rows is the 1 KiB that one load instruction of a wavefront fills.  In a run, 64-byte groups of
// four chunks lie row after row, and the runs are PAD bytes apart from each other, so that row reads and transpose
// reads are free of bank conflicts; for 64, the lowest bit of the chunk is turned in every second four rows.
template <int DH>
struct RunTile {
  static constexpr int RPR = 512 / DH, RUN = 1024 + (DH == 128 ? 16 : 32);
  static constexpr int bytes(int rows) { return rows / RPR * RUN; }
  // this lane's row (in the run) and 16-byte chunk in a load
  static __device__ inline int load_row(int l) { return (l >> 2) & (RPR - 1); }
  static __device__ inline int load_chunk(int l) {
    return DH == 128 ? (l >> 4) * 4 + (l & 3) : (l >> 5) * 4 + ((l & 3) ^ ((l >> 4) & 1));
  }
  // operand with rows as MFMA rows: lane l holds row l % 32 of a block, dh = ks * 16 + (l / 32) * 8 .. + 7
  static __device__ inline int rows_at(int l) {
    const int r = l & 31, half = l >> 5;
    return r / RPR * RUN + (r & (RPR - 1)) * 64 + (DH == 128 ? half : half ^ ((r >> 2) & 1)) * 16;
  }
  static constexpr int rows_imm(int block, int ks) { return block * (32 / RPR) * RUN + (ks >> 1) * (RPR * 64) + (ks & 1) * 32; }
  // transposed operand: MFMA row = dh index j * 32 + l % 32, k index = tile rows r16 * 16 .. (see frag_cols)
  static __device__ inline int cols_at(int l) {
    const int gi = l >> 4, s = l & 15, c = (gi & 1) * 2 + ((s & 3) >> 1);
    return DH == 128 ? (gi >> 1) * RUN + (s >> 2) * 64 + c * 16 + (s & 1) * 8
                     : ((gi >> 1) * 4 + (s >> 2)) * 64 + (c ^ (gi >> 1)) * 16 + (s & 1) * 8;
  }
  static constexpr int cols_imm(int j, int r16) { return j * (RPR * 64) + r16 * (16 / RPR) * RUN; }
  static __device__ inline bf16x8 read_rows(const unsigned char* base, int block, int ks) {
    return *reinterpret_cast<const bf16x8*>(base + rows_imm(block, ks));
  }
  static __device__ inline bf16x8 read_cols(const unsigned char* base, int j, int r16) {
    const unsigned char* a = base + cols_imm(j, r16);
    s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)a);
    s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(a + 8 / RPR * RUN));
    union { struct { s16x4 a, b; } s; bf16x8 v; } u;
    u.s.a = lo; u.s.b = hi;
    return u.v;
  }
};

// end of a phase: this wavefront's LDS accesses are done, then the workgroup meets
__device__ inline void phase_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Forward with two groups of wavefronts that take turns (head sizes 64 and 128, long sequences): wavefronts w and
// w + 4 share a SIMD, and while one multiplies -- P V of a key tile, then Q K of the next -- the other one does
// the softmax of its tile.  Left to themselves (two workgroups of four wavefronts), two wavefronts of a SIMD
// often want the same unit: matrix pipe busy 50 % of the cycles at head size 128, vector unit 56 %.
// Two workgroups of four wavefronts -> this, us: 4 x 4096 bidirectional, 16 heads of 128, 577 -> 482 (1140 TFLOP/s), of
// 64, 369 -> 330; 32768 tokens of causal documents, 32 / 8 heads of 128, 2914 -> 2501; 16 samples of about 1130, 24 heads,
// 360 -> 327.  Bound by the vector unit at head size 64 (78 % busy before) and by power at 128.
constexpr int AQ = 256;   // query rows per workgroup

template <int DH, bool CAUSAL>
__global__ __launch_bounds__(512, 2) void fa_fwd_alt_kernel(
    const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v, int ld,
    int ldk, const int32_t* __restrict__ cu, const int32_t* __restrict__ cuk, int S,
    bf16_t* __restrict__ o, int ldo, float* __restrict__ lse, int Ttot, int Hq, int group,
    float scale_log2, SeqOrder ord) {
  using RT = RunTile<DH>;
  constexpr int KS = DH / 16, NB = DH / 32, KBL = FK / 32, TILE = RT::bytes(FK), RUNS = FK / RT::RPR / 8;
  constexpr int RING = 3;
  __shared__ __attribute__((aligned(1024))) unsigned char Kbuf[RING * TILE];
  __shared__ __attribute__((aligned(1024))) unsigned char Vbuf[RING * TILE];
  int seq, qt, nqt, tile_id, hq;
  tile_and_head(Hq, &tile_id, &hq, blockIdx.x);
  if (!find_tile(cu, ord, S, AQ, tile_id, &seq, &qt, &nqt)) return;
  const int hk = hq / group;
  const int lo = cu[seq], L = cu[seq + 1] - lo;
  const int lok = cuk[seq], Lk = cuk[seq + 1] - lok;
  const int q0 = qt * AQ;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qfirst = q0 + wave * 32;
  const int qpos = qfirst + (lane & 31);                  // this lane's query (column of S^T)
  bf16x8 qf[KS];
  {
    const bf16_t* qp = q + (size_t)(lo + min(qpos, L - 1)) * ld + hq * DH;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = load_chunk<DH>(qp, ks * 2 + half);
  }
  f32x16 oacc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) oacc[j] = f32x16{};
  float m = -INFINITY, lsum = 0.f;
  // key tiles of the workgroup, and those of this wavefront (none if its queries lie past the sequence)
  const int nkt = ((CAUSAL ? min(Lk, q0 + AQ) : Lk) + FK - 1) / FK;
  const int mine = qfirst >= L ? 0 : CAUSAL ? min(nkt, (qfirst + 31) / FK + 1) : nkt;
  const int plain = CAUSAL ? min(Lk / FK, (qfirst + 1) / FK) : Lk / FK;   // leading tiles that need no mask test
  const bf16_t* kbase = scalar_ptr(k + (size_t)lok * ldk + hk * DH);
  const bf16_t* vbase = scalar_ptr(v + (size_t)lok * ldk + hk * DH);
  const uint32_t klds = (uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char*)Kbuf;
  const uint32_t vlds = (uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char*)Vbuf;
  const uint32_t lrow = RT::load_row(lane), lchunk = RT::load_chunk(lane) * 16;
  // tile t of K or V into ring slot `slot` (t % 3); rows past the keys are clamped (their P is 0)
  auto fetch = [&](const bf16_t* base, uint32_t lds, int t, int slot) {
    if (t >= nkt) return;
    const bf16_t* src = base + (size_t)t * FK * ldk;
    const int last = Lk - t * FK - 1;
    const uint32_t dst = lds + slot * TILE;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      const int r = wave * RUNS + i;
      const uint32_t off = (uint32_t)min(r * RT::RPR + (int)lrow, last) * (uint32_t)ldk * 2u + lchunk;
      TileAsync<FK, DH, 512>::load16(src, off, dst + r * RT::RUN);
    }
  };
  f32x16 sacc[KBL];
  bf16x8 pb[KBL][2];
  static_assert(KBL == 2, "one factor between the blocks of a tile");
  bool late = false;                                      // the maximum moved in the tile's second block, by late_corr
  float late_corr = 1.f;
  const int rows_at = RT::rows_at(lane), cols_at = RT::cols_at(lane);
  auto scores = [&](int slot) {                           // S^T = K Q^T of the key tile in a ring slot
    int at = slot * TILE + rows_at;
    asm volatile("" : "+v"(at));                           // one register; the rest is immediates
    const unsigned char* base = Kbuf + at;
    constexpr int NSTEP = KBL * KS, AHEAD = 3;
    bf16x8 f[AHEAD + 1];
#pragma unroll
    for (int b = 0; b < KBL; ++b) sacc[b] = f32x16{};
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) f[n] = RT::read_rows(base, n % KBL, n / KBL);
#pragma unroll
    for (int n = 0; n < NSTEP; ++n) {
      if (n + AHEAD < NSTEP) f[(n + AHEAD) % (AHEAD + 1)] = RT::read_rows(base, (n + AHEAD) % KBL, (n + AHEAD) / KBL);
      sacc[n % KBL] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n % (AHEAD + 1)], qf[n / KBL], sacc[n % KBL], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto values = [&](int slot) {                           // O^T += V^T P^T
    int at = slot * TILE + cols_at;
    asm volatile("" : "+v"(at));
    const unsigned char* base = Vbuf + at;
    constexpr int NSTEP = KBL * 2 * NB, AHEAD = 3;         // step n: 16 keys n / NB, 32 columns n % NB
    bf16x8 f[AHEAD + 1];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) f[n] = RT::read_cols(base, n % NB, n / NB);
#pragma unroll
    for (int n = 0; n < NSTEP; ++n) {
      if (n == 2 * NB && late) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[j][r] *= late_corr;
      }
      if (n + AHEAD < NSTEP) f[(n + AHEAD) % (AHEAD + 1)] = RT::read_cols(base, (n + AHEAD) % NB, (n + AHEAD) / NB);
      oacc[n % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n % (AHEAD + 1)], pb[n / NB / 2][n / NB % 2], oacc[n % NB], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto softmax = [&](int t) {
    if (t >= plain) {
      asm volatile("");                                    // keeps the tests out of the tiles that need none
      // element (b, r): key t * 64 + b * 32 + (r / 4) * 8 + half * 4 + r % 4
      const int left = Lk - t * FK - half * 4, ahead = qpos - t * FK - half * 4;
#pragma unroll
      for (int b = 0; b < KBL; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int e = b * 32 + (r >> 2) * 8 + (r & 3);
          if (e >= left || (CAUSAL && e > ahead)) sacc[b][r] = -INFINITY;
        }
    }
    late = false;
#pragma unroll
    for (int b = 0; b < KBL; ++b) {
      float mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[b][r]);
      mx = max_with_other_half(mx) * scale_log2;
      // lazy rescaling, as in the kernel above; the output takes the factor of a later block between the
      // blocks' products (see values)
      if (__builtin_amdgcn_ballot_w64(mx > m + 8.0f) != 0) {
        const float m_new = fmaxf(m, mx);
        const float corr = __builtin_amdgcn_exp2f(m - m_new);   // m = -inf at the start: 0
        m = m_new;
        lsum *= corr;
        if (b == 0) {
#pragma unroll
          for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) oacc[j][r] *= corr;
        } else {
          late = true;
          late_corr = corr;
        }
      }
      float psum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sacc[b][r], scale_log2, -m));   // masked: exp2(-inf) = 0
        sacc[b][r] = p;
        psum += p;
      }
      lsum += psum;
      pb[b][0] = acc_to_operand(sacc[b], 0);
      pb[b][1] = acc_to_operand(sacc[b], 1);
    }
  };
  settle_compiler_loads();                                // Q fragments, offsets
  fetch(kbase, klds, 0, 0);
  fetch(vbase, vlds, 0, 0);
  fetch(kbase, klds, 1, 1);
  wait_async_tiles();
  phase_barrier();
  if (wave >= 4) phase_barrier();                         // the second group stays one phase behind
  if (mine > 0) scores(0);
  phase_barrier();
  for (int t = 0, s0 = 0, s1 = 1, s2 = 2; t < nkt; ++t) {   // ring slots of tiles t, t + 1, t + 2
    // both groups are past the tiles these overwrite (V t - 2, K t - 1); they are read two phases from now
    fetch(vbase, vlds, t + 1, s1);
    fetch(kbase, klds, t + 2, s2);
    if (t < mine) softmax(t);
    phase_barrier();
    if (t < mine) values(s0);
    if (t + 1 < mine) scores(s1);
    wait_async_tiles();
    phase_barrier();
    const int s = s0;
    s0 = s1; s1 = s2; s2 = s;
  }
  if (wave < 4) phase_barrier();
  lsum = sum_with_other_half(lsum);
  if (qpos < L) {
    // no key in this chunk: zero output, lse = -inf
    const float inv = Lk > 0 ? 1.0f / lsum : 0.f;
    bf16_t* op = o + (size_t)(lo + qpos) * ldo + hq * DH;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (bf16_t)(oacc[j][g * 4 + e] * inv);
        *reinterpret_cast<bf16x4*>(op + j * 32 + g * 8 + half * 4) = w;
      }
    if (half == 0) lse[(size_t)hq * Ttot + lo + qpos] = Lk > 0 ? (m + log2f(lsum)) * LN2 : -INFINITY;
  }
}

int count_tiles(const int32_t* cu_host, int S, int rows) {
  long n = 0;
  for (int s = 0; s < S; ++s) n += (cu_host[s + 1] - cu_host[s] + rows - 1) / rows;
  return (int)n;
}

// keys a query walks on average
double keys_per_query(const AttnArgs& a) {
  const int32_t* ck = a.kv_cu_host();
  double pairs = 0;
  for (int s = 0; s < a.S; ++s) pairs += (double)(a.cu_host[s + 1] - a.cu_host[s]) * (ck[s + 1] - ck[s]);
  return a.T > 0 ? (a.causal ? 0.5 : 1.0) * pairs / a.T : 0.0;
}

// 256-row tiles and alternating groups, or 128-row tiles and two workgroups per CU?  The former where they cut the
// sequences about as well and come to two per CU or more, and
//  - where a query walks enough keys to pay for the turns' start and end.  Forward, 128 -> 256 rows, us: head size 128,
//    bidirectional, 24 x 256, 32 heads, 55 -> 62; 16 x 512, 24 heads, 74 -> 78; 4 x 2048, 24 heads, 217 -> 197; causal 12 x 520,
//    24 heads, 60 -> 70; 8 documents of 411 to 1800, 32 heads, 128 -> 122.  Head size 64, bidirectional, 4 x 900, 32 heads, 48 -> 44.
//  - under a full mask, where the last round is nearly full, since all tiles of a sequence take equally long: head size 64,
//    8 x 768, 24 heads (2.25 rounds), 47 -> 52; 128, 6 x 1000, 16 heads (1.5 rounds), 65 -> 69.
//  - not at head size 64 under a causal mask, where the vector unit bounds both and long tiles cannot be evened out: 4 x 2048,
//    16 heads, 66 -> 72; 2 x 2600, 24 heads, 73 -> 87; ahead only with 64 heads (4096, 172 -> 157).
// 189 packs of 577 to 18432 tokens, both masks, 16 to 64 heads: no choice of 256 rows is more than 4 % behind 128.
bool queries_alternating(const AttnArgs& a) {
  if (a.causal && a.dh == 64) return false;
  const long ta = count_tiles(a.cu_host, a.S, AQ), tn = count_tiles(a.cu_host, a.S, FQ), wgs = ta * a.Hq;
  if (wgs < 2 * NUM_CU || ta * 8 > tn * 5) return false;
  if (a.causal) return keys_per_query(a) >= 600;
  return keys_per_query(a) >= 800 && (long)cdiv(wgs, NUM_CU) * NUM_CU * 4 <= wgs * 5;
}

template <int DH>
bm_status fwd_launch(const AttnArgs& a, void* o, float* lse, hipStream_t st) {
  const float sl2 = LOG2E / sqrtf((float)a.dh);
  if constexpr (DH != 72) {
    if (queries_alternating(a)) {
      const dim3 grid(count_tiles(a.cu_host, a.S, AQ) * a.Hq);
      const SeqOrder ord = make_seq_order(a.cu_host, a.kv_cu_host(), a.S, AQ, !a.causal);
      auto kern = fa_fwd_alt_kernel<DH, false>;
      if constexpr (DH == 128) if (a.causal) kern = fa_fwd_alt_kernel<DH, true>;
      hipLaunchKernelGGL(kern, grid, dim3(512), 0, st, (const bf16_t*)a.q, (const bf16_t*)a.k, (const bf16_t*)a.v,
                         a.ld_qkv, a.kv_ld(), a.cu_dev, a.kv_cu_dev(), a.S, (bf16_t*)o, a.Hq * a.dh, lse, a.T, a.Hq,
                         a.Hq / a.Hkv, sl2, ord);
      BM_CHECK_LAUNCH("fa_fwd_alt");
      return BM_OK;
    }
  }
  dim3 grid(count_tiles(a.cu_host, a.S, FQ) * a.Hq), block(256);
  if (grid.x == 0) return BM_OK;
  // a query tile runs as long as its sequence has keys
  const SeqOrder ord = make_seq_order(a.cu_host, a.kv_cu_host(), a.S, FQ, !a.causal);
#define BM_L(C)                                                                                  \
  hipLaunchKernelGGL((fa_fwd_kernel<DH, C, false>), grid, block, 0, st, (const bf16_t*)a.q,             \
                     (const bf16_t*)a.k, (const bf16_t*)a.v, a.ld_qkv, a.kv_ld(), a.cu_dev,      \
                     a.kv_cu_dev(), a.S, (bf16_t*)o, a.Hq * a.dh, lse, a.T, a.Hq, a.Hq / a.Hkv, sl2, ord, a.local)
  if (a.causal) BM_L(true); else BM_L(false);
#undef BM_L
  BM_CHECK_LAUNCH("fa_fwd");
  return BM_OK;
}

// =============================================================================
// backward
// =============================================================================
// delta[h, t] = sum_c dO[t,h,c] * O[t,h,c]; 8 (head size 64) or 16 lanes share one (row, head),
// 16 bytes each, so a wavefront reads whole contiguous row segments
template <int DH> struct DeltaLanes { static constexpr int N = DH <= 64 ? 8 : 16, SHIFT = DH <= 64 ? 3 : 4; };
template <int DH>
__global__ void fa_delta_kernel(const bf16_t* __restrict__ o, const bf16_t* __restrict__ d_o, int ldo,
                                float* __restrict__ delta, int Ttot, int Hq) {
  constexpr int LP = DeltaLanes<DH>::N;
  const long gid = ((long)blockIdx.x * blockDim.x + threadIdx.x) >> DeltaLanes<DH>::SHIFT;
  const int c = (threadIdx.x & (LP - 1)) * 8;
  float s = 0.f;
  const bool live = gid < (long)Ttot * Hq;
  const int t = live ? (int)(gid / Hq) : 0, hq = live ? (int)(gid % Hq) : 0;
  if (live && c < DH) {
    float a[8], b[8];
    load16(o + (size_t)t * ldo + hq * DH + c, a);
    load16(d_o + (size_t)t * ldo + hq * DH + c, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(a[e], b[e], s);
  }
#pragma unroll
  for (int off = LP / 2; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  if (live && c == 0) delta[(size_t)hq * Ttot + t] = s;
}

constexpr int WIDE_KEYS = 256;  // keys per workgroup of the wide dK/dV kernel
constexpr int BK_KEYS = 128;   // keys per workgroup in the dK/dV kernel (32 per wavefront)
constexpr int BK_Q = 64;       // query rows per step

// Sliding window: the first tokens of a sequence, which all of its queries see, are among its first `keys` keys (32 or 128).  Where that
// is more than `rows` query rows, these keys are split into parts of so many, which leave fp32 partials,
// [part][kv head x split][dK, dV][keys][DH].
struct FirstKeys {
  LocalMask mask = {0, 0, nullptr};
  int keys = 0, rows = 0, wgs = 0;    // query rows of a part; workgroups of the parts, in front of the key tiles'
  float* out = nullptr;
  SeqOrder ord = {};                  // the parts of the sequences, in pack order
  __host__ __device__ inline int parts(int Lq) const { return mask.sinks > 0 && Lq > rows ? (Lq + rows - 1) / rows : 0; }
};
// which sequence's part `id` is, and which of its parts; parts number from 0 in pack order
__device__ inline bool find_part(const FirstKeys& f, const int32_t* __restrict__ cuq, int S, int id, int* seq, int* part) {
  int n;
  if (f.ord.n) {
    if (!find_tile(cuq, f.ord, S, f.rows, id, seq, part, &n)) return false;
    *part = n - 1 - *part;                                 // (find_tile counts tiles from the last one)
    return true;
  }
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < S; s0 += 64) {
    const int s = min(s0 + lane, S - 1), mine = s0 + lane < S ? f.parts(cuq[s + 1] - cuq[s]) : 0, upto = scan_lanes(mine);
    const uint64_t past = __builtin_amdgcn_ballot_w64(id < upto);
    if (past != 0) {
      const int l = __builtin_ctzll(past);
      *seq = s0 + l;
      *part = id - __builtin_amdgcn_readlane(upto - mine, l);
      return true;
    }
    id -= __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}
// The queries that see a key, as a range of elements counted from row `base`: from .. from + n - 1; rows from `qend` on do not take part
struct SeenBy { int from; uint32_t n; };
__device__ inline SeenBy seen_by(const LocalMask& w, int key, int L, int off, int base, int qend) {
  const int from = key - off - base, to = min(qend - base, key >= w.sinks ? from + w.window : qend - base);
  return SeenBy{from, key < L ? (uint32_t)max(0, to - from) : 0u};
}
// Where a workgroup of dK/dV works with it: a tile of KEYS keys, or a part of the first one, and the query rows that it walks
struct KeyTile { int seq, kt, part, hk_gs, qlo, qhi, from; };      // from: the first key that is not the parts'
template <int KEYS>
__device__ inline bool find_key_tile(const FirstKeys& f, const SeqOrder& ord, const int32_t* __restrict__ cu,
                                     const int32_t* __restrict__ cuq, int S, int heads, int block, KeyTile* t) {
  int tile_id, n;
  if (block < f.wgs) {
    tile_and_head(heads, &tile_id, &t->hk_gs, block);
    if (!find_part(f, cuq, S, tile_id, &t->seq, &n)) return false;
    t->kt = 0;
    t->part = tile_id;
    t->from = 0;
    t->qlo = n * f.rows;
    t->qhi = min(cuq[t->seq + 1] - cuq[t->seq], t->qlo + f.rows);
    return true;
  }
  tile_and_head(heads, &tile_id, &t->hk_gs, block - f.wgs);
  if (!find_tile(cu, f.mask.key_end, ord, S, KEYS, tile_id, &t->seq, &t->kt, &n)) return false;
  t->kt = n - 1 - t->kt;
  t->part = -1;
  const int L = f.mask.key_end[t->seq] - cu[t->seq], Lq = cuq[t->seq + 1] - cuq[t->seq], off = L - Lq;
  const bool in_parts = t->kt == 0 && f.parts(Lq) > 0, seen_by_all = t->kt == 0 && f.mask.sinks > 0 && !in_parts;
  t->from = in_parts ? f.keys : 0;
  if (in_parts && (KEYS <= f.keys || L <= f.keys)) return false;
  t->qlo = max(0, t->kt * KEYS + t->from - off);
  t->qhi = seen_by_all ? Lq : min(Lq, min((t->kt + 1) * KEYS, L) - 1 - off + f.mask.window);
  return true;
}

// dK, dV of one 128-key tile of one kv head: walks the q heads of the group and the
// query tiles; scores are kept as S[q, key] so that P and dS are B operands as they are.
template <int DH> constexpr int dkdv_lds_bytes() { return 4 * BK_Q * HeadDim<DH>::DHL * 2 + 4 * BK_Q * 4; }
template <int DH, bool CAUSAL, bool WINDOW = false>
__device__ inline void dkdv_tile(unsigned char* lds, int block, const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v, int ld,
    int ldk, const bf16_t* __restrict__ d_o, int ldo, const float* __restrict__ lse,
    const float* __restrict__ delta, const int32_t* __restrict__ cuq, const int32_t* __restrict__ cu,
    int S, bf16_t* __restrict__ dk, bf16_t* __restrict__ dv, int ldd, int Tq, int Ttot, int Hkv, int group,
    float scale, float scale_log2, int gsplit,
    float* __restrict__ part /* [gsplit][2][Ttot][Hkv*DH] fp32 when gsplit > 1 */, SeqOrder ord, const FirstKeys& first = {}) {
  // cu, Ttot, ldk: the packing of the keys/values (and of dk, dv); cuq, Tq, ld: of the queries
  // Q and dO tiles are double-buffered and streamed into LDS (see TileAsync)
  constexpr int TILE = BK_Q * HeadDim<DH>::DHL;
  bf16_t* const Qbuf = reinterpret_cast<bf16_t*>(lds);
  bf16_t* const Dbuf = Qbuf + 2 * TILE;
  float* const Lbuf = reinterpret_cast<float*>(Dbuf + 2 * TILE);
  float* const Dlbuf = Lbuf + 2 * BK_Q;
  int seq, kt, nkt, tile_id, hk;
  // with gsplit > 1 a workgroup takes group/gsplit of the q heads that share this kv head
  // and leaves an fp32 partial; the (kv head, q-head part) pair plays the head's role
  int hk_gs;
  KeyTile where;                                       // sliding window
  if constexpr (WINDOW) {
    if (!find_key_tile<BK_KEYS>(first, ord, cu, cuq, S, Hkv * gsplit, block, &where)) return;
    hk_gs = where.hk_gs; seq = where.seq; kt = where.kt;
  } else {
    tile_and_head(Hkv * gsplit, &tile_id, &hk_gs, block);
  }
  hk = hk_gs / gsplit;
  const int gs = hk_gs % gsplit;
  const int gpart = group / gsplit;
  if constexpr (!WINDOW) {
    if (!find_tile(cu, ord, S, BK_KEYS, tile_id, &seq, &kt, &nkt)) return;
    kt = nkt - 1 - kt;                                   // early key tiles see the most queries
  }
  const int lo = cu[seq], L = (WINDOW ? first.mask.key_end[seq] : cu[seq + 1]) - lo;
  const int loq = cuq[seq], Lq = cuq[seq + 1] - loq;
  const int off = WINDOW ? L - Lq : 0;
  const int kb0 = kt * BK_KEYS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  const int kpos = kb0 + wave * 32 + (lane & 31);       // this lane's key (column of S)
  const int krow = min(kpos, L - 1);

  // With several resident wavefronts to hide the LDS read, dP starts at -delta of its query row, so that the
  // MFMAs leave dP - delta.  (With one wavefront per SIMD the read in front of the MFMAs costs more.)
  constexpr bool FOLD_DELTA = DH <= 64;
  bf16x8 kf[HeadDim<DH>::KS], vf[HeadDim<DH>::KS];
  {
    const bf16_t* kp = k + (size_t)(lo + krow) * ldk + hk * DH;
    const bf16_t* vp = v + (size_t)(lo + krow) * ldk + hk * DH;
#pragma unroll
    for (int ks = 0; ks < HeadDim<DH>::KS; ++ks) {
      kf[ks] = load_chunk<DH>(kp, ks * 2 + half);
      vf[ks] = load_chunk<DH>(vp, ks * 2 + half);
    }
  }
  f32x16 dkacc[HeadDim<DH>::NB], dvacc[HeadDim<DH>::NB];
#pragma unroll
  for (int j = 0; j < HeadDim<DH>::NB; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) { dkacc[j][r] = 0.f; dvacc[j][r] = 0.f; }

  const int qstart = CAUSAL ? ((WINDOW ? where.qlo : kb0) / BK_Q) * BK_Q : 0, qend = WINDOW ? where.qhi : Lq;
  const int nqt = qend > qstart ? (qend - qstart + BK_Q - 1) / BK_Q : 0;   // no query: dk = dv = 0
  const int iters = nqt * gpart;
  using Tile = TileAsync<BK_Q, DH, 256>;
  Tile tq, td;
  tq.init(ld, tid);
  td.init(ldo, tid);
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  float st_l = 0.f, st_d = 0.f;
  auto fetch = [&](int it, int par) {
    const int hq = hk * group + gs * gpart + it / nqt;
    const int q0 = qstart + (it % nqt) * BK_Q;
    tq.issue(q + ((size_t)loq + q0) * ld + hq * DH, ld, Lq - q0, Qbuf + par * TILE, wave_u);
    td.issue(d_o + ((size_t)loq + q0) * ldo + hq * DH, ldo, Lq - q0, Dbuf + par * TILE, wave_u);
    if (tid < BK_Q) {
      const int qi = min(q0 + tid, Lq - 1);
      st_l = lse[(size_t)hq * Tq + loq + qi];      // used (and waited for) when the next step opens
      st_d = delta[(size_t)hq * Tq + loq + qi];
    }
  };
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    Tile::zero_padding(Qbuf + b * TILE, tid);
    Tile::zero_padding(Dbuf + b * TILE, tid);
  }
  if (iters > 0) fetch(0, 0);
  settle_compiler_loads();                              // K and V fragments, lse, delta (and, with them, tile 0)
  // one step; MASKED is a compile-time copy with the per-element tests (see the forward kernel)
  auto step = [&](int it, auto masked, auto parity) {
    constexpr bool MASKED = decltype(masked)::value;
    constexpr int PAR = decltype(parity)::value;
    const bf16_t* Qs = Qbuf + PAR * TILE;
    const bf16_t* Ds = Dbuf + PAR * TILE;
    const float* Ls = Lbuf + PAR * BK_Q;
    const float* Dl = Dlbuf + PAR * BK_Q;
    if (tid < BK_Q) { Lbuf[PAR * BK_Q + tid] = st_l * LOG2E; Dlbuf[PAR * BK_Q + tid] = st_d; }
    wait_async_tiles();
    __syncthreads();      // tile `it` is there for everyone, and everyone is done with tile it-1
    if (it + 1 < iters) fetch(it + 1, 1 - PAR);
    const int q0 = qstart + (it % nqt) * BK_Q;
    SeenBy seen = {0, 0};
    if constexpr (WINDOW && MASKED) seen = seen_by(first.mask, kpos, L, off, q0 + half * 4, qend);
    // S = Q K^T and dP = dO V^T for both 32-query blocks first, then per block the
    // softmax arithmetic (under the other block's MFMAs) followed by its dV / dK MFMAs.
    f32x16 sacc[BK_Q / 32], dpacc[BK_Q / 32];
#pragma unroll
    for (int qb = 0; qb < BK_Q / 32; ++qb) {
      sacc[qb] = f32x16{};
      if (!FOLD_DELTA) dpacc[qb] = f32x16{};
      if (FOLD_DELTA) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 d4 = *reinterpret_cast<const f32x4*>(Dl + qb * 32 + g * 8 + half * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) dpacc[qb][g * 4 + e] = -d4[e];
        }
      }
    }
    {
      // the operand fragments of step n + AHEAD are requested from LDS before the MFMAs of step n
      // are issued (a ring of AHEAD + 1 register sets): with one wavefront per SIMD nothing else
      // would cover the LDS latency in front of every MFMA
      constexpr int KS = HeadDim<DH>::KS, NSTEP = (BK_Q / 32) * KS, AHEAD = 2;
      bf16x8 fq[AHEAD + 1], fd[AHEAD + 1];
#pragma unroll
      for (int n = 0; n < AHEAD && n < NSTEP; ++n) {
        fq[n] = frag_rows<HeadDim<DH>::DHL>(Qs, (n / KS) * 32, n % KS, lane);
        fd[n] = frag_rows<HeadDim<DH>::DHL>(Ds, (n / KS) * 32, n % KS, lane);
      }
#pragma unroll
      for (int n = 0; n < NSTEP; ++n) {
        const int qb = n / KS, ks = n % KS, m = n + AHEAD;
        if (m < NSTEP) {
          fq[m % (AHEAD + 1)] = frag_rows<HeadDim<DH>::DHL>(Qs, (m / KS) * 32, m % KS, lane);
          fd[m % (AHEAD + 1)] = frag_rows<HeadDim<DH>::DHL>(Ds, (m / KS) * 32, m % KS, lane);
        }
        sacc[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[n % (AHEAD + 1)], kf[ks], sacc[qb], 0, 0, 0);
        dpacc[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fd[n % (AHEAD + 1)], vf[ks], dpacc[qb], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int qb = 0; qb < BK_Q / 32; ++qb) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int qoff = qb * 32 + g * 8 + half * 4;
        const f32x4 l4 = *reinterpret_cast<const f32x4*>(Ls + qoff);
        f32x4 d4 = {0.f, 0.f, 0.f, 0.f};
        if (!FOLD_DELTA) d4 = *reinterpret_cast<const f32x4*>(Dl + qoff);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = g * 4 + e;
          float p = __builtin_amdgcn_exp2f(fmaf(sacc[qb][r], scale_log2, -l4[e]));
          if (WINDOW && MASKED) p = (uint32_t)(qb * 32 + g * 8 + e - seen.from) < seen.n ? p : 0.f;
          if (!WINDOW && MASKED) {
            const int qi = q0 + qoff + e;
            if (qi >= qend || kpos >= L || (CAUSAL && kpos > qi)) p = 0.f;
          }
          sacc[qb][r] = p;
          dpacc[qb][r] = FOLD_DELTA ? p * dpacc[qb][r] : p * (dpacc[qb][r] - d4[e]);
        }
      }
      const bf16x8 p0 = acc_to_operand(sacc[qb], 0), p1 = acc_to_operand(sacc[qb], 1);
      const bf16x8 s0 = acc_to_operand(dpacc[qb], 0), s1 = acc_to_operand(dpacc[qb], 1);
      {
        // dV += dO^T P, dK += Q^T dS: 4 MFMAs per 32 columns of dh, their transposed operands
        // requested one group ahead
        constexpr int NB = HeadDim<DH>::NB;
        bf16x8 fr[2][4];
        auto request = [&](int j, bf16x8 (&f)[4]) {
          f[0] = frag_cols<HeadDim<DH>::DHL>(Ds, j * 32, qb * 32, lane);
          f[1] = frag_cols<HeadDim<DH>::DHL>(Ds, j * 32, qb * 32 + 16, lane);
          f[2] = frag_cols<HeadDim<DH>::DHL>(Qs, j * 32, qb * 32, lane);
          f[3] = frag_cols<HeadDim<DH>::DHL>(Qs, j * 32, qb * 32 + 16, lane);
        };
        request(0, fr[0]);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          if (j + 1 < NB) request(j + 1, fr[(j + 1) & 1]);
          dvacc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[j & 1][0], p0, dvacc[j], 0, 0, 0);
          dvacc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[j & 1][1], p1, dvacc[j], 0, 0, 0);
          dkacc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[j & 1][2], s0, dkacc[j], 0, 0, 0);
          dkacc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[j & 1][3], s1, dkacc[j], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  };
  // Which query tiles need the tests: all of them when this key tile is cut by the sequence end;
  // else, per q head, the first ones under a causal mask (queries before this wavefront's last
  // key) and the last one when it is cut by the sequence end.  Every wavefront runs `iters`
  // steps; only the split between the copies differs.
  {
    // (one call site per copy of the step: with two the compiler stops inlining them)
    using P0 = std::integral_constant<int, 0>;
    using P1 = std::integral_constant<int, 1>;
    const bool all_masked = kb0 + BK_KEYS > L;
    const int n_front = CAUSAL ? min(nqt, (wave * 32 + 32 + BK_Q - 1) / BK_Q) : 0;
    const int n_whole = max(n_front, (Lq - qstart) % BK_Q ? nqt - 1 : nqt);
    // a tile whose queries see none of this wavefront's keys: most of those behind the window of the first keys
    auto idle = [&](int it) {
      const int par = it & 1;
      if (tid < BK_Q) { Lbuf[par * BK_Q + tid] = st_l * LOG2E; Dlbuf[par * BK_Q + tid] = st_d; }
      wait_async_tiles();
      __syncthreads();
      if (it + 1 < iters) fetch(it + 1, 1 - par);
    };
    for (int it = 0, t = 0; it < iters; ++it, t = (t + 1 == nqt ? 0 : t + 1)) {
      const int q0 = qstart + t * BK_Q;
      if (WINDOW && (kb0 + wave_u * 32 < where.from || none_visible(first.mask, kb0 + wave_u * 32, 32, off + q0, BK_Q))) { idle(it); continue; }
      const bool masked = WINDOW ? all_masked || q0 + BK_Q > qend || !all_visible(first.mask, kb0 + wave_u * 32, 32, off + q0, BK_Q)
                                 : all_masked || t < n_front || t >= n_whole;
      if (it & 1) { if (masked) step(it, std::true_type{}, P1{}); else step(it, std::false_type{}, P1{}); }
      else { if (masked) step(it, std::true_type{}, P0{}); else step(it, std::false_type{}, P0{}); }
    }
  }
  const bool leaves_part = WINDOW && where.part >= 0;
  if (WINDOW && kpos < where.from) return;
  if (kpos < L && (gsplit > 1 || leaves_part)) {
    const size_t plane = (size_t)Ttot * Hkv * DH;
    float* pk = part + ((size_t)gs * 2 + 0) * plane + (size_t)(lo + kpos) * (Hkv * DH) + hk * DH;
    float* pv = part + ((size_t)gs * 2 + 1) * plane + (size_t)(lo + kpos) * (Hkv * DH) + hk * DH;
    if (leaves_part) {
      pk = first.out + (((size_t)where.part * (Hkv * gsplit) + hk_gs) * 2 * BK_KEYS + kpos) * DH;
      pv = pk + BK_KEYS * DH;
    }
#pragma unroll
    for (int j = 0; j < HeadDim<DH>::NB; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        if (DH % 32 == 0 || j * 32 + g * 8 + half * 4 < DH) {
          *reinterpret_cast<f32x4*>(pk + j * 32 + g * 8 + half * 4) =
              f32x4{dkacc[j][g * 4] * scale, dkacc[j][g * 4 + 1] * scale, dkacc[j][g * 4 + 2] * scale, dkacc[j][g * 4 + 3] * scale};
          *reinterpret_cast<f32x4*>(pv + j * 32 + g * 8 + half * 4) =
              f32x4{dvacc[j][g * 4], dvacc[j][g * 4 + 1], dvacc[j][g * 4 + 2], dvacc[j][g * 4 + 3]};
        }
  } else if (kpos < L) {
    bf16_t* pk = dk + (size_t)(lo + kpos) * ldd + hk * DH;
    bf16_t* pv = dv + (size_t)(lo + kpos) * ldd + hk * DH;
#pragma unroll
    for (int j = 0; j < HeadDim<DH>::NB; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 wk, wv;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          wk[e] = (bf16_t)(dkacc[j][g * 4 + e] * scale);
          wv[e] = (bf16_t)dvacc[j][g * 4 + e];
        }
        if (DH % 32 == 0 || j * 32 + g * 8 + half * 4 < DH) {
          *reinterpret_cast<bf16x4*>(pk + j * 32 + g * 8 + half * 4) = wk;
          *reinterpret_cast<bf16x4*>(pv + j * 32 + g * 8 + half * 4) = wv;
        }
      }
  }
}

// dK, dV at head sizes above 64, where one wavefront cannot hold both accumulators next to a
// second resident wavefront: every 32-key block of the 128-key tile is shared by a PAIR of
// wavefronts that sit on the same SIMD (wavefronts w and w+4 of the 512-thread workgroup).
//   role 0 ("value" wavefront): S = Q K^T -> P = exp2(S*scale - lse), hands P to its partner
//                               through LDS, dV += dO^T P
//   role 1 ("key" wavefront):   dP = dO V^T, takes P, dS = P (dP - delta), dK += Q^T dS
// Each wavefront keeps one accumulator and one of K / V in registers (about 200 registers), so
// two are resident per SIMD and one's vector work runs under the other's MFMAs.  P travels as
// bf16 in the operand layout: role 0 feeds exactly these values to its own MFMAs, and role 1
// owns the same (key, query) elements in the same lanes, so the exchange is lane-private.
// (sliding windows: dS from P in fp16 times 2^15, 2^-12 off down to probabilities of 2^-29 and 0 below 2^-40, instead of from what bf16
// leaves; dK carries the factor to the end.  No probability is above 1: what rounds there -- at scores of 2^22 and more the roundings of a score and of its
// row's lse are whole powers of e -- is 1, since from 2 on fp16 would make it infinite.)
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));
constexpr float HANDED_SCALE = 32768.f;
__device__ inline f16x8 handed_p(const f32x16& p, int t) {
  f16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (_Float16)(p[t * 8 + e] * HANDED_SCALE);
  return __builtin_elementwise_min(r, (f16x8)(_Float16)HANDED_SCALE);
}
template <int DH> constexpr int dkdv_pair_lds_bytes() { return 4 * BK_Q * HeadDim<DH>::DHL * 2 + 4 * (BK_Q / 32) * 2 * 64 * 16 + 4 * BK_Q * 4; }
template <int DH, bool CAUSAL, bool WINDOW = false>
__device__ inline void dkdv_pair_tile(
    unsigned char* lds, int block, const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v, int ld,
    int ldk, const bf16_t* __restrict__ d_o, int ldo, const float* __restrict__ lse,
    const float* __restrict__ delta, const int32_t* __restrict__ cuq, const int32_t* __restrict__ cu,
    int S, bf16_t* __restrict__ dk, bf16_t* __restrict__ dv, int ldd, int Tq, int Ttot, int Hkv, int group,
    float scale, float scale_log2, int gsplit,
    float* __restrict__ part /* [gsplit][2][Ttot][Hkv*DH] fp32 when gsplit > 1 */, SeqOrder ord, const FirstKeys& first = {}) {
  constexpr int DHL = HeadDim<DH>::DHL, KS = HeadDim<DH>::KS, NB = HeadDim<DH>::NB, NQB = BK_Q / 32;
  // Q and dO tiles are double-buffered and streamed into LDS (see TileAsync): with one workgroup
  // per CU nothing else runs while a tile is parked between two barriers
  constexpr int TILE = BK_Q * DHL;
  // (in this order: with lse and delta behind 64 KiB, out of an immediate offset's reach, the bidirectional kernel of
  // head size 128 spills 22 registers)
  bf16_t* const Qbuf = reinterpret_cast<bf16_t*>(lds);
  bf16_t* const Ps = Qbuf + 2 * TILE;                    // [key block][q block][half k-step][lane] x 16 B
  float* const Lbuf = reinterpret_cast<float*>(Ps + 4 * NQB * 2 * 64 * 8);
  float* const Dlbuf = Lbuf + 2 * BK_Q;
  bf16_t* const Dbuf = reinterpret_cast<bf16_t*>(Dlbuf + 2 * BK_Q);
  int seq, kt, nkt, tile_id, hk, hk_gs;
  KeyTile where;                                       // sliding window
  if constexpr (WINDOW) {
    if (!find_key_tile<BK_KEYS>(first, ord, cu, cuq, S, Hkv * gsplit, block, &where)) return;
    hk_gs = where.hk_gs; seq = where.seq; kt = where.kt;
  } else {
    tile_and_head(Hkv * gsplit, &tile_id, &hk_gs, block);
  }
  hk = hk_gs / gsplit;
  const int gs = hk_gs % gsplit;
  const int gpart = group / gsplit;
  if constexpr (!WINDOW) {
    if (!find_tile(cu, ord, S, BK_KEYS, tile_id, &seq, &kt, &nkt)) return;
    kt = nkt - 1 - kt;                                   // early key tiles see the most queries
  }
  const int lo = cu[seq], L = (WINDOW ? first.mask.key_end[seq] : cu[seq + 1]) - lo;
  const int loq = cuq[seq], Lq = cuq[seq + 1] - loq;
  const int off = WINDOW ? L - Lq : 0;
  const int kb0 = kt * BK_KEYS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  const int kb = wave & 3, role = wave >> 2;            // wavefronts w and w+4 share a SIMD
  const int tid_r = tid & 255;                          // index inside the role's 256 threads
  const int kpos = kb0 + kb * 32 + (lane & 31);         // this lane's key (column of S)
  const int krow = min(kpos, L - 1);

  // role 0 keeps K (for S), role 1 keeps V (for dP)
  bf16x8 kvf[KS];
  {
    const bf16_t* p = (role == 0 ? k : v) + (size_t)(lo + krow) * ldk + hk * DH;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kvf[ks] = load_chunk<DH>(p, ks * 2 + half);
  }
  f32x16 acc[NB];                                       // role 0: dV^T, role 1: dK^T (unscaled)
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[j][r] = 0.f;

  const int qstart = CAUSAL ? ((WINDOW ? where.qlo : kb0) / BK_Q) * BK_Q : 0, qend = WINDOW ? where.qhi : Lq;
  const int nqt = qend > qstart ? (qend - qstart + BK_Q - 1) / BK_Q : 0;   // no query: dk = dv = 0
  const int iters = nqt * gpart;
  // role 0's wavefronts bring in the Q tile, role 1's the dO tile; lse and delta of the tile's
  // queries pass through registers of the first wavefront
  using Tile = TileAsync<BK_Q, DH, 256>;
  Tile tile;
  tile.init(role == 0 ? ld : ldo, tid_r);
  const int wave_r = __builtin_amdgcn_readfirstlane(wave & 3);
  const int role_u = __builtin_amdgcn_readfirstlane(role);
  float st_l = 0.f, st_d = 0.f;
  auto fetch = [&](int it, int par) {
    const int hq = hk * group + gs * gpart + it / nqt;
    const int q0 = qstart + (it % nqt) * BK_Q;
    if (role_u == 0) tile.issue(q + ((size_t)loq + q0) * ld + hq * DH, ld, Lq - q0, Qbuf + par * TILE, wave_r);
    else tile.issue(d_o + ((size_t)loq + q0) * ldo + hq * DH, ldo, Lq - q0, Dbuf + par * TILE, wave_r);
    if (tid < BK_Q) {
      const int qi = min(q0 + tid, Lq - 1);
      st_l = lse[(size_t)hq * Tq + loq + qi];     // used (and waited for) when the next step opens
      st_d = delta[(size_t)hq * Tq + loq + qi];
    }
  };
#pragma unroll
  for (int b = 0; b < 2; ++b) Tile::zero_padding((role == 0 ? Qbuf : Dbuf) + b * TILE, tid_r);
  if (iters > 0) fetch(0, 0);
  settle_compiler_loads();                              // K / V fragments, lse, delta (and, with them, tile 0)
  bf16_t* my_p = Ps + (size_t)kb * (NQB * 2 * 64 * 8) + lane * 8;

  auto step = [&](int it, auto masked, auto parity) {
    constexpr bool MASKED = decltype(masked)::value;
    constexpr int PAR = decltype(parity)::value;
    const bf16_t* Qs = Qbuf + PAR * TILE;
    const bf16_t* Ds = Dbuf + PAR * TILE;
    const float* Ls = Lbuf + PAR * BK_Q;
    const float* Dl = Dlbuf + PAR * BK_Q;
    const bf16_t* rows_src = role == 0 ? Qs : Ds;       // phase 1 operand: Q (S) or dO (dP)
    const bf16_t* cols_src = role == 0 ? Ds : Qs;       // phase 2 operand: dO^T (dV) or Q^T (dK)
    if (tid < BK_Q) { Lbuf[PAR * BK_Q + tid] = st_l * LOG2E; Dlbuf[PAR * BK_Q + tid] = st_d; }
    // tile `it` is there for everyone, and everyone is done with tile it-1 and its P
    wait_async_tiles();
    __syncthreads();
    if (it + 1 < iters) fetch(it + 1, 1 - PAR);
    const int q0 = qstart + (it % nqt) * BK_Q;
    // phase 1: X[q, key] = rows(Q or dO) . (K or V)^T for both 32-query blocks
    f32x16 xacc[NQB];
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) xacc[qb] = f32x16{};
    {
      constexpr int NSTEP = NQB * KS, AHEAD = 2;
      bf16x8 fx[AHEAD + 1];
#pragma unroll
      for (int n = 0; n < AHEAD && n < NSTEP; ++n) fx[n] = frag_rows<DHL>(rows_src, (n / KS) * 32, n % KS, lane);
#pragma unroll
      for (int n = 0; n < NSTEP; ++n) {
        const int m = n + AHEAD;
        if (m < NSTEP) fx[m % (AHEAD + 1)] = frag_rows<DHL>(rows_src, (m / KS) * 32, m % KS, lane);
        xacc[n / KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[n % (AHEAD + 1)], kvf[n % KS], xacc[n / KS], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    bf16x8 op[NQB][2];                                  // B operands of phase 2: P (role 0) or dS (role 1)
    if (role == 0) {
      SeenBy seen = {0, 0};
      if constexpr (WINDOW && MASKED) seen = seen_by(first.mask, kpos, L, off, q0 + half * 4, qend);
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int qoff = qb * 32 + g * 8 + half * 4;
          const f32x4 l4 = *reinterpret_cast<const f32x4*>(Ls + qoff);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = g * 4 + e;
            float p = __builtin_amdgcn_exp2f(fmaf(xacc[qb][r], scale_log2, -l4[e]));
            if (WINDOW && MASKED) p = (uint32_t)(qb * 32 + g * 8 + e - seen.from) < seen.n ? p : 0.f;
            if (!WINDOW && MASKED) {
              const int qi = q0 + qoff + e;
              if (qi >= qend || kpos >= L || (CAUSAL && kpos > qi)) p = 0.f;
            }
            xacc[qb][r] = p;
          }
        }
        op[qb][0] = acc_to_operand(xacc[qb], 0);
        op[qb][1] = acc_to_operand(xacc[qb], 1);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if constexpr (WINDOW) *reinterpret_cast<f16x8*>(my_p + (qb * 2 + t) * 64 * 8) = handed_p(xacc[qb], t);
          else *reinterpret_cast<bf16x8*>(my_p + (qb * 2 + t) * 64 * 8) = op[qb][t];
        }
      }
    }
    __syncthreads();                                    // P of this step is in LDS
    if (role == 1) {
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) {
        using Handed = std::conditional_t<WINDOW, f16x8, bf16x8>;
        const Handed pa = *reinterpret_cast<const Handed*>(my_p + (qb * 2 + 0) * 64 * 8);
        const Handed pb = *reinterpret_cast<const Handed*>(my_p + (qb * 2 + 1) * 64 * 8);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 d4 = *reinterpret_cast<const f32x4*>(Dl + qb * 32 + g * 8 + half * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = g * 4 + e;
            const float p = (float)(r < 8 ? pa[r] : pb[r - 8]);
            xacc[qb][r] = p * (xacc[qb][r] - d4[e]);
          }
        }
        op[qb][0] = acc_to_operand(xacc[qb], 0);
        op[qb][1] = acc_to_operand(xacc[qb], 1);
      }
    }
    // phase 2: acc^T[c, key] += cols(dO or Q)^T . (P or dS), transposed operands requested one pair ahead
    {
      constexpr int NSTEP = NQB * NB;
      bf16x8 fr[2][2];
      fr[0][0] = frag_cols<DHL>(cols_src, 0, 0, lane);
      fr[0][1] = frag_cols<DHL>(cols_src, 0, 16, lane);
#pragma unroll
      for (int n = 0; n < NSTEP; ++n) {
        const int qb = n / NB, j = n % NB, m = n + 1;
        if (m < NSTEP) {
          fr[m & 1][0] = frag_cols<DHL>(cols_src, (m % NB) * 32, (m / NB) * 32, lane);
          fr[m & 1][1] = frag_cols<DHL>(cols_src, (m % NB) * 32, (m / NB) * 32 + 16, lane);
        }
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[n & 1][0], op[qb][0], acc[j], 0, 0, 0);
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[n & 1][1], op[qb][1], acc[j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  // which query tiles need the mask tests: as in the single-wavefront kernel, per 32-key block
  using P0 = std::integral_constant<int, 0>;
  using P1 = std::integral_constant<int, 1>;
  auto step_of = [&](int it, bool masked) {
    if (it & 1) { if (masked) step(it, std::true_type{}, P1{}); else step(it, std::false_type{}, P1{}); }
    else { if (masked) step(it, std::true_type{}, P0{}); else step(it, std::false_type{}, P0{}); }
  };
  {
    // (one call site per copy of the step: with two the compiler stops inlining them)
    const bool all_masked = kb0 + BK_KEYS > L;
    const int n_front = CAUSAL ? min(nqt, (kb * 32 + 32 + BK_Q - 1) / BK_Q) : 0;
    const int n_whole = max(n_front, (Lq - qstart) % BK_Q ? nqt - 1 : nqt);
    // a tile whose queries see none of this pair's keys: most of those behind the window of the first keys
    auto idle = [&](int it) {
      const int par = it & 1;
      if (tid < BK_Q) { Lbuf[par * BK_Q + tid] = st_l * LOG2E; Dlbuf[par * BK_Q + tid] = st_d; }
      wait_async_tiles();
      __syncthreads();
      if (it + 1 < iters) fetch(it + 1, 1 - par);
      __syncthreads();
    };
    for (int it = 0, t = 0; it < iters; ++it, t = (t + 1 == nqt ? 0 : t + 1)) {
      if (WINDOW && (kb0 + wave_r * 32 < where.from || none_visible(first.mask, kb0 + wave_r * 32, 32, off + qstart + t * BK_Q, BK_Q))) { idle(it); continue; }
      step_of(it, WINDOW ? all_masked || qstart + (t + 1) * BK_Q > qend ||
                               !all_visible(first.mask, kb0 + wave_r * 32, 32, off + qstart + t * BK_Q, BK_Q)
                         : all_masked || t < n_front || t >= n_whole);
    }
  }
  // dV as it is, dK times the softmax scale
  const float out_scale = role == 0 ? 1.0f : WINDOW ? scale * (1.0f / HANDED_SCALE) : scale;
  const bool leaves_part = WINDOW && where.part >= 0;
  if (WINDOW && kpos < where.from) return;
  if (kpos < L && (gsplit > 1 || leaves_part)) {
    const size_t plane = (size_t)Ttot * Hkv * DH;
    float* pp = part + ((size_t)gs * 2 + (role == 0 ? 1 : 0)) * plane + (size_t)(lo + kpos) * (Hkv * DH) + hk * DH;
    if (leaves_part)
      pp = first.out + ((((size_t)where.part * (Hkv * gsplit) + hk_gs) * 2 + (role == 0 ? 1 : 0)) * BK_KEYS + kpos) * DH;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        if (DH % 32 == 0 || j * 32 + g * 8 + half * 4 < DH)
          *reinterpret_cast<f32x4*>(pp + j * 32 + g * 8 + half * 4) =
              f32x4{acc[j][g * 4] * out_scale, acc[j][g * 4 + 1] * out_scale, acc[j][g * 4 + 2] * out_scale,
                    acc[j][g * 4 + 3] * out_scale};
  } else if (kpos < L) {
    bf16_t* pp = (role == 0 ? dv : dk) + (size_t)(lo + kpos) * ldd + hk * DH;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (bf16_t)(acc[j][g * 4 + e] * out_scale);
        if (DH % 32 == 0 || j * 32 + g * 8 + half * 4 < DH)
          *reinterpret_cast<bf16x4*>(pp + j * 32 + g * 8 + half * 4) = w;
      }
  }
}

// dK, dV at head size 128 over many keys: the pair scheme with 64 keys per pair (256 per workgroup).
// Every Q / dO fragment read from LDS feeds two MFMAs instead of one, and a Q / dO tile is brought in
// for twice the keys: with 32 keys per pair the LDS pipe is busy as long as the matrix pipe (fragment
// reads, fills and the P exchange of a 32x32 block: about 1130 clocks of LDS for 1024 of MFMAs).
// 128 accumulator registers and 64 of K or V leave 64 for everything else, so
//  - a step is one 32-query block;
//  - tiles lie in LDS as RunTile has them, so that every read is one lane constant plus an immediate offset.
// Tiles go through a ring of four buffers, requested three steps ahead; one barrier per step hands over
// P and the next tile.
// Against 32 keys per pair, us: 8192 queries x 8192 keys, 32 / 8 heads, 2207 -> 1875 (1.17 PFLOP/s of MFMAs), causal
// 1138 -> 1002; 16 samples of about 1160 tokens, 24 heads, 848 -> 657; 8192 tokens of causal documents, 32
// heads, 435 -> 365.  Fragments requested three steps ahead and a raised wave priority around the MFMAs
// changed nothing.
struct WideTile {
  static constexpr int ROWS = 32, PART = RunTile<128>::bytes(ROWS);
  static constexpr int Q = 0, D = PART, LSE = 2 * PART, DELTA = LSE + ROWS * 4, BYTES = DELTA + ROWS * 4;
  static constexpr int RING = 4;
};

// the lane index, computed anew
__device__ inline int fresh_lane() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

constexpr int DKDV_WIDE_LDS_BYTES = WideTile::RING * WideTile::BYTES + 2 * 4 * 4096;
template <bool CAUSAL, bool WINDOW = false>
__device__ inline void dkdv_wide_tile(
    unsigned char* lds, int block, const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v, int ld,
    int ldk, const bf16_t* __restrict__ d_o, int ldo, const float* __restrict__ lse,
    const float* __restrict__ delta, const int32_t* __restrict__ cuq, const int32_t* __restrict__ cu,
    int S, bf16_t* __restrict__ dk, bf16_t* __restrict__ dv, int ldd, int Tq, int Ttot, int Hkv, int group,
    float scale, float scale_log2, int gsplit,
    float* __restrict__ part /* [gsplit][2][Ttot][Hkv*DH] fp32 when gsplit > 1 */, SeqOrder ord, const FirstKeys& first = {}) {
  constexpr int DH = 128, KS = 8, NB = 4, KB = 2;
  using W = WideTile;
  using RT = RunTile<DH>;
  static_assert(W::RING * W::BYTES % 1024 == 0, "P starts where a tile run may");
  unsigned char* const tiles = lds;
  unsigned char* const Pbuf = lds + W::RING * W::BYTES;  // [parity][pair][key block, half k-step][lane]
  int seq, kt, nkt, tile_id, hk, hk_gs;
  KeyTile where;                                       // sliding window
  if constexpr (WINDOW) {
    if (!find_key_tile<WIDE_KEYS>(first, ord, cu, cuq, S, Hkv * gsplit, block, &where)) return;
    hk_gs = where.hk_gs; seq = where.seq; kt = where.kt;
    where.qlo = __builtin_amdgcn_readfirstlane(where.qlo);
    where.qhi = __builtin_amdgcn_readfirstlane(where.qhi);
  } else {
    tile_and_head(Hkv * gsplit, &tile_id, &hk_gs, block);
  }
  hk = hk_gs / gsplit;
  const int gs = hk_gs % gsplit;
  const int gpart = group / gsplit;
  if constexpr (!WINDOW) {
    if (!find_tile(cu, ord, S, WIDE_KEYS, tile_id, &seq, &kt, &nkt)) return;
    kt = nkt - 1 - kt;                                   // early key tiles see the most queries
  }
  const int lo = cu[seq], L = (WINDOW ? first.mask.key_end[seq] : cu[seq + 1]) - lo;
  const int loq = cuq[seq], Lq = cuq[seq + 1] - loq;
  const int kb0 = kt * WIDE_KEYS;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pair = wave & 3;                            // wavefronts w and w+4 share a SIMD
  const int key0 = kb0 + pair * 64;                     // the pair's first key
  const int off = WINDOW ? L - Lq : 0, qstart = WINDOW ? where.qlo : CAUSAL ? kb0 : 0, qend = WINDOW ? where.qhi : Lq;
  const int nqt = qend > qstart ? (qend - qstart + W::ROWS - 1) / W::ROWS : 0;   // no query: dk = dv = 0
  const int iters = nqt * gpart;
  const int head0 = hk * group + gs * gpart;
  // A pair needs the mask tests where its keys are cut by the sequence end, on the last query tile when that is
  // cut, and up to its last key under a causal mask; it sits out the query tiles before its first key,
  // and all of them if it lies past the sequence.
  const bool keys_cut = key0 + 64 > L;
  // (WINDOW: and those behind the window of its last key, if its keys are no first tokens)
  const int skip = key0 >= L || (WINDOW && key0 + 64 <= where.from) ? nqt
                   : CAUSAL ? min(nqt, (WINDOW ? max(0, key0 - off - qstart) : key0 - qstart) / W::ROWS)
                            : 0;
  const int stop = WINDOW && key0 >= first.mask.sinks
                       ? max(skip, min(nqt, (key0 + 63 - off + first.mask.window - qstart + W::ROWS - 1) / W::ROWS))
                       : nqt;
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char*)tiles;
  constexpr int LOADS = 3;

  // Everything of a role is compiled on its own: its registers are allocated for it alone.  Addresses are derived
  // from the lane index in every step; kept in registers, they would push K or V fragments out to memory.
  auto run = [&](auto role_t) {
    constexpr int ROLE = decltype(role_t)::value;
    constexpr int ROWS_AT = ROLE == 0 ? W::Q : W::D, COLS_AT = ROLE == 0 ? W::D : W::Q;
    constexpr int STATS_AT = ROLE == 0 ? W::LSE : W::DELTA;
    bf16x8 kvf[KB][KS];                                   // role 0 keeps K (for S), role 1 keeps V (for dP)
    {
      const int l = fresh_lane();
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        const bf16_t* p = (ROLE == 0 ? k : v) + (size_t)(lo + min(key0 + b * 32 + (l & 31), L - 1)) * ldk + hk * DH;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kvf[b][ks] = load_chunk<DH>(p, ks * 2 + (l >> 5));
      }
    }
    f32x16 acc[NB][KB];                                   // role 0: dV^T, role 1: dK^T (unscaled)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[j][b][r] = 0.f;

    // role 0's wavefronts bring in Q and lse, role 1's dO and delta: two runs and a quarter of the row
    // statistics each, three loads per wavefront and step
    const int sld = ROLE == 0 ? ld : ldo;
    const bf16_t* src = scalar_ptr((ROLE == 0 ? q : d_o) + ((size_t)loq + qstart) * sld + head0 * DH);
    const float* stat = reinterpret_cast<const float*>(scalar_ptr((ROLE == 0 ? lse : delta) + (size_t)head0 * Tq + loq + qstart));
    int fn = 0, ft = 0;                                   // next tile to request: step, query tile of its head
    auto fetch = [&] {
      if (fn >= iters) return;
      const int last = Lq - qstart - 1 - ft * W::ROWS;    // rows past the sequence are clamped: their P is 0
      const uint32_t dst = lds0 + (fn & (W::RING - 1)) * W::BYTES;
      const int l = fresh_lane();
      const int row = RT::load_row(l), chunk = RT::load_chunk(l) * 16;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = pair * 2 + i;
        const uint32_t off = (uint32_t)min(r * RT::RPR + row, last) * (uint32_t)sld * 2u + (uint32_t)chunk;
        TileAsync<32, DH, 256>::load16(src, off, dst + ROWS_AT + r * RT::RUN);
      }
      const uint32_t off = (uint32_t)min(pair * 8 + (l & 7), last) * 4u;
      if (l < 8)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
                     :: "s"(dst + STATS_AT + pair * 32), "v"(off), "s"(stat) : "memory", "m0");
      ++fn;
      src += (size_t)W::ROWS * sld;
      stat += W::ROWS;
      if (++ft == nqt) {                                  // first query tile of the next head
        ft = 0;
        src += DH - (size_t)nqt * W::ROWS * sld;
        stat += Tq - (size_t)nqt * W::ROWS;
      }
    };
    auto tile_of = [&](int n) { return tiles + (n & (W::RING - 1)) * W::BYTES; };
    auto p_of = [&](int n) { return Pbuf + (n & 1) * (4 * 4096) + pair * 4096 + fresh_lane() * 16; };
    auto barrier = [] {
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
    };
    // between the phases of step n: its P is in LDS, and the next step's tile; the one after may still be on its way
    auto hand_over = [&](int n) {
      if (n + 2 < iters) asm volatile("s_waitcnt vmcnt(%0)" :: "n"((W::RING - 3) * LOADS) : "memory");
      else wait_async_tiles();
      barrier();
    };
    // phase 1: X[q, key] += rows(Q or dO) . (K or V)^T
    auto scores = [&](int n, f32x16 (&x)[KB]) {
      const unsigned char* rows = tile_of(n) + ROWS_AT + RT::rows_at(fresh_lane());
      constexpr int AHEAD = 2;
      bf16x8 fx[AHEAD + 1];
      auto request = [&](int ks) { fx[ks % (AHEAD + 1)] = RT::read_rows(rows, 0, ks); };
#pragma unroll
      for (int ks = 0; ks < AHEAD; ++ks) request(ks);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (ks + AHEAD < KS) request(ks + AHEAD);
#pragma unroll
        for (int b = 0; b < KB; ++b)
          x[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[ks % (AHEAD + 1)], kvf[b][ks], x[b], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // phase 2: acc^T[c, key] += cols(dO or Q)^T . (P or dS), transposed operands requested ahead
    auto accumulate = [&](int n, const bf16x8 (&op)[KB][2]) {
      const unsigned char* cols = tile_of(n) + COLS_AT + RT::cols_at(fresh_lane());
      auto request = [&](int m) { return RT::read_cols(cols, m >> 1, m & 1); };   // m = j * 2 + t: 32 columns of dh, 16 query rows
      constexpr int AHEAD = 2;
      bf16x8 fc[AHEAD + 1];
#pragma unroll
      for (int m = 0; m < AHEAD; ++m) fc[m] = request(m);
      if (ROLE == 0) fetch();                              // step n + 3, over the tile of step n - 1
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < NB * 2; ++m) {
        if (m + AHEAD < NB * 2) fc[(m + AHEAD) % (AHEAD + 1)] = request(m + AHEAD);
#pragma unroll
        for (int b = 0; b < KB; ++b)
          acc[m >> 1][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fc[m % (AHEAD + 1)], op[b][m & 1], acc[m >> 1][b], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto step = [&](int n, int q0) {
      // accumulator element (g, b, e) of a lane: query q0 + 4 half + (8 g + e), key key0 + lane % 32 + 32 b
      f32x16 x[KB];
      bf16x8 op[KB][2];
      if constexpr (ROLE == 0) {
        x[0] = x[1] = f32x16{};
        scores(n, x);
        if (WINDOW ? keys_cut || q0 + W::ROWS > qend || !all_visible(first.mask, key0, 64, off + q0, W::ROWS)
                   : keys_cut || q0 + W::ROWS > Lq || (CAUSAL && q0 < key0 + 63)) {
          asm volatile("");                                 // keeps the tests out of the steps that need none
          const int l = fresh_lane(), h4 = (l >> 5) * 4, ki = key0 + (l & 31);
          if constexpr (WINDOW) {
#pragma unroll
            for (int b = 0; b < KB; ++b) {
              const SeenBy seen = seen_by(first.mask, ki + b * 32, L, off, q0 + h4, qend);
#pragma unroll
              for (int r = 0; r < 16; ++r)
                x[b][r] = (uint32_t)((r >> 2) * 8 + (r & 3) - seen.from) < seen.n ? x[b][r] : -INFINITY;      // P = 0
            }
          } else {
            const int q_left = Lq - q0 - h4, k_left = L - ki, ahead = ki - q0 - h4;
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
              for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (q_left <= g * 8 + e || k_left <= b * 32 || (CAUSAL && ahead > g * 8 + e - b * 32))
                    x[b][g * 4 + e] = -INFINITY;            // P = 0
          }
        }
        const unsigned char* stats = tile_of(n) + STATS_AT + (fresh_lane() >> 5) * 16;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 l4 = *reinterpret_cast<const f32x4*>(stats + g * 32) * LOG2E;
#pragma unroll
          for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              x[b][g * 4 + e] = __builtin_amdgcn_exp2f(fmaf(x[b][g * 4 + e], scale_log2, -l4[e]));
        }
        unsigned char* my_p = p_of(n);
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            op[b][t] = acc_to_operand(x[b], t);
            if constexpr (WINDOW) *reinterpret_cast<f16x8*>(my_p + (b * 2 + t) * 1024) = handed_p(x[b], t);
            else *reinterpret_cast<bf16x8*>(my_p + (b * 2 + t) * 1024) = op[b][t];
          }
        hand_over(n);
      } else {
        x[0] = x[1] = f32x16{};
        scores(n, x);
        // dP - delta while the partner takes its exponentials (dP that starts at -delta saves the subtractions and
        // 2 % of the kernel, and rounds some sums differently)
        const unsigned char* stats = tile_of(n) + STATS_AT + (fresh_lane() >> 5) * 16;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 d4 = *reinterpret_cast<const f32x4*>(stats + g * 32);
#pragma unroll
          for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[b][g * 4 + e] -= d4[e];
        }
        asm volatile("" : "+v"(x[0]), "+v"(x[1]));          // (subtracted here: behind the barrier, delta would push V fragments out)
        hand_over(n);
        const unsigned char* my_p = p_of(n);
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int t = 0; t < 2; ++t) op[b][t] = *reinterpret_cast<const bf16x8*>(my_p + (b * 2 + t) * 1024);
        fetch();                                           // step n + 3, over the tile of step n - 1
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[b][t * 8 + e] *= WINDOW ? (float)__builtin_bit_cast(f16x8, op[b][t])[e] : (float)op[b][t][e];
            op[b][t] = acc_to_operand(x[b], t);
          }
      }
      accumulate(n, op);
    };

    settle_compiler_loads();                              // K / V fragments, offsets
    for (int n = 0; n < W::RING - 1; ++n) fetch();
    if (iters > W::RING - 2) asm volatile("s_waitcnt vmcnt(%0)" :: "n"((W::RING - 2) * LOADS) : "memory");
    else wait_async_tiles();
    barrier();
    for (int n = 0; n < iters;) {
      for (int t = 0; t < skip; ++t, ++n) { hand_over(n); fetch(); }
      for (int t = skip; t < stop; ++t, ++n) step(n, qstart + t * W::ROWS);
      if constexpr (WINDOW)
        for (int t = stop; t < nqt; ++t, ++n) { hand_over(n); fetch(); }
    }

    // dV as it is, dK times the softmax scale
    const float out_scale = ROLE == 0 ? 1.0f : WINDOW ? scale * (1.0f / HANDED_SCALE) : scale;
    const int l = fresh_lane();
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      const int key = key0 + b * 32 + (l & 31);
      if (key >= L || (WINDOW && key < where.from)) continue;
      const size_t row = (size_t)(lo + key);
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int c = hk * DH + j * 32 + g * 8 + (l >> 5) * 4;
          f32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = acc[j][b][g * 4 + e] * out_scale;
          if (gsplit > 1) {
            *reinterpret_cast<f32x4*>(part + ((size_t)gs * 2 + (ROLE == 0 ? 1 : 0)) * Ttot * Hkv * DH + row * (Hkv * DH) + c) = w;
          } else {
            bf16x4 h;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = (bf16_t)w[e];
            *reinterpret_cast<bf16x4*>((ROLE == 0 ? dv : dk) + row * ldd + c) = h;
          }
        }
    }
  };
  if (wave < 4) run(std::integral_constant<int, 0>{});
  else run(std::integral_constant<int, 1>{});
}

// dQ of one 128-row query tile of one q head: walks the key tiles, scores kept as
// S^T[key, q] as in the forward kernel.
template <int DH> constexpr int dq_lds_bytes() { return 4 * (DH > 72 ? 32 : FK) * HeadDim<DH>::DHL * 2; }
template <int DH, bool CAUSAL, bool WINDOW = false>
__device__ inline void dq_tile(unsigned char* lds, int tid, int tile_id, int hq, bool live, const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v, int ld,
    int ldk, const bf16_t* __restrict__ d_o, int ldo, const float* __restrict__ lse,
    const float* __restrict__ delta, const int32_t* __restrict__ cu, const int32_t* __restrict__ cuk,
    int S, bf16_t* __restrict__ dq, int ldd, int Ttot, int group, float scale, float scale_log2,
    SeqOrder ord, LocalMask w = {0, 0, nullptr}) {
  // K and V tiles are double-buffered and streamed into LDS as in the forward kernel; Q and dO of
  // this wavefront's 32 queries stay in registers.  At head size 128 a step is one 32-key block:
  // with two blocks' fragments and masks in flight next to Q, dO and the dQ accumulator the
  // kernel spills at two wavefronts per SIMD.  (dO read from LDS instead, a quarter more fragment
  // reads per key block, measured 1 % slower.)
  constexpr int FKD = DH > 72 ? 32 : FK;
  constexpr int TILE = FKD * HeadDim<DH>::DHL;
  bf16_t* const Kbuf = reinterpret_cast<bf16_t*>(lds);
  bf16_t* const Vbuf = Kbuf + 2 * TILE;
  int seq, qt, nqt;
  if (WINDOW ? !find_tile(cu, cu + 1, ord, S, FQ, tile_id, &seq, &qt, &nqt) : !find_tile(cu, ord, S, FQ, tile_id, &seq, &qt, &nqt)) return;
  const int hk = hq / group;
  const int lo = cu[seq], L = cu[seq + 1] - lo;
  const int lok = cuk[seq], Lk = (WINDOW ? w.key_end[seq] : cuk[seq + 1]) - lok;
  const int q0 = qt * FQ;
  const int lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  const int qpos = q0 + wave * 32 + (lane & 31);
  const int qrow = min(qpos, L - 1);
  if (Lk == 0) {
    // no key in this chunk (workgroup-uniform): dq = 0
    if (live && qpos < L) {
      bf16_t* pq = dq + (size_t)(lo + qpos) * ldd + hq * DH;
      for (int c = half * (DH / 2); c < (half + 1) * (DH / 2); c += 4) {
        bf16x4 z = {(bf16_t)0.f, (bf16_t)0.f, (bf16_t)0.f, (bf16_t)0.f};
        *reinterpret_cast<bf16x4*>(pq + c) = z;
      }
    }
    return;
  }

  bf16x8 qf[HeadDim<DH>::KS], dof[HeadDim<DH>::KS];
  {
    const bf16_t* qp = q + (size_t)(lo + qrow) * ld + hq * DH;
    const bf16_t* dp = d_o + (size_t)(lo + qrow) * ldo + hq * DH;
#pragma unroll
    for (int ks = 0; ks < HeadDim<DH>::KS; ++ks) {
      qf[ks] = load_chunk<DH>(qp, ks * 2 + half);
      dof[ks] = load_chunk<DH>(dp, ks * 2 + half);
    }
  }
  const float my_lse = lse[(size_t)hq * Ttot + lo + qrow] * LOG2E;
  const float my_delta = delta[(size_t)hq * Ttot + lo + qrow];
  f32x16 dqacc[HeadDim<DH>::NB];
#pragma unroll
  for (int j = 0; j < HeadDim<DH>::NB; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) dqacc[j][r] = 0.f;

  const int off = WINDOW ? Lk - L : 0;
  const auto walk = [&] {
    if constexpr (WINDOW) return KeyWalk<FKD>(w, off, q0, FQ, Lk);
    else return AllKeys<FKD>(CAUSAL, q0, FQ, Lk);
  }();
  const int nkt = walk.n;
  const bf16_t* kbase = k + (size_t)lok * ldk + hk * DH;
  const bf16_t* vbase = v + (size_t)lok * ldk + hk * DH;
  using Tile = TileAsync<FKD, DH, 256>;
  Tile tile;
  tile.init(ldk, tid);
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    Tile::zero_padding(Kbuf + b * TILE, tid);
    Tile::zero_padding(Vbuf + b * TILE, tid);
  }
  const size_t first = WINDOW ? (size_t)walk.tile(0) * FKD * ldk : 0;
  tile.issue(kbase + first, ldk, Lk - walk.tile(0) * FKD, Kbuf, wave_u);
  tile.issue(vbase + first, ldk, Lk - walk.tile(0) * FKD, Vbuf, wave_u);
  settle_compiler_loads();                 // the Q and dO fragments, lse, delta (and, with them, tile 0)
  // two copies of the step, without and with the mask test, as in the forward kernel
  constexpr bool FOLD_DELTA = DH <= 64;      // dP accumulators start at -delta: the MFMAs leave dP - delta
  f32x16 dp_start = {};
  if (FOLD_DELTA)
#pragma unroll
    for (int r = 0; r < 16; ++r) dp_start[r] = -my_delta;
  auto step = [&](int kt, auto masked, auto parity) {
    constexpr bool MASKED = decltype(masked)::value;
    constexpr int PAR = decltype(parity)::value;
    const bf16_t* Ks = Kbuf + PAR * TILE;
    const bf16_t* Vs = Vbuf + PAR * TILE;
    wait_async_tiles();
    __syncthreads();      // tile kt is there for everyone, and everyone is done with tile kt-1
    if (kt + 1 < nkt) {
      const int nt = walk.tile(kt + 1);
      const size_t next = (size_t)nt * FKD * ldk;
      tile.issue(kbase + next, ldk, Lk - nt * FKD, Kbuf + (1 - PAR) * TILE, wave_u);
      tile.issue(vbase + next, ldk, Lk - nt * FKD, Vbuf + (1 - PAR) * TILE, wave_u);
    }
    const int key0 = walk.tile(kt) * FKD;
    // S^T = K Q^T and dP^T = V dO^T of BP 32-key blocks are issued before any softmax arithmetic,
    // so that one block's MFMAs run under the other's vector work; at head size 128 that is one
    // block at a time (two sets of accumulators do not fit next to two resident wavefronts).
    constexpr int NBLK = FKD / 32, BP = DH > 72 ? 1 : NBLK, KS = HeadDim<DH>::KS;
#pragma unroll
    for (int b0 = 0; b0 < NBLK; b0 += BP) {
      f32x16 sacc[BP], dpacc[BP];
#pragma unroll
      for (int bi = 0; bi < BP; ++bi) { sacc[bi] = f32x16{}; dpacc[bi] = dp_start; }
      {
        // operand fragments are requested AHEAD MFMA pairs before their use (see the dK/dV kernel)
        constexpr int NSTEP = BP * KS, AHEAD = 2;
        bf16x8 fk[AHEAD + 1], fv[AHEAD + 1];
        auto request = [&](int n) {
          fk[n % (AHEAD + 1)] = frag_rows<HeadDim<DH>::DHL>(Ks, (b0 + n / KS) * 32, n % KS, lane);
          fv[n % (AHEAD + 1)] = frag_rows<HeadDim<DH>::DHL>(Vs, (b0 + n / KS) * 32, n % KS, lane);
        };
#pragma unroll
        for (int n = 0; n < AHEAD && n < NSTEP; ++n) request(n);
#pragma unroll
        for (int n = 0; n < NSTEP; ++n) {
          const int bi = n / KS, ks = n % KS;
          if (n + AHEAD < NSTEP) request(n + AHEAD);
          sacc[bi] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[n % (AHEAD + 1)], qf[ks], sacc[bi], 0, 0, 0);
          dpacc[bi] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv[n % (AHEAD + 1)], dof[ks],
                                                              dpacc[bi], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if constexpr (WINDOW && MASKED) {
        const int first_key = key0 + b0 * 32;
        hide_scores<BP>(w, first_key, off + q0 + wave_u * 32, off + qpos - first_key - half * 4, half * 4, sacc);
      }
#pragma unroll
      for (int bi = 0; bi < BP; ++bi) {
        const int b = b0 + bi;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float p = __builtin_amdgcn_exp2f(fmaf(sacc[bi][r], scale_log2, -my_lse));
          if (MASKED && !WINDOW) {
            const int key = key0 + b * 32 + (r >> 2) * 8 + half * 4 + (r & 3);
            if (key >= Lk || (CAUSAL && key > qpos)) p = 0.f;
          }
          dpacc[bi][r] = FOLD_DELTA ? p * dpacc[bi][r] : p * (dpacc[bi][r] - my_delta);
        }
        const bf16x8 s0 = acc_to_operand(dpacc[bi], 0), s1 = acc_to_operand(dpacc[bi], 1);
        {
          // dQ += dS K, the transposed K operands requested one pair of MFMAs ahead
          constexpr int NB = HeadDim<DH>::NB;
          bf16x8 fr[2][2];
          fr[0][0] = frag_cols<HeadDim<DH>::DHL>(Ks, 0, b * 32, lane);
          fr[0][1] = frag_cols<HeadDim<DH>::DHL>(Ks, 0, b * 32 + 16, lane);
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            if (j + 1 < NB) {
              fr[(j + 1) & 1][0] = frag_cols<HeadDim<DH>::DHL>(Ks, (j + 1) * 32, b * 32, lane);
              fr[(j + 1) & 1][1] = frag_cols<HeadDim<DH>::DHL>(Ks, (j + 1) * 32, b * 32 + 16, lane);
            }
            dqacc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[j & 1][0], s0, dqacc[j], 0, 0, 0);
            dqacc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[j & 1][1], s1, dqacc[j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
    }
  };
  int n_plain = Lk / FKD;
  if (CAUSAL) n_plain = min(n_plain, (q0 + wave * 32 + 1) / FKD);
  n_plain = min(n_plain, nkt);
  using P0 = std::integral_constant<int, 0>;
  using P1 = std::integral_constant<int, 1>;
  // a tile that none of this wavefront's queries see (left inside the step, this cost 44 registers at head size 128)
  auto idle = [&](int kt) {
    wait_async_tiles();
    __syncthreads();
    if (kt + 1 < nkt) {
      const int nt = walk.tile(kt + 1);
      const size_t next = (size_t)nt * FKD * ldk;
      tile.issue(kbase + next, ldk, Lk - nt * FKD, Kbuf + (1 - (kt & 1)) * TILE, wave_u);
      tile.issue(vbase + next, ldk, Lk - nt * FKD, Vbuf + (1 - (kt & 1)) * TILE, wave_u);
    }
  };
  for (int kt = 0; kt < nkt; ++kt) {
    if (WINDOW && none_visible(w, walk.tile(kt) * FKD, FKD, off + q0 + wave_u * 32, 32)) { idle(kt); continue; }
    const bool plain = WINDOW ? all_visible(w, walk.tile(kt) * FKD, FKD, off + q0 + wave_u * 32, 32) : kt < n_plain;
    if (kt & 1) { if (plain) step(kt, std::false_type{}, P1{}); else step(kt, std::true_type{}, P1{}); }
    else { if (plain) step(kt, std::false_type{}, P0{}); else step(kt, std::true_type{}, P0{}); }
  }
  if (live && qpos < L) {
    bf16_t* pq = dq + (size_t)(lo + qpos) * ldd + hq * DH;
#pragma unroll
    for (int j = 0; j < HeadDim<DH>::NB; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (bf16_t)(dqacc[j][g * 4 + e] * scale);
        if (DH % 32 == 0 || j * 32 + g * 8 + half * 4 < DH)
          *reinterpret_cast<bf16x4*>(pq + j * 32 + g * 8 + half * 4) = w;
      }
  }
}

// head sizes above 64, two workgroups per CU: packs whose dK/dV tiles alone fill the chip (see bwd_plan)
template <int DH, bool CAUSAL>
__global__ __launch_bounds__(256, 2) void fa_bwd_dq_kernel(
    const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v, int ld,
    int ldk, const bf16_t* __restrict__ d_o, int ldo, const float* __restrict__ lse,
    const float* __restrict__ delta, const int32_t* __restrict__ cu, const int32_t* __restrict__ cuk,
    int S, bf16_t* __restrict__ dq, int ldd, int Ttot, int Hq, int group, float scale, float scale_log2,
    SeqOrder ord) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[dq_lds_bytes<DH>()];
  int tile, head;
  tile_and_head(Hq, &tile, &head, blockIdx.x);
  dq_tile<DH, CAUSAL>(lds, threadIdx.x, tile, head, true, q, k, v, ld, ldk, d_o, ldo, lse, delta, cu, cuk, S, dq, ldd, Ttot,
                      group, scale, scale_log2, ord);
}

// The whole backward of head size 64 behind delta in one grid: the dK/dV tiles, which run longer, then the dQ tiles, which
// fill the CUs that the last of them leave.  Both have two wavefronts per SIMD.  They share one piece of LDS (with one
// each the dK/dV tile spills).  16 heads, two launches -> one: 577 tokens 41 -> 26 us, 6 images 47 -> 34, 26 images 236 -> 223, 8192
// tokens 985 -> 970; causal 41 -> 26, 45 -> 31, 179 -> 165, 547 -> 507.
template <int DH, bool CAUSAL>
__global__ __launch_bounds__(256, 2) void fa_bwd_joint_kernel(
    const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v, int ld, int ldk,
    const bf16_t* __restrict__ d_o, int ldo, const float* __restrict__ lse, const float* __restrict__ delta,
    const int32_t* __restrict__ cuq, const int32_t* __restrict__ cuk, int S, bf16_t* __restrict__ dq, int ldd,
    bf16_t* __restrict__ dk, bf16_t* __restrict__ dv, int ldd_kv, int Tq, int Tk, int Hkv, int group, float scale,
    float scale_log2, int gsplit, float* __restrict__ part, int kv_wgs, SeqOrder ord_kv, SeqOrder ord_q) {
  constexpr int LDS = dkdv_lds_bytes<DH>() > dq_lds_bytes<DH>() ? dkdv_lds_bytes<DH>() : dq_lds_bytes<DH>();
  __shared__ __attribute__((aligned(1024))) unsigned char lds[LDS];
  if ((int)blockIdx.x < kv_wgs)
    dkdv_tile<DH, CAUSAL>(lds, blockIdx.x, q, k, v, ld, ldk, d_o, ldo, lse, delta, cuq, cuk, S, dk, dv, ldd_kv, Tq, Tk, Hkv,
                          group, scale, scale_log2, gsplit, part, ord_kv);
  else
  {
    int tile, head;
    tile_and_head(Hkv * group, &tile, &head, blockIdx.x - kv_wgs);
    dq_tile<DH, CAUSAL>(lds, threadIdx.x, tile, head, true, q, k, v, ld, ldk, d_o, ldo, lse, delta, cuq, cuk, S, dq, ldd, Tq,
                        group, scale, scale_log2, ord_q);
  }
}

// dQ with two groups of wavefronts that take turns (see the forward kernel): while one multiplies -- dS K of a key
// tile, then Q K and dO V of the next -- the other one turns its scores into dS.  At head size 64, where the
// MFMAs of a tile are no longer than its softmax, the kernel above is ahead (96 against 112 us on 16384 tokens of images).
// us, two workgroups of four wavefronts -> this: 8192 x 8192 keys, 32 / 8 heads, 1522 -> 1332, causal 782 -> 687; 32768 tokens
// of causal documents 4217 -> 3630; 8192 tokens of documents, 32 heads, 262 -> 253; 16 samples of about 1130, 24 heads, 445 both.
constexpr int DQ_ALT_LDS_BYTES = (4 + 3) * RunTile<128>::bytes(FK);
template <bool CAUSAL, bool WINDOW = false>
__device__ inline void dq_alt_tile(
    unsigned char* lds, int block, const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v, int ld,
    int ldk, const bf16_t* __restrict__ d_o, int ldo, const float* __restrict__ lse,
    const float* __restrict__ delta, const int32_t* __restrict__ cu, const int32_t* __restrict__ cuk,
    int S, bf16_t* __restrict__ dq, int ldd, int Ttot, int Hq, int group, float scale, float scale_log2,
    SeqOrder ord, LocalMask w = {0, 0, nullptr}) {
  constexpr int DH = 128;
  using RT = RunTile<DH>;
  constexpr int KS = DH / 16, NB = DH / 32, KBL = FK / 32, TILE = RT::bytes(FK), RUNS = FK / RT::RPR / 8;
  constexpr int KRING = 4, VRING = 3;                     // a K tile is read as rows in one phase, as columns two later
  static_assert((KRING + VRING) * TILE == DQ_ALT_LDS_BYTES && TILE % 16 == 0, "the caller's piece of LDS");
  unsigned char* const Kbuf = lds;
  unsigned char* const Vbuf = lds + KRING * TILE;
  int seq, qt, nqt, tile_id, hq;
  tile_and_head(Hq, &tile_id, &hq, block);
  if (WINDOW ? !find_tile(cu, cu + 1, ord, S, AQ, tile_id, &seq, &qt, &nqt) : !find_tile(cu, ord, S, AQ, tile_id, &seq, &qt, &nqt)) return;
  const int hk = hq / group;
  const int lo = cu[seq], L = cu[seq + 1] - lo;
  const int lok = cuk[seq], Lk = (WINDOW ? w.key_end[seq] : cuk[seq + 1]) - lok, off = WINDOW ? Lk - L : 0;
  const int q0 = qt * AQ;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qfirst = q0 + wave * 32;
  const int qpos = qfirst + (lane & 31);                  // this lane's query (column of S^T)
  const int qrow = min(qpos, L - 1);
  bf16x8 qf[KS], dof[KS];
  {
    const bf16_t* qp = q + (size_t)(lo + qrow) * ld + hq * DH;
    const bf16_t* dp = d_o + (size_t)(lo + qrow) * ldo + hq * DH;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[ks] = load_chunk<DH>(qp, ks * 2 + half);
      dof[ks] = load_chunk<DH>(dp, ks * 2 + half);
    }
  }
  const float my_lse = lse[(size_t)hq * Ttot + lo + qrow] * LOG2E;
  const float my_delta = delta[(size_t)hq * Ttot + lo + qrow];
  f32x16 dqacc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) dqacc[j] = f32x16{};
  // key tiles of the workgroup, and those of this wavefront (none if its queries lie past the sequence)
  const auto walk = [&] {
    if constexpr (WINDOW) return KeyWalk<FK>(w, off, q0, AQ, Lk);
    else return AllKeys<FK>(CAUSAL, q0, AQ, Lk);
  }();
  const int nkt = walk.n;
  const int mine = qfirst >= L ? 0 : CAUSAL ? min(nkt, (qfirst + 31) / FK + 1) : nkt;
  const int plain = CAUSAL ? min(Lk / FK, (qfirst + 1) / FK) : Lk / FK;   // leading tiles that need no mask test
  const bf16_t* kbase = scalar_ptr(k + (size_t)lok * ldk + hk * DH);
  const bf16_t* vbase = scalar_ptr(v + (size_t)lok * ldk + hk * DH);
  const uint32_t klds = (uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char*)Kbuf;
  const uint32_t vlds = (uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char*)Vbuf;
  // does this wavefront take part in tile t
  auto takes = [&](int t) {
    if constexpr (WINDOW) return t < nkt && qfirst < L && !none_visible(w, walk.tile(t) * FK, FK, off + qfirst, 32);
    else return t < mine;
  };
  // tile t of K or V into a ring slot; rows past the keys are clamped (their dS is 0)
  auto fetch = [&](const bf16_t* base, uint32_t dst, int t) {
    if (t >= nkt) return;
    const int l = fresh_lane();
    const int key0 = walk.tile(t) * FK;
    const bf16_t* src = base + (size_t)key0 * ldk;
    const int last = Lk - key0 - 1;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      const int r = wave * RUNS + i;
      const uint32_t at = (uint32_t)min(r * RT::RPR + RT::load_row(l), last) * (uint32_t)ldk * 2u + (uint32_t)RT::load_chunk(l) * 16u;
      TileAsync<FK, DH, 512>::load16(src, at, dst + r * RT::RUN);
    }
  };
  f32x16 sacc[KBL], dpacc[KBL];
  bf16x8 ds[KBL][2];
  auto scores = [&](int kslot, int vslot) {               // S^T = K Q^T, dP^T = V dO^T of a key tile
    const int at = RT::rows_at(fresh_lane());
    int ka = kslot * TILE + at, va = vslot * TILE + at;
    asm volatile("" : "+v"(ka), "+v"(va));                 // one register each; the rest is immediates
    constexpr int NSTEP = KBL * KS, AHEAD = 2;             // step n: key block n % KBL, k-step n / KBL
    bf16x8 fk[AHEAD + 1], fv[AHEAD + 1];
    auto request = [&](int n) {
      fk[n % (AHEAD + 1)] = RT::read_rows(Kbuf + ka, n % KBL, n / KBL);
      fv[n % (AHEAD + 1)] = RT::read_rows(Vbuf + va, n % KBL, n / KBL);
    };
#pragma unroll
    for (int b = 0; b < KBL; ++b) sacc[b] = dpacc[b] = f32x16{};
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) request(n);
#pragma unroll
    for (int n = 0; n < NSTEP; ++n) {
      if (n + AHEAD < NSTEP) request(n + AHEAD);
      sacc[n % KBL] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[n % (AHEAD + 1)], qf[n / KBL], sacc[n % KBL], 0, 0, 0);
      dpacc[n % KBL] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv[n % (AHEAD + 1)], dof[n / KBL], dpacc[n % KBL], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto accumulate = [&](int kslot) {                      // dQ^T += K^T dS^T
    int at = kslot * TILE + RT::cols_at(fresh_lane());
    asm volatile("" : "+v"(at));
    constexpr int NSTEP = KBL * 2 * NB, AHEAD = 3;         // step n: 16 keys n / NB, 32 columns n % NB
    bf16x8 f[AHEAD + 1];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) f[n] = RT::read_cols(Kbuf + at, n % NB, n / NB);
#pragma unroll
    for (int n = 0; n < NSTEP; ++n) {
      if (n + AHEAD < NSTEP) f[(n + AHEAD) % (AHEAD + 1)] = RT::read_cols(Kbuf + at, (n + AHEAD) % NB, (n + AHEAD) / NB);
      dqacc[n % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n % (AHEAD + 1)], ds[n / NB / 2][n / NB % 2], dqacc[n % NB], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto softmax = [&](int t) {
    const int key0 = walk.tile(t) * FK;
    if constexpr (WINDOW) {
      if (!all_visible(w, key0, FK, off + qfirst, 32)) {
        asm volatile("");                                  // keeps the tests out of the tiles that need none
        const int h4 = (fresh_lane() >> 5) * 4;
        hide_scores<KBL>(w, key0, off + qfirst, off + qfirst + (fresh_lane() & 31) - key0 - h4, h4, sacc);
      }
    } else if (t >= plain) {
      asm volatile("");                                    // keeps the tests out of the tiles that need none
      const int h4 = (fresh_lane() >> 5) * 4, left = Lk - key0 - h4, ahead = qfirst + (fresh_lane() & 31) - key0 - h4;
#pragma unroll
      for (int b = 0; b < KBL; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int e = b * 32 + (r >> 2) * 8 + (r & 3);
          if (e >= left || (CAUSAL && e > ahead)) sacc[b][r] = -INFINITY;   // P = 0
        }
    }
#pragma unroll
    for (int b = 0; b < KBL; ++b) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sacc[b][r], scale_log2, -my_lse));
        dpacc[b][r] = p * (dpacc[b][r] - my_delta);
      }
      ds[b][0] = acc_to_operand(dpacc[b], 0);
      ds[b][1] = acc_to_operand(dpacc[b], 1);
    }
  };
  settle_compiler_loads();                                // Q and dO fragments, lse, delta, offsets
  fetch(kbase, klds, 0);
  fetch(vbase, vlds, 0);
  fetch(kbase, klds + TILE, 1);
  fetch(vbase, vlds + TILE, 1);
  wait_async_tiles();
  phase_barrier();
  if (wave >= 4) phase_barrier();                         // the second group stays one phase behind
  if (takes(0)) scores(0, 0);
  phase_barrier();
  for (int t = 0, v1 = 1, v2 = 2; t < nkt; ++t) {         // V slots of tiles t + 1, t + 2
    // both groups are past the tiles these overwrite (K t - 2, V t - 1); they are read two phases from now
    fetch(kbase, klds + ((t + 2) & (KRING - 1)) * TILE, t + 2);
    fetch(vbase, vlds + v2 * TILE, t + 2);
    if (takes(t)) softmax(t);
    phase_barrier();
    if (takes(t)) accumulate(t & (KRING - 1));
    if (takes(t + 1)) scores((t + 1) & (KRING - 1), v1);
    wait_async_tiles();
    phase_barrier();
    v1 = v2;
    v2 = v2 == VRING - 1 ? 0 : v2 + 1;
  }
  if (wave < 4) phase_barrier();
  if (qpos < L) {
    bf16_t* pq = dq + (size_t)(lo + qpos) * ldd + hq * DH;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (bf16_t)(dqacc[j][g * 4 + e] * scale);
        *reinterpret_cast<bf16x4*>(pq + j * 32 + g * 8 + half * 4) = w;
      }
  }
}

// ... and of the head sizes above 64, in workgroups of eight wavefronts: dK/dV by pairs of wavefronts (WIDE: with 64 keys a
// pair), dQ with turns (ALT) or as the 128 rows of two heads side by side -- the same sequence and tile, so that both
// halves of the workgroup make the same steps and meet at the same barriers; with an odd number of heads the last
// workgroup's second half repeats the first and stores nothing.  Two launches -> one, us: 32 heads, 300 tokens 39 -> 27, causal
// documents of 8192 tokens 561 -> 534; 32 / 8 heads, 777 causal tokens 76 -> 55, 39000 tokens of heavy-tailed documents 9349 -> 8839;
// 16 two-stream samples of 1170 tokens, 24 heads, 1104 -> 1028.  The kernels with turns hold more than the 102 scalar registers there
// are (5 to 16 spill into lanes of a vector register; apart, dQ spilled two).
template <int DH, bool CAUSAL, bool WIDE, bool ALT>
__global__ __launch_bounds__(512, 2) void fa_bwd_joint512_kernel(
    const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v, int ld, int ldk,
    const bf16_t* __restrict__ d_o, int ldo, const float* __restrict__ lse, const float* __restrict__ delta,
    const int32_t* __restrict__ cuq, const int32_t* __restrict__ cuk, int S, bf16_t* __restrict__ dq, int ldd,
    bf16_t* __restrict__ dk, bf16_t* __restrict__ dv, int ldd_kv, int Tq, int Tk, int Hkv, int group, float scale,
    float scale_log2, int gsplit, float* __restrict__ part, int kv_wgs, SeqOrder ord_kv, SeqOrder ord_q) {
  constexpr int KV = WIDE ? DKDV_WIDE_LDS_BYTES : dkdv_pair_lds_bytes<DH>(), Q = ALT ? DQ_ALT_LDS_BYTES : 2 * dq_lds_bytes<DH>();
  __shared__ __attribute__((aligned(1024))) unsigned char lds[KV > Q ? KV : Q];
  const int Hq = Hkv * group;
  if ((int)blockIdx.x < kv_wgs) {
    if constexpr (WIDE)
      dkdv_wide_tile<CAUSAL>(lds, blockIdx.x, q, k, v, ld, ldk, d_o, ldo, lse, delta, cuq, cuk, S, dk, dv, ldd_kv, Tq, Tk, Hkv,
                             group, scale, scale_log2, gsplit, part, ord_kv);
    else
      dkdv_pair_tile<DH, CAUSAL>(lds, blockIdx.x, q, k, v, ld, ldk, d_o, ldo, lse, delta, cuq, cuk, S, dk, dv, ldd_kv, Tq, Tk,
                                 Hkv, group, scale, scale_log2, gsplit, part, ord_kv);
  } else if constexpr (ALT) {
    dq_alt_tile<CAUSAL>(lds, blockIdx.x - kv_wgs, q, k, v, ld, ldk, d_o, ldo, lse, delta, cuq, cuk, S, dq, ldd, Tq, Hq, group,
                        scale, scale_log2, ord_q);
  } else {
    int tile, heads;
    tile_and_head((Hq + 1) / 2, &tile, &heads, blockIdx.x - kv_wgs);
    const int side = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), head = heads * 2 + side;
    dq_tile<DH, CAUSAL>(lds + side * dq_lds_bytes<DH>(), threadIdx.x & 255, tile, min(head, Hq - 1), head < Hq, q, k, v, ld, ldk,
                        d_o, ldo, lse, delta, cuq, cuk, S, dq, ldd, Tq, group, scale, scale_log2, ord_q);
  }
}

// dk, dv = sum over the q-head parts of the fp32 partials, in part order
__global__ void fa_dkdv_reduce_kernel(const float* __restrict__ part, int gsplit, int Ttot, int W /* Hkv*dh */,
                                      bf16_t* __restrict__ dk, bf16_t* __restrict__ dv, int ldd) {
  const long i = ((long)blockIdx.x * blockDim.x + threadIdx.x) * 4;
  const long plane = (long)Ttot * W;
  if (i >= plane) return;
  const int t = (int)(i / W), c = (int)(i % W);
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int g = 0; g < gsplit; ++g) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(part + ((size_t)g * 2 + which) * plane + i);
      s[0] += v[0]; s[1] += v[1]; s[2] += v[2]; s[3] += v[3];
    }
    bf16x4 w = {(bf16_t)s[0], (bf16_t)s[1], (bf16_t)s[2], (bf16_t)s[3]};
    *reinterpret_cast<bf16x4*>((which == 0 ? dk : dv) + (size_t)t * ldd + c) = w;
  }
}

// q-head parts per kv head in the dK/dV kernel: more workgroups when few key tiles x kv
// heads would leave most CUs idle (grouped-query attention over a short pack)
int dkdv_group_split(int tiles, int Hkv, int group) {
  const long wgs = (long)tiles * Hkv;
  int want = (int)((1024 + wgs - 1) / wgs);
  int gsplit = 1;
  for (int s = 1; s <= group; ++s)
    if (group % s == 0 && s <= want) gsplit = s;
  return gsplit;
}

// The wide dK/dV kernel (head size 128) or the one with 128 keys per workgroup?  Both hold a CU alone.  Whole
// backward, us, narrow -> wide.  The wide one needs
//  - sequences that 256-key tiles cut about as well: 32 x 257, 16 heads, 168 -> 190;
//  - three workgroups per CU to even out its tiles (8 documents of 411 to 1800, 32 heads, 473 -> 431; 777 tokens, 32 heads, 70 ->
//    88), or, when all tiles take equally long, to be done in one round where the other is not: bidirectional 4 x 400,
//    24 heads, 85 -> 71; under a causal mask the longest tile decides: 4096, 16 heads, 297 -> 360; 2048 + 900 + two short, 16
//    heads, 145 -> 187;
//  - heads of a group that it splits no further than the other, or enough queries per key to pay for the fp32 partials:
//    32 / 8 heads, bidirectional, 24 x 256 (split 4 against 2), 193 -> 243; 12 x 640 403 -> 465; 16 x 1152 1398 -> 1371;
//    causal 4 x 2048 618 -> 639.  dK/dV alone of 8192 x 8192 keys 2207 -> 1875, causal 1138 -> 1002.
bool dkdv_wide(const AttnArgs& a) {
  const int tw = count_tiles(a.kv_cu_host(), a.S, WIDE_KEYS), tn = count_tiles(a.kv_cu_host(), a.S, BK_KEYS);
  if (tw == 0 || tw * 2L * 4 > tn * 5L) return false;
  const int group = a.Hq / a.Hkv, split_w = dkdv_group_split(tw, a.Hkv, group), split_n = dkdv_group_split(tn, a.Hkv, group);
  if (split_w != split_n && keys_per_query(a) < (a.causal ? 3000 : 1100)) return false;
  const long wide = (long)tw * a.Hkv * split_w, narrow = (long)tn * a.Hkv * split_n;
  return wide >= 3 * NUM_CU || (!a.causal && wide <= NUM_CU && narrow > NUM_CU);
}

// What a backward pass launches behind delta: tiles, workgroups, and whether dK/dV and dQ share a grid.
struct BwdPlan { bool wide, alt, together; int key_rows, query_rows, gsplit, kv_wgs, qtiles, q_wgs; };

BwdPlan bwd_plan(const AttnArgs& a) {
  BwdPlan p;
  p.wide = a.dh == 128 && dkdv_wide(a);
  p.alt = a.dh == 128 && queries_alternating(a);
  p.key_rows = p.wide ? WIDE_KEYS : BK_KEYS;
  p.query_rows = p.alt ? AQ : FQ;
  const int ktiles = count_tiles(a.kv_cu_host(), a.S, p.key_rows);
  p.gsplit = ktiles > 0 ? dkdv_group_split(ktiles, a.Hkv, a.Hq / a.Hkv) : 1;
  p.kv_wgs = ktiles * a.Hkv * p.gsplit;
  p.qtiles = count_tiles(a.cu_host, a.S, p.query_rows);
  const bool same_wgs = a.dh <= 64 || p.alt;              // dQ takes the workgroups of dK/dV
  p.q_wgs = p.qtiles * (same_wgs ? a.Hq : (a.Hq + 1) / 2);
  // One launch or two?  One, where dQ takes the same workgroups anyway: head size 64, and 256-row query tiles (60 packs of
  // 1500 to 36000 tokens: 57 faster, 3 % on average, 12 % at best, the slowest -1.6 %).  Where both parts fill whole rounds there is nothing to
  // gain: 32 / 8 heads, 8192 queries and keys 3217 -> 3172, causal 1729 -> 1733; the four pairs of a rank 14668 -> 14612, in eight runs +1.0 %
  // to -0.8 %.  The 128 rows of two heads side by
  // side are slower than two workgroups on a CU, so that is for packs whose workgroups all run at once, or nearly so where a
  // causal mask makes most of them short or the wide dK/dV ones are few and long, and for those whose dQ fits into what
  // a second round of dK/dV leaves idle.
  // Two launches -> one, us: 16 / 4 heads, 777 tokens (168 workgroups) 83 -> 55; 24 heads, 1100 tokens (324) 92 -> 103, causal
  // 86 -> 61; 32 heads, 777 (336) 69 -> 80, causal 69 -> 48; causal 8 x 256 (384) 50 -> 52.5; wide 500 + 700 (320) 89 -> 78, 1300 (368)
  // 147 both; causal 1100 (288 of dK/dV, 432) 91 -> 82; 1500 (384, 576) 168 -> 170, causal 117 -> 121.
  const int both = p.kv_wgs + p.q_wgs;
  const int at_once = p.wide ? NUM_CU * 5 / 4 : a.causal && p.qtiles >= 3 * a.S ? NUM_CU * 3 / 2 : NUM_CU;
  p.together = !a.in_place && (same_wgs || both <= at_once || (p.kv_wgs > NUM_CU && both <= 2 * NUM_CU));
  if (!p.together && !same_wgs) p.q_wgs = p.qtiles * a.Hq;   // a kernel of its own, two workgroups per CU
  return p;
}

template <int DH>
bm_status bwd_launch(const AttnArgs& a, const void* o, const void* d_o, const float* lse, void* dq,
                     void* dk, void* dv, int ldd, float* delta, hipStream_t st) {
  const int ldo = a.Hq * a.dh;
  const int ldd_kv = a.ld_dkv ? a.ld_dkv : ldd;
  const float scale = 1.0f / sqrtf((float)a.dh);
  const float sl2 = scale * LOG2E;
  const long n = (long)a.T * a.Hq;
  if (n > 0)
    hipLaunchKernelGGL((fa_delta_kernel<DH>), dim3(cdiv(n * DeltaLanes<DH>::N, 256)), dim3(256), 0, st, (const bf16_t*)o,
                       (const bf16_t*)d_o, ldo, delta, a.T, a.Hq);
  const BwdPlan p = bwd_plan(a);
  const bool wide = p.wide, alt = p.alt;
  const int gsplit = p.gsplit;
  float* part = delta + align_up((size_t)a.Hq * a.T, 64);      // after the delta plane
  const int Tk = a.kv_T();
  // a key tile runs as long as its sequence has queries, a query tile as long as it has keys
  const SeqOrder ord_kv = make_seq_order(a.kv_cu_host(), a.cu_host, a.S, p.key_rows, !a.causal);
  const SeqOrder ord_q = make_seq_order(a.cu_host, a.kv_cu_host(), a.S, p.query_rows, !a.causal);
  // workgroups of dK/dV, then of dQ
  auto launch = [&](int kv, int q) {
    auto go = [&](auto kern, int threads) {
      hipLaunchKernelGGL(kern, dim3(kv + q), dim3(threads), 0, st, (const bf16_t*)a.q, (const bf16_t*)a.k, (const bf16_t*)a.v,
                         a.ld_qkv, a.kv_ld(), (const bf16_t*)d_o, ldo, lse, (const float*)delta, a.cu_dev, a.kv_cu_dev(), a.S,
                         (bf16_t*)dq, ldd, (bf16_t*)dk, (bf16_t*)dv, ldd_kv, a.T, Tk, a.Hkv, a.Hq / a.Hkv, scale, sl2, gsplit, part,
                         kv, ord_kv, ord_q);
    };
    if (kv + q == 0) return;
    if constexpr (DH <= 64) {
      go(a.causal ? fa_bwd_joint_kernel<DH, true> : fa_bwd_joint_kernel<DH, false>, 256);
    } else if constexpr (DH == 128) {
      if (wide && alt) go(a.causal ? fa_bwd_joint512_kernel<DH, true, true, true> : fa_bwd_joint512_kernel<DH, false, true, true>, 512);
      else if (wide) go(a.causal ? fa_bwd_joint512_kernel<DH, true, true, false> : fa_bwd_joint512_kernel<DH, false, true, false>, 512);
      else if (alt) go(a.causal ? fa_bwd_joint512_kernel<DH, true, false, true> : fa_bwd_joint512_kernel<DH, false, false, true>, 512);
      else go(a.causal ? fa_bwd_joint512_kernel<DH, true, false, false> : fa_bwd_joint512_kernel<DH, false, false, false>, 512);
    } else {
      go(a.causal ? fa_bwd_joint512_kernel<DH, true, false, false> : fa_bwd_joint512_kernel<DH, false, false, false>, 512);
    }
  };
  if (p.together) {
    launch(p.kv_wgs, p.q_wgs);
  } else {
    launch(p.kv_wgs, 0);
    bool same_wgs = true;
    if constexpr (DH > 64) same_wgs = alt;
    if (same_wgs) {
      launch(0, p.q_wgs);
    } else if constexpr (DH > 64) {
      if (p.q_wgs > 0) {
        auto kern = a.causal ? fa_bwd_dq_kernel<DH, true> : fa_bwd_dq_kernel<DH, false>;
        hipLaunchKernelGGL(kern, dim3(p.q_wgs), dim3(256), 0, st, (const bf16_t*)a.q, (const bf16_t*)a.k, (const bf16_t*)a.v,
                           a.ld_qkv, a.kv_ld(), (const bf16_t*)d_o, ldo, lse, (const float*)delta, a.cu_dev, a.kv_cu_dev(), a.S,
                           (bf16_t*)dq, ldd, a.T, a.Hq, a.Hq / a.Hkv, scale, sl2, ord_q);
      }
    }
  }
  if (gsplit > 1 && p.kv_wgs > 0) {
    const long n4 = (long)Tk * a.Hkv * a.dh / 4;
    hipLaunchKernelGGL(fa_dkdv_reduce_kernel, dim3(cdiv(n4, 256)), dim3(256), 0, st, part, gsplit, Tk,
                       a.Hkv * a.dh, (bf16_t*)dk, (bf16_t*)dv, ldd_kv);
  }
  BM_CHECK_LAUNCH("fa_bwd");
  return BM_OK;
}

// =============================================================================
// sliding window: the kernels above with WINDOW, and what joins the parts of first keys
// =============================================================================
// The backward pass in one grid: the parts of first keys, the other key tiles, then dQ, which fills what they leave (as in
// fa_bwd_joint_kernel and fa_bwd_joint512_kernel; head size 72, 16 heads, dQ of 128 rows apart -> here: 8192 tokens 280 -> 275 us, 4096 178 -> 160,
// 777 59 -> 38, 32768 2765 -> 2796).  At head size 128 dQ takes 256 rows and turns: 128 rows of two heads side by side are behind by 0 to 6 %
// (8192 tokens, 32 / 8 heads, window 256 435 -> 455, 2048 957 -> 972, before tests of a tile's front and back came apart).
struct WindowBwdArgs {
  const bf16_t *q, *k, *v, *d_o;
  const float *lse, *delta;
  const int32_t *cuq, *cuk;
  bf16_t *dq, *dk, *dv;
  float* part;
  int ld, ldk, ldo, ldd, ldd_kv, S, Tq, Tk, Hkv, group, gsplit, kv_wgs;      // kv_wgs: the parts' among them
  float scale, scale_log2;
};
// A part of 32 first keys: every wavefront walks 32-query tiles of its own (heads of the group, then rows) through its own piece of LDS,
// without a barrier, with both accumulators in registers; K and V are read from LDS by all, the sums meet there at the end, in pairs.
// Bound by latency, which the wavefronts hide from one another.
template <int DH, int W> constexpr int first_keys_lds_bytes() { return (2 + 2 * W) * 32 * HeadDim<DH>::DHL * 2 + W * 64 * 4; }
template <int DH, int W>
__device__ inline void first_keys_part(unsigned char* lds, int block, const WindowBwdArgs& a, const FirstKeys& f) {
  constexpr int DHL = HeadDim<DH>::DHL, KS = HeadDim<DH>::KS, NB = HeadDim<DH>::NB, TILE = 32 * DHL;
  using Tile = TileAsync<32, DH, 64>;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  bf16_t* const Ks = reinterpret_cast<bf16_t*>(lds);
  bf16_t* const Vs = Ks + TILE;
  bf16_t* const Qs = Ks + (2 + 2 * wave) * TILE;
  bf16_t* const Ds = Qs + TILE;
  float* const stats = reinterpret_cast<float*>(Ks + (2 + 2 * W) * TILE) + wave * 64;
  int part_id, hk_gs, seq, n;
  tile_and_head(a.Hkv * a.gsplit, &part_id, &hk_gs, block);
  if (!find_part(f, a.cuq, a.S, part_id, &seq, &n)) return;
  const int hk = hk_gs / a.gsplit, gpart = a.group / a.gsplit, head0 = hk * a.group + hk_gs % a.gsplit * gpart;
  const int lo = a.cuk[seq], L = f.mask.key_end[seq] - lo, loq = a.cuq[seq], Lq = a.cuq[seq + 1] - loq, off = L - Lq;
  const int qlo = n * f.rows, qhi = min(Lq, qlo + f.rows), nqt = (qhi - qlo + 31) / 32, iters = nqt * gpart, kpos = lane & 31;
  Tile tq, td;
  tq.init(a.ld, lane);
  td.init(a.ldo, lane);
  Tile::zero_padding(Qs, lane);
  Tile::zero_padding(Ds, lane);
  if (wave < 2) {
    Tile tk;
    tk.init(a.ldk, lane);
    Tile::zero_padding(wave == 0 ? Ks : Vs, lane);
    tk.issue((wave == 0 ? a.k : a.v) + (size_t)lo * a.ldk + hk * DH, a.ldk, L, wave == 0 ? Ks : Vs, 0);
  }
  f32x16 dk[NB], dv[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) dk[j] = dv[j] = f32x16{};
  wait_async_tiles();
  __syncthreads();                                         // K and V
  for (int it = wave; it < iters; it += W) {
    const int hq = head0 + it / nqt, q0 = qlo + it % nqt * 32;
    tq.issue(a.q + (size_t)(loq + q0) * a.ld + hq * DH, a.ld, Lq - q0, Qs, 0);
    td.issue(a.d_o + (size_t)(loq + q0) * a.ldo + hq * DH, a.ldo, Lq - q0, Ds, 0);
    const float x = (half ? a.delta : a.lse)[(size_t)hq * a.Tq + loq + min(q0 + kpos, Lq - 1)];
    stats[lane] = half ? x : x * LOG2E;                    // lse in base 2, then delta
    wait_async_tiles();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (a wavefront's own rows: no barrier)
    __builtin_amdgcn_wave_barrier();
    const SeenBy seen = seen_by(f.mask, kpos, L, off, q0 + half * 4, qhi);
    f32x16 s = {}, dp = {};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<DHL>(Qs, 0, ks, lane), frag_rows<DHL>(Ks, 0, ks, lane), s, 0, 0, 0);
      dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<DHL>(Ds, 0, ks, lane), frag_rows<DHL>(Vs, 0, ks, lane), dp, 0, 0, 0);
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 l4 = *reinterpret_cast<const f32x4*>(stats + g * 8 + half * 4), d4 = *reinterpret_cast<const f32x4*>(stats + 32 + g * 8 + half * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = g * 4 + e;
        const float x = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale_log2, -l4[e])), p = (uint32_t)(g * 8 + e - seen.from) < seen.n ? x : 0.f;
        s[r] = p;
        dp[r] = fminf(p, 1.0f) * (dp[r] - d4[e]);          // (no probability is above 1, see handed_p)
      }
    }
    const bf16x8 p0 = acc_to_operand(s, 0), p1 = acc_to_operand(s, 1), s0 = acc_to_operand(dp, 0), s1 = acc_to_operand(dp, 1);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      dv[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DHL>(Ds, j * 32, 0, lane), p0, dv[j], 0, 0, 0);
      dv[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DHL>(Ds, j * 32, 16, lane), p1, dv[j], 0, 0, 0);
      dk[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DHL>(Qs, j * 32, 0, lane), s0, dk[j], 0, 0, 0);
      dk[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DHL>(Qs, j * 32, 16, lane), s1, dk[j], 0, 0, 0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // Q, dO and the statistics have been read
  }
  // a wavefront's 2 NB x 16 sums a lane take the place of its partner's tiles
  float* const sums = reinterpret_cast<float*>(Ks + 2 * TILE);
  auto meet = [&](float* at, bool give) {
#pragma unroll
    for (int j = 0; j < 2 * NB; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x16& acc = j < NB ? dk[j] : dv[j - NB];
        f32x4* const to = reinterpret_cast<f32x4*>(at + (j * 4 + g) * 256 + lane * 4);
        if (give) {
          *to = f32x4{acc[g * 4], acc[g * 4 + 1], acc[g * 4 + 2], acc[g * 4 + 3]};
        } else {
          const f32x4 x = *to;
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[g * 4 + e] += x[e];
        }
      }
  };
#pragma unroll
  for (int h = W / 2; h > 0; h /= 2) {
    __syncthreads();                                       // tiles and earlier sums have been read
    if (wave >= h && wave < 2 * h) meet(sums + (wave - h) * 2 * TILE, true);
    __syncthreads();
    if (wave < h) meet(sums + wave * 2 * TILE, false);
  }
  if (wave != 0) return;
  float* const pk = f.out + (((size_t)part_id * (a.Hkv * a.gsplit) + hk_gs) * 2 * 32 + kpos) * DH;
#pragma unroll
  for (int j = 0; j < 2 * NB; ++j)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = (j < NB ? j : j - NB) * 32 + g * 8 + half * 4;
      const f32x16& acc = j < NB ? dk[j] : dv[j - NB];
      const float m = j < NB ? a.scale : 1.0f;
      if (DH % 32 == 0 || c < DH)
        *reinterpret_cast<f32x4*>(pk + (j < NB ? 0 : 32 * DH) + c) = f32x4{acc[g * 4] * m, acc[g * 4 + 1] * m, acc[g * 4 + 2] * m, acc[g * 4 + 3] * m};
    }
}

template <int DH>
__global__ __launch_bounds__(256, 2) void fa_window_bwd_kernel(WindowBwdArgs a, SeqOrder ord_kv, SeqOrder ord_q, FirstKeys first) {
  constexpr int TILES = dkdv_lds_bytes<DH>() > dq_lds_bytes<DH>() ? dkdv_lds_bytes<DH>() : dq_lds_bytes<DH>();
  constexpr int LDS = first_keys_lds_bytes<DH, 4>() > TILES ? first_keys_lds_bytes<DH, 4>() : TILES;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[LDS];
  if (first.keys == 32 && (int)blockIdx.x < first.wgs) {
    first_keys_part<DH, 4>(lds, blockIdx.x, a, first);
  } else if ((int)blockIdx.x < a.kv_wgs) {
    dkdv_tile<DH, true, true>(lds, blockIdx.x, a.q, a.k, a.v, a.ld, a.ldk, a.d_o, a.ldo, a.lse, a.delta, a.cuq, a.cuk, a.S, a.dk, a.dv,
                              a.ldd_kv, a.Tq, a.Tk, a.Hkv, a.group, a.scale, a.scale_log2, a.gsplit, a.part, ord_kv, first);
  } else {
    int tile, head;
    tile_and_head(a.Hkv * a.group, &tile, &head, blockIdx.x - a.kv_wgs);
    dq_tile<DH, true, true>(lds, threadIdx.x, tile, head, true, a.q, a.k, a.v, a.ld, a.ldk, a.d_o, a.ldo, a.lse, a.delta, a.cuq, a.cuk,
                            a.S, a.dq, a.ldd, a.Tq, a.group, a.scale, a.scale_log2, ord_q, first.mask);
  }
}

template <int DH, bool WIDE>
__global__ __launch_bounds__(512, 2) void fa_window_bwd512_kernel(WindowBwdArgs a, SeqOrder ord_kv, SeqOrder ord_q, FirstKeys first) {
  constexpr int PAIR = dkdv_pair_lds_bytes<DH>(), KV = WIDE && DKDV_WIDE_LDS_BYTES > PAIR ? DKDV_WIDE_LDS_BYTES : PAIR;
  constexpr int Q = DH == 128 ? DQ_ALT_LDS_BYTES : 2 * dq_lds_bytes<DH>();
  constexpr int TILES = KV > Q ? KV : Q, LDS = first_keys_lds_bytes<DH, 8>() > TILES ? first_keys_lds_bytes<DH, 8>() : TILES;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[LDS];
  const int Hq = a.Hkv * a.group;
  if (first.keys == 32 && (int)blockIdx.x < first.wgs) {
    first_keys_part<DH, 8>(lds, blockIdx.x, a, first);
  } else if ((int)blockIdx.x < (WIDE ? first.wgs : a.kv_wgs)) {
    dkdv_pair_tile<DH, true, true>(lds, blockIdx.x, a.q, a.k, a.v, a.ld, a.ldk, a.d_o, a.ldo, a.lse, a.delta, a.cuq, a.cuk, a.S, a.dk, a.dv,
                                   a.ldd_kv, a.Tq, a.Tk, a.Hkv, a.group, a.scale, a.scale_log2, a.gsplit, a.part, ord_kv, first);
  } else if (WIDE && (int)blockIdx.x < a.kv_wgs) {
    if constexpr (WIDE)
      dkdv_wide_tile<true, true>(lds, blockIdx.x, a.q, a.k, a.v, a.ld, a.ldk, a.d_o, a.ldo, a.lse, a.delta, a.cuq, a.cuk, a.S, a.dk, a.dv,
                                 a.ldd_kv, a.Tq, a.Tk, a.Hkv, a.group, a.scale, a.scale_log2, a.gsplit, a.part, ord_kv, first);
  } else if constexpr (DH == 128) {
    dq_alt_tile<true, true>(lds, blockIdx.x - a.kv_wgs, a.q, a.k, a.v, a.ld, a.ldk, a.d_o, a.ldo, a.lse, a.delta, a.cuq, a.cuk, a.S, a.dq,
                            a.ldd, a.Tq, Hq, a.group, a.scale, a.scale_log2, ord_q, first.mask);
  } else {
    int tile, heads;
    tile_and_head((Hq + 1) / 2, &tile, &heads, blockIdx.x - a.kv_wgs);
    const int side = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), head = heads * 2 + side;
    dq_tile<DH, true, true>(lds + side * dq_lds_bytes<DH>(), threadIdx.x & 255, tile, min(head, Hq - 1), head < Hq, a.q, a.k, a.v, a.ld,
                            a.ldk, a.d_o, a.ldo, a.lse, a.delta, a.cuq, a.cuk, a.S, a.dq, a.ldd, a.Tq, a.group, a.scale, a.scale_log2,
                            ord_q, first.mask);
  }
}

template <int DH>
__global__ __launch_bounds__(256, 2) void fa_window_dq_kernel(WindowBwdArgs a, SeqOrder ord, LocalMask w) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[dq_lds_bytes<DH>()];
  int tile, head;
  tile_and_head(a.Hkv * a.group, &tile, &head, blockIdx.x);
  dq_tile<DH, true, true>(lds, threadIdx.x, tile, head, true, a.q, a.k, a.v, a.ld, a.ldk, a.d_o, a.ldo, a.lse, a.delta, a.cuq, a.cuk, a.S,
                          a.dq, a.ldd, a.Tq, a.group, a.scale, a.scale_log2, ord, w);
}

// the sequence that is the id-th of those whose first keys are in parts
__device__ inline bool find_split(const FirstKeys& f, const int32_t* __restrict__ cuq, int S, int id, int* seq) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < S; s0 += 64) {
    const int s = min(s0 + lane, S - 1);
    uint64_t split = __builtin_amdgcn_ballot_w64(s0 + lane < S && f.parts(cuq[s + 1] - cuq[s]) > 0);
    const int n = __builtin_popcountll(split);
    if (id < n) {
      for (; id > 0; --id) split &= split - 1;
      *seq = s0 + __builtin_ctzll(split);
      return true;
    }
    id -= n;
  }
  return false;
}
// dk, dv of the key tiles that were left in fp32 -- parts of the first keys, q-head parts of any -- summed in order and
// rounded once.  grid: x the key tiles (all of them, or with one q-head part the first ones that are in parts), y kv heads, z few rows, so
// that a thread has one column to sum (up to hundreds of partials, eight in flight).
constexpr int REDUCE_ROWS = 4;
__global__ __launch_bounds__(256) void fa_window_reduce_kernel(
    const float* __restrict__ part, int gsplit, const int32_t* __restrict__ cuq, const int32_t* __restrict__ cuk, int S, int Ttot,
    int Hkv, int dh, bf16_t* __restrict__ dk, bf16_t* __restrict__ dv, int ldd, int all_tiles, SeqOrder ord, FirstKeys first) {
  __shared__ int before;
  int seq, kt = 0, nkt;
  if (all_tiles) {
    if (!find_tile(cuk, first.mask.key_end, ord, S, BK_KEYS, blockIdx.x, &seq, &kt, &nkt)) return;
    kt = nkt - 1 - kt;
  } else if (!find_split(first, cuq, S, blockIdx.x, &seq)) {
    return;
  }
  const int row0 = blockIdx.z * REDUCE_ROWS, parts = kt == 0 && row0 < first.keys ? first.parts(cuq[seq + 1] - cuq[seq]) : 0;
  if (!all_tiles && parts == 0) return;
  const int lo = cuk[seq], L = first.mask.key_end[seq] - lo, hk = blockIdx.y;
  const float* src;
  size_t step_gs, step_part, row_stride, which_stride;
  int n = 1;
  if (parts > 0) {
    if (threadIdx.x == 0) before = 0;
    __syncthreads();
    int mine = 0;
    for (int s = threadIdx.x; s < seq; s += 256) mine += first.parts(cuq[s + 1] - cuq[s]);
    if (mine) atomicAdd(&before, mine);                    // (whole numbers: any order)
    __syncthreads();
    n = parts;
    which_stride = (size_t)first.keys * dh;
    step_gs = 2 * which_stride;
    step_part = step_gs * Hkv * gsplit;
    row_stride = dh;
    src = first.out + before * step_part + (size_t)hk * gsplit * step_gs;
  } else {
    which_stride = (size_t)Ttot * Hkv * dh;
    step_gs = 2 * which_stride;
    step_part = 0;
    row_stride = (size_t)Hkv * dh;
    src = part + (size_t)(lo + kt * BK_KEYS) * row_stride + hk * dh;
  }
  const int rows = min(REDUCE_ROWS, L - kt * BK_KEYS - row0), quads = dh / 4;
  for (int i = threadIdx.x; i < 2 * rows * quads; i += 256) {
    const int c = i % quads * 4, r = i / quads % rows, which = i / quads / rows;
    const float* p = src + which * which_stride + (size_t)(row0 + r) * row_stride + c;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int j = 0; j < n * gsplit; ++j) {                 // parts in order, q-head parts within them
      const f32x4 v = *reinterpret_cast<const f32x4*>(p + (j / gsplit) * step_part + (j % gsplit) * step_gs);
      s[0] += v[0]; s[1] += v[1]; s[2] += v[2]; s[3] += v[3];
    }
    const bf16x4 w = {(bf16_t)s[0], (bf16_t)s[1], (bf16_t)s[2], (bf16_t)s[3]};
    *reinterpret_cast<bf16x4*>((which == 0 ? dk : dv) + (size_t)(lo + kt * BK_KEYS + row0 + r) * ldd + hk * dh + c) = w;
  }
}

int count_tiles(const int32_t* begin, const int32_t* end, int S, int rows) {
  long n = 0;
  for (int s = 0; s < S; ++s) n += (end[s] - begin[s] + rows - 1) / rows;
  return (int)n;
}

// (256-row tiles and turns, as the backward pass has them, are slower: us, 32 / 8 heads of 128, 8192 tokens, window 1024 172 -> 216, 256 92 ->
// 145; 4 documents of 8192, window 4096, 1776 -> 1787.)
template <int DH>
bm_status window_fwd_launch(const AttnArgs& a, void* o, float* lse, hipStream_t st) {
  const SeqOrder ord = make_seq_order(a.cu_host, a.kv_cu_host(), a.S, FQ, false);
  hipLaunchKernelGGL((fa_fwd_kernel<DH, true, true>), dim3(count_tiles(a.cu_host, a.S, FQ) * a.Hq), dim3(256), 0, st, (const bf16_t*)a.q,
                     (const bf16_t*)a.k, (const bf16_t*)a.v, a.ld_qkv, a.kv_ld(), a.cu_dev, a.kv_cu_dev(), a.S, (bf16_t*)o, a.Hq * a.dh, lse,
                     a.T, a.Hq, a.Hq / a.Hkv, LOG2E / sqrtf((float)a.dh), ord, a.local);
  BM_CHECK_LAUNCH("fa_window_fwd");
  return BM_OK;
}

// Few queries of a sequence (rows x heads of a group <= 32) behind long key lists: a workgroup takes a part of the keys of one
// sequence and kv head, its four wavefronts a quarter of it each.  The rows -- token by token, head by head of the group -- are the
// 32 columns of S^T, so K and V are read once for the whole group.  Each wavefront streams its own tiles of 32 keys through places of
// its own in LDS, without a barrier: the next tile's K follows as soon as this one's is in registers, its V behind the products with
// V.  The four meet in LDS at the end, the parts of a sequence in window_join_kernel.
// Bound by reading K and V: 64 sequences of up to 4096 visible keys, 8 kv heads of 128, 153 us, 5.75 TB/s; 1000 of 1024 6.4 (places for two tiles in a
// workgroup that has a CU alone: 186 us; 59 sequences of 300, 16 heads of 64, 42 instead of 15).
template <int DH> constexpr int token_ring() { return DH == 64 ? 2 : 1; }
template <int DH, bool STREAM>
__global__ __launch_bounds__(256, 2) void fa_window_token_kernel(
    const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v, int ld, int ldk,
    const int32_t* __restrict__ cu, const int32_t* __restrict__ cuk, int S, bf16_t* __restrict__ o, int ldo,
    float* __restrict__ lse, int Ttot, int Hkv, int group, float scale_log2, LocalMask w, TokenSplit split) {
  constexpr int DHL = HeadDim<DH>::DHL, KS = HeadDim<DH>::KS, NB = HeadDim<DH>::NB, TILE = TOKEN_KEYS * DHL;
  constexpr int RING = token_ring<DH>(), OS = DH == 128 ? DH : DH + 4;       // OS: row stride of what a wavefront leaves
  using Tile = TileAsync<TOKEN_KEYS, DH, 64, STREAM>;
  constexpr int CH = Tile::CH;                             // loads of a tile of K or V
  static_assert(RING * 2 * TILE * 2 >= 32 * OS * 4, "a wavefront's sums take its tiles' place");
  __shared__ __attribute__((aligned(1024))) bf16_t ring[4 * RING * 2 * TILE];
  __shared__ float stats[4][32][2];
  int hk;
  const int slot = token_slot(split, Hkv, blockIdx.x, &hk);
  TokenPart where;
  if (!find_token_part(split, S, slot, &where)) return;
  const int seq = where.seq, nparts = where.parts;
  const int lo = cu[seq], L = cu[seq + 1] - lo, lok = cuk[seq], Lk = w.key_end[seq] - lok, off = Lk - L;
  const KeyWalk<TOKEN_KEYS> walk(w, off, 0, L, Lk);
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int per = (walk.n + nparts - 1) / nparts, first = where.part * per, last = min(walk.n, first + per), share = (last - first + 3) / 4;
  const int t0 = first + wave * share, t1 = min(last, t0 + share), n = t1 - t0;   // this wavefront's tiles (n <= 0: none)
  const int rows = L * group, row = min(lane & 31, rows - 1), at = off + row / group, begin = window_begin(w, off);
  bf16_t* const mine = ring + wave * (RING * 2 * TILE);
  Tile tile;
  tile.init(ldk, lane);
#pragma unroll
  for (int b = 0; b < 2 * RING; ++b) Tile::zero_padding(mine + b * TILE, lane);
  const bf16_t* kbase = k + (size_t)lok * ldk + hk * DH;
  const bf16_t* vbase = v + (size_t)lok * ldk + hk * DH;
  bf16x8 qf[KS];
  {
    const bf16_t* qp = q + (size_t)(lo + row / group) * ld + (hk * group + row % group) * DH;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = load_chunk<DH>(qp, ks * 2 + half);
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the padding
  // this wavefront's tile i into its place; K and V lie behind one another
  auto fetch = [&](const bf16_t* base, int i, bf16_t* dst) {
    tile.issue(w, begin, base, ldk, walk.tile(t0 + i) * TOKEN_KEYS, Lk, dst, 0);
  };
  f32x16 oacc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) oacc[j] = f32x16{};
  float m = NO_MAX, lsum = 0.f;
  settle_compiler_loads();                                 // Q, offsets
#pragma unroll
  for (int i = 0; i < RING; ++i)
    if (i < n) {
      fetch(kbase, i, mine + i * 2 * TILE);
      fetch(vbase, i, mine + i * 2 * TILE + TILE);
    }
  int place = 0;                                           // i % RING
  for (int i = 0; i < n; ++i) {
    bf16_t* const Ks = mine + place * 2 * TILE;
    bf16_t* const Vs = Ks + TILE;
    // K of tile i is there: behind it only its V and the whole tiles up to i + RING - 1
    if (RING == 2 && i + 1 < n) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(3 * CH) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" :: "n"(CH) : "memory");
    f32x16 sacc = {};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 f = frag_rows<DHL>(Ks, 0, ks, lane);
      sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[ks], sacc, 0, 0, 0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // K has been read: its place is free
    const bool more = i + RING < n;
    if (more) fetch(kbase, i + RING, Ks);
    const int key0 = walk.tile(t0 + i) * TOKEN_KEYS;
    if (!all_visible(w, key0, TOKEN_KEYS, off, L))
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (hidden(w, key0 + (r >> 2) * 8 + half * 4 + (r & 3), at)) sacc[r] = -INFINITY;
    float mx = sacc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sacc[r]);
    mx = max_with_other_half(mx) * scale_log2;
    if (__builtin_amdgcn_ballot_w64(mx > m + 8.0f) != 0) {  // lazy rescaling, as in fa_fwd_kernel
      const float m_new = fmaxf(m, mx), corr = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      lsum *= corr;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[j][r] *= corr;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sacc[r] = __builtin_amdgcn_exp2f(fmaf(sacc[r], scale_log2, -m));
      lsum += sacc[r];
    }
    const bf16x8 p0 = acc_to_operand(sacc, 0), p1 = acc_to_operand(sacc, 1);
    // V of tile i is there: behind it only the loads of later tiles
    if (more) asm volatile("s_waitcnt vmcnt(%0)" :: "n"((2 * RING - 1) * CH) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      oacc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DHL>(Vs, j * 32, 0, lane), p0, oacc[j], 0, 0, 0);
      oacc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DHL>(Vs, j * 32, 16, lane), p1, oacc[j], 0, 0, 0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // so has V
    if (more) fetch(vbase, i + RING, Vs);
    place = place + 1 == RING ? 0 : place + 1;
  }
  lsum = sum_with_other_half(lsum);
  float* const sums = reinterpret_cast<float*>(mine);
  if ((lane & 31) < rows) {
    if (half == 0) { stats[wave][lane & 31][0] = m; stats[wave][lane & 31][1] = lsum; }
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        if (DH % 32 == 0 || j * 32 + g * 8 + half * 4 < DH)
          *reinterpret_cast<f32x4*>(sums + (lane & 31) * OS + j * 32 + g * 8 + half * 4) =
              f32x4{oacc[j][g * 4], oacc[j][g * 4 + 1], oacc[j][g * 4 + 2], oacc[j][g * 4 + 3]};
  }
  __syncthreads();
  const float* all = reinterpret_cast<const float*>(ring);
  constexpr int WSTRIDE = RING * TILE;                     // floats between the wavefronts' sums
  for (int e = tid; e < rows * DH; e += 256) {
    const int r = e / DH, c = e % DH;
    float top = NO_MAX;
#pragma unroll
    for (int x = 0; x < 4; ++x) top = fmaxf(top, stats[x][r][0]);
    float sum = 0.f, val = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float f = __builtin_amdgcn_exp2f(stats[x][r][0] - top);
      sum = fmaf(f, stats[x][r][1], sum);
      val = fmaf(f, all[x * WSTRIDE + r * OS + c], val);
    }
    const int t = lo + r / group, h = hk * group + r % group;
    if (nparts == 1) {
      o[(size_t)t * ldo + h * DH + c] = (bf16_t)(val / sum);
      if (c == 0) lse[(size_t)h * Ttot + t] = (top + log2f(sum)) * LN2;
    } else {
      const size_t at_row = ((size_t)where.place * Hkv + hk) * split.rows + r;
      split.sums[at_row * DH + c] = val;
      if (c == 0) {
        split.stats[at_row * 2] = top;
        split.stats[at_row * 2 + 1] = sum;
      }
    }
  }
}

template <int DH>
bm_status window_token_launch(const AttnArgs& a, const TokenSplit& split, void* o, float* lse, hipStream_t st) {
  auto kern = split.stream ? fa_window_token_kernel<DH, true> : fa_window_token_kernel<DH, false>;
  hipLaunchKernelGGL(kern, dim3(token_grid(split, a.Hkv)), dim3(256), 0, st, (const bf16_t*)a.q, (const bf16_t*)a.k, (const bf16_t*)a.v, a.ld_qkv,
                     a.kv_ld(), a.cu_dev, a.kv_cu_dev(), a.S, (bf16_t*)o, a.Hq * a.dh, lse, a.T, a.Hkv,
                     a.Hq / a.Hkv, LOG2E / sqrtf((float)a.dh), a.local, split);
  BM_CHECK_LAUNCH("fa_window_token");
  return BM_OK;
}

// What the backward pass of a window takes as workspace, by sizes that do not depend on single lengths
struct WindowBwd {
  int gsplit, keys, part_rows;
  long parts;                          // at most
  size_t delta, split, first;          // floats of the three pieces
};
WindowBwd window_bwd(int window, int sinks, int Hq, int Hkv, int dh, int S, int Tq, int Tk) {
  WindowBwd w;
  const int tiles = cdiv(Tk, BK_KEYS) > S ? cdiv(Tk, BK_KEYS) : S;
  // as without a window, but for 512 workgroups: dQ follows in the same grid, and the tiles of a window are short for the fp32 partials.
  // us, for 1024 -> 512 -> 256, 4 first tokens: 32 / 8 heads of 128, 8192 tokens, window 2048 940 -> 882 -> 881, 256 378 -> 304 -> 303; 4096, 1024, 348 -> 306
  // -> 298; 32 / 8 of 64, 4096, 1024, 184 -> 174 -> 156, 2048 90 all three; 8 / 1 of 128, 32768, window 4096, 1827 -> 1771 -> 1937.
  w.gsplit = dkdv_group_split(2 * tiles, Hkv, Hq / Hkv);
  // Up to 32 first tokens: the 128-key tile would compute four times what they need.  us, parts of 128 keys -> of 32, 32 / 8 heads of 128, 4 first tokens:
  // 8192 tokens, window 2048 903 -> 882, 1024 587 -> 557, 256 340 -> 304, 64 234 -> 222; 2048, 128 115 -> 104; 16 / 16 heads of 64, 8192, 256 101 -> 92.
  w.keys = sinks <= 32 ? 32 : BK_KEYS;
  // Rows of a part: short where the longest workgroup decides, long where partials cost more.  us, 256 -> 512 -> 1024 rows for 32 keys: 439 tokens, window 16,
  // 32 / 8 heads of 128 37.5 -> 42 -> 42, 16 / 16 of 64 23.5 all three; 4096, 256, 16 / 16 of 128 109 -> 103 -> 107; 32 / 8 of 128, 8192, 1024 595 -> 552 -> 557, 256
  // 317 -> 310 -> 304, 24 documents, 1024, 286 -> 272 -> 262.  Of 128 keys, as long as the tiles of other keys; 192 -> 512: 780 tokens, window 1, 16 / 16 heads of
  // 64 24 -> 28; 8192, 256, 5 / 1 of 128 150 -> 118.
  const bool few = (long)Tq * Hq <= 20480;
  if (w.keys == 32) {
    w.part_rows = few ? 256 : Tq < 6144 ? 512 : 1024;
  } else {
    const int rows = (int)align_up(window < 4096 ? window : 4096, BK_Q), least = few ? 192 : 512;
    w.part_rows = rows < least ? least : rows;
  }
  w.parts = sinks > 0 ? 2L * Tq / w.part_rows : 0;         // a sequence that is split has more rows than one part
  w.delta = align_up((size_t)Hq * Tq, 64);
  w.split = w.gsplit > 1 ? (size_t)w.gsplit * 2 * Tk * Hkv * dh : 0;
  w.first = (size_t)w.parts * Hkv * w.gsplit * 2 * w.keys * dh;
  return w;
}

// The wide dK/dV kernel (head size 128) or the one with 128 keys per workgroup?  dQ fills what either leaves of the chip, so the wide one needs no
// whole rounds, but windows as long as its tile, sequences that 256-key tiles cut about as well, and enough workgroups.  Whole backward, us, narrow ->
// wide, 32 / 8 heads: 8192 tokens, window 2048 943 -> 881, 1024 592 -> 552, 256 312 -> 306, but 64 229 -> 242; 24 documents, 1024, 275 -> 261; 16 / 16 heads,
// 8192, 256 196 -> 188, 2048 tokens (128 workgroups), 1024, 101 -> 95; but 2 documents in 777 (128 of 32 / 8, 64 of 16 / 16 heads) 53 -> 60, 38 -> 47; 5 / 1
// heads, 2048 (40) 39 -> 48.
bool window_wide(const AttnArgs& a, int gsplit) {
  const int tw = count_tiles(a.kv_cu_host(), a.key_end_host, a.S, WIDE_KEYS), tn = count_tiles(a.kv_cu_host(), a.key_end_host, a.S, BK_KEYS);
  const long wgs = (long)tw * a.Hkv * gsplit;
  return a.local.window >= 256 && tw * 8L <= tn * 5L && (wgs >= NUM_CU || (wgs >= NUM_CU / 2 && tw >= 4 * a.S));
}

// What a backward pass launches
struct WindowBwdPlan {
  WindowBwd sizes;
  bool apart, wide;                    // dQ in a launch of its own, 256 keys a workgroup of dK/dV
  int query_rows, key_rows, key_tiles, part_wgs, kv_wgs, q_wgs, split_seqs;      // key_tiles: of 128; kv_wgs: the parts' among them; split_seqs: in parts
  int wgs() const { return kv_wgs + (apart ? 0 : q_wgs); }                       // of the grid that holds dK/dV
};
template <int DH>
WindowBwdPlan window_bwd_plan(const AttnArgs& a) {
  WindowBwdPlan p;
  p.sizes = window_bwd(a.local.window, a.local.sinks, a.Hq, a.Hkv, a.dh, a.S, a.T, a.kv_T());
  FirstKeys first;
  first.mask = a.local;
  first.rows = p.sizes.part_rows;
  long parts = 0;
  p.split_seqs = 0;
  for (int s = 0; s < a.S; ++s) {
    const int n = first.parts(a.cu_host[s + 1] - a.cu_host[s]);
    parts += n;
    p.split_seqs += n > 0;
  }
  // dQ of narrow windows apart, in tiles of 128 rows and two workgroups to a CU, where there are enough of them: us, together -> apart, 8192 tokens, 32 / 8
  // heads, 4 first tokens: window 16 230 -> 217, 64 226 -> 222, 128 259 -> 261, 256 303 -> 313; 16 / 16 heads 149 -> 139, 148 -> 142, 168 -> 164, 184 -> 186; but 2048
  // tokens, 16 / 16 heads, 64 (256 of them) 52 -> 57.  Without first tokens 208 -> 177, 203 -> 180, 229 -> 207, 277 -> 257.
  p.apart = DH == 128 && a.local.window <= 64 && count_tiles(a.cu_host, a.S, FQ) * a.Hq >= 2 * NUM_CU;
  p.query_rows = DH == 128 && !p.apart ? AQ : FQ;
  p.wide = DH == 128 && window_wide(a, p.sizes.gsplit);
  p.key_rows = p.wide ? WIDE_KEYS : BK_KEYS;
  p.key_tiles = count_tiles(a.kv_cu_host(), a.key_end_host, a.S, BK_KEYS);
  p.part_wgs = (int)parts * a.Hkv * p.sizes.gsplit;
  p.kv_wgs = p.part_wgs + (p.wide ? count_tiles(a.kv_cu_host(), a.key_end_host, a.S, WIDE_KEYS) : p.key_tiles) * a.Hkv * p.sizes.gsplit;
  p.q_wgs = count_tiles(a.cu_host, a.S, p.query_rows) * cdiv(a.Hq, DH == 72 ? 2 : 1);
  return p;
}

template <int DH>
bm_status window_bwd_launch(const AttnArgs& a, const void* o, const void* d_o, const float* lse, void* dq, void* dk, void* dv,
                            int ldd, float* delta, hipStream_t st) {
  const int ldo = a.Hq * a.dh, Tk = a.kv_T(), group = a.Hq / a.Hkv;
  const float scale = 1.0f / sqrtf((float)a.dh), sl2 = scale * LOG2E;
  const WindowBwdPlan p = window_bwd_plan<DH>(a);
  const WindowBwd& wb = p.sizes;
  float* part = delta + wb.delta;
  FirstKeys first;
  first.mask = a.local;
  first.keys = wb.keys;
  first.rows = wb.part_rows;
  first.wgs = p.part_wgs;
  first.out = part + wb.split;
  first.ord = make_seq_order(a.cu_host, a.cu_host, a.S, wb.part_rows, false);
  for (int i = 0; i < first.ord.n && i < a.S; ++i)
    first.ord.w[i] = (uint32_t)first.parts(a.cu_host[i + 1] - a.cu_host[i]) << 8 | (uint32_t)i;
  const SeqOrder ord_kv = make_seq_order(a.kv_cu_host(), a.cu_host, a.S, p.key_rows, false, a.key_end_host);
  const SeqOrder ord_q = make_seq_order(a.cu_host, a.cu_host, a.S, p.query_rows, false);
  const WindowBwdArgs w{(const bf16_t*)a.q, (const bf16_t*)a.k, (const bf16_t*)a.v, (const bf16_t*)d_o, lse, delta, a.cu_dev, a.kv_cu_dev(),
                        (bf16_t*)dq, (bf16_t*)dk, (bf16_t*)dv, part, a.ld_qkv, a.kv_ld(), ldo, ldd, a.ld_dkv, a.S, a.T, Tk, a.Hkv, group,
                        wb.gsplit, p.kv_wgs, scale, sl2};
  const int wgs = p.wgs();
  // Workgroups of 512 threads for both kinds of tiles: at head size 128 tens of thousands of sequences of many heads come to more.
  BM_ARG_CHECK((long)wgs * (DH <= 64 ? 256 : 512) < (1L << 32), "window attention: the gradients' %d workgroups are past a grid of 2^32 threads", wgs);
  if (a.T > 0)
    hipLaunchKernelGGL((fa_delta_kernel<DH>), dim3(cdiv((long)a.T * a.Hq * DeltaLanes<DH>::N, 256)), dim3(256), 0, st,
                       (const bf16_t*)o, (const bf16_t*)d_o, ldo, delta, a.T, a.Hq);
  if (wgs > 0) {
    if constexpr (DH <= 64) hipLaunchKernelGGL(fa_window_bwd_kernel<DH>, dim3(wgs), dim3(256), 0, st, w, ord_kv, ord_q, first);
    else {
      auto kern = fa_window_bwd512_kernel<DH, false>;
      if constexpr (DH == 128) if (p.wide) kern = fa_window_bwd512_kernel<DH, true>;
      hipLaunchKernelGGL(kern, dim3(wgs), dim3(512), 0, st, w, ord_kv, ord_q, first);
    }
  }
  if constexpr (DH == 128)
    if (p.apart && p.q_wgs > 0) hipLaunchKernelGGL((fa_window_dq_kernel<DH>), dim3(p.q_wgs), dim3(256), 0, st, w, ord_q, a.local);
  const int all_tiles = wb.gsplit > 1;
  if (p.kv_wgs > 0 && (all_tiles || p.part_wgs > 0)) {
    const SeqOrder ord = p.wide ? make_seq_order(a.kv_cu_host(), a.cu_host, a.S, BK_KEYS, false, a.key_end_host) : ord_kv;
    hipLaunchKernelGGL(fa_window_reduce_kernel, dim3(all_tiles ? p.key_tiles : p.split_seqs, a.Hkv, BK_KEYS / REDUCE_ROWS), dim3(256), 0, st, part,
                       wb.gsplit, a.cu_dev, a.kv_cu_dev(), a.S, Tk, a.Hkv, a.dh, (bf16_t*)dk, (bf16_t*)dv, a.ld_dkv, all_tiles,
                       ord, first);
  }
  BM_CHECK_LAUNCH("fa_window_bwd");
  return BM_OK;
}

}  // namespace

size_t window_backward_mfma_scratch_bytes(int window, int sinks, int Hq, int Hkv, int dh, int S, int Tq, int Tk) {
  const WindowBwd w = window_bwd(window, sinks, Hq, Hkv, dh, S, Tq, Tk);
  return align_up((w.delta + w.split + w.first) * sizeof(float), 256);
}

bm_status window_forward_mfma(const AttnArgs& a, void* o, float* lse, hipStream_t st) {
  if (a.dh == 128) return window_fwd_launch<128>(a, o, lse, st);
  if (a.dh == 72) return window_fwd_launch<72>(a, o, lse, st);
  return window_fwd_launch<64>(a, o, lse, st);
}

bm_status window_tokens_mfma(const AttnArgs& a, const TokenSplit& split, void* o, float* lse, hipStream_t st) {
  if (a.dh == 128) return window_token_launch<128>(a, split, o, lse, st);
  if (a.dh == 72) return window_token_launch<72>(a, split, o, lse, st);
  return window_token_launch<64>(a, split, o, lse, st);
}

bm_status window_backward_mfma(const AttnArgs& a, const void* o, const void* d_o, const float* lse, void* dq, void* dk,
                               void* dv, int ld_dq, void* scratch, hipStream_t st) {
  if (a.dh == 128) return window_bwd_launch<128>(a, o, d_o, lse, dq, dk, dv, ld_dq, (float*)scratch, st);
  if (a.dh == 72) return window_bwd_launch<72>(a, o, d_o, lse, dq, dk, dv, ld_dq, (float*)scratch, st);
  return window_bwd_launch<64>(a, o, d_o, lse, dq, dk, dv, ld_dq, (float*)scratch, st);
}

// keys of a workgroup of dK/dV, rows of one of dQ, launches of both, parts of first keys (times their heads)
void window_backward_mfma_plan(const AttnArgs& a, int32_t* out) {
  const WindowBwdPlan p = a.dh == 128 ? window_bwd_plan<128>(a) : a.dh == 72 ? window_bwd_plan<72>(a) : window_bwd_plan<64>(a);
  out[0] = p.key_rows;
  out[1] = p.query_rows;
  out[2] = p.apart ? 2 : 1;
  out[3] = p.part_wgs;
}

bool attention_mfma_supported(const AttnArgs& a) {
  return a.dtype == BM_DTYPE_BF16 && (a.dh == 64 || a.dh == 72 || a.dh == 128) && a.ld_qkv % 8 == 0 &&
         a.kv_ld() % 8 == 0;
}

bm_status attention_forward_mfma(const AttnArgs& a, void* o, float* lse, hipStream_t st) {
  if (a.dh == 128) return fwd_launch<128>(a, o, lse, st);
  if (a.dh == 72) return fwd_launch<72>(a, o, lse, st);
  return fwd_launch<64>(a, o, lse, st);
}

void attention_mfma_plan(const AttnArgs& a, int* fwd_rows, int* dq_rows, int* dkdv_rows) {
  const bool alt = a.dh != 72 && queries_alternating(a);
  *fwd_rows = alt ? AQ : FQ;
  *dq_rows = alt && a.dh == 128 ? AQ : FQ;
  *dkdv_rows = a.dh == 128 && dkdv_wide(a) ? WIDE_KEYS : BK_KEYS;
}

void attention_mfma_backward_plan(const AttnArgs& a, int* launches, int* dkdv_wgs, int* dq_wgs) {
  const BwdPlan p = bwd_plan(a);
  *launches = p.together ? 1 : 2;
  *dkdv_wgs = p.kv_wgs;
  *dq_wgs = p.q_wgs;
}

size_t attention_backward_mfma_scratch_bytes(int Hq, int Hkv, int dh, int Tq, int Tk) {
  // the delta plane of the query rows, then room for the fp32 dK/dV partials of the largest
  // q-head split
  const size_t delta = align_up((size_t)Hq * Tq, 64) * sizeof(float);
  const int group = Hq / Hkv;
  const size_t part = group > 1 ? (size_t)group * 2 * Tk * Hkv * dh * sizeof(float) : 0;
  return align_up(delta + part, 256);
}

bm_status attention_backward_mfma(const AttnArgs& a, const void* o, const void* d_o, const float* lse,
                                  void* dq, void* dk, void* dv, int ld_dqkv, void* scratch,
                                  size_t, hipStream_t st) {
  if (a.dh == 128) return bwd_launch<128>(a, o, d_o, lse, dq, dk, dv, ld_dqkv, (float*)scratch, st);
  if (a.dh == 72) return bwd_launch<72>(a, o, d_o, lse, dq, dk, dv, ld_dqkv, (float*)scratch, st);
  return bwd_launch<64>(a, o, d_o, lse, dq, dk, dv, ld_dqkv, (float*)scratch, st);
}

}  // namespace bm
