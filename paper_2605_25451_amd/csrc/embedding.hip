// Token embeddings: the scaled lookup and the gradient of the table.
//
// The lookup is a copy of rows: bound by HBM (the rows written, and the distinct rows read).
//
// The gradient sums the rows of dy that belong to the same word.  Three launches (one for up to 128 tokens), none of them
// with floating-point atomics:
//   group    the text tokens, word by word, each word's in the order of the pack.  256 workgroups, one
//            for the ids with the same low 8 bits: words are drawn by frequency, and neighbouring ids
//            are about equally frequent, so low bits share a pack far better than ranges of ids would.
//            A workgroup reads all ids (they lie in L2), counts those of the buckets before its own --
//            where its tokens go -- and collects its own; a stable counting sort by the other bits in
//            LDS puts them into order.
//   sum      chunks of equally many grouped rows, whatever words they are, so that a word with a tenth
//            of the pack costs no more than as many rows of rare ones.  A word that lies inside a chunk
//            is added to the table at once, its pieces in several chunks go to the workspace.
//   fold     adds up the pieces of those words, in order.
// Bound by HBM: dy once, the rows of distinct words read and written in fp32.
#include "train.h"

#include <algorithm>

namespace bm {

namespace {

// ---- lookup ---------------------------------------------------------------------------------

// lanes: threads of a row, a power of two up to 64; VEC: whole 16 bytes
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void embed_kernel(const T* __restrict__ table, long ld_table, const int32_t* __restrict__ ids,
                                                    int n, int V, int d, float scale, T* __restrict__ y, long ld_y, int log_lanes) {
  constexpr int W = VEC ? Elt<T>::VEC : 1;
  const long row = ((long)blockIdx.x * 256 + threadIdx.x) >> log_lanes;
  if (row >= n) return;
  const int id = ids[row];
  if (id < 0) return;
  const bool known = id < V;
  const T* src = table + (size_t)(known ? id : 0) * ld_table;
  T* dst = y + (size_t)row * ld_y;
  const int step = W << log_lanes;
  const float nan = __builtin_nanf("");
#pragma unroll 8
  for (int c = (threadIdx.x & ((1 << log_lanes) - 1)) * W; c < d; c += step) {
    if constexpr (VEC) {
      float v[W];
      load16(src + c, v);
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] = known ? v[e] * scale : nan;
      store16(dst + c, v);
    } else {
      dst[c] = Elt<T>::from_f(known ? Elt<T>::to_f(src[c]) * scale : nan);
    }
  }
}

// ---- group ----------------------------------------------------------------------------------

constexpr int BUCKET_BITS = 8, BUCKETS = 1 << BUCKET_BITS;
constexpr int DIGIT_BITS = 10, DIGITS = 1 << DIGIT_BITS;
constexpr int GROUP_THREADS = 1024, GROUP_WAVES = GROUP_THREADS / WAVE;
constexpr int RANKED = 256;                    // tokens of a bucket that are ordered by comparing all with all ...
constexpr int HELD = 8192;                     // ... and that are kept in LDS
constexpr int BATCH = 8;                       // loads of ids in flight

// a wavefront's share of n tokens, in whole 64
__device__ inline int share(int n) { return (n + GROUP_WAVES * WAVE - 1) / (GROUP_WAVES * WAVE) * WAVE; }

// word[i], pos[i]: the id and the row of the i-th grouped token; *count: how many there are
struct Grouped { int32_t *word, *pos, *word2, *pos2, *count; };

// f(index, id) for first <= index < last, 64 at a time and all lanes together (id -1 past the end); the ids are loaded in batches
template <typename F>
__device__ inline void for_ids(const int32_t* __restrict__ ids, int first, int last, int lane, F f) {
  for (int i0 = first; i0 < last; i0 += BATCH * WAVE) {
    int id[BATCH];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) id[k] = ids[min(i0 + k * WAVE + lane, last - 1)];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = i0 + k * WAVE + lane;
      if (i0 + k * WAVE < last) f(i, i < last ? id[k] : -1);
    }
  }
}

// digit_bits: of a pass, so that `digit_passes` of them hold the bits above the bucket's
__global__ __launch_bounds__(GROUP_THREADS) void group_kernel(const int32_t* __restrict__ ids, int n, int V, int digit_passes, int digit_bits,
                                                              Grouped g) {
  __shared__ int below[GROUP_WAVES], mine[GROUP_WAVES], wave_total[GROUP_WAVES];
  __shared__ int counts[GROUP_WAVES][DIGITS];
  __shared__ int keys[HELD], rows[HELD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int bucket = blockIdx.x;
  const uint64_t lower_lanes = (1ull << lane) - 1;
  // every wavefront has a contiguous range
  const int per = share(n);
  const int first = min(n, wave * per), last = min(n, first + per);
  auto bucket_of = [&](int id) { return (uint32_t)id < (uint32_t)V ? id & (BUCKETS - 1) : BUCKETS; };
  // Where a lane has up to 64 ids, bit k of `hits` says that the k-th is one of the bucket's: the tokens are then collected without a
  // second look at all ids.
  const int steps = (last - first + WAVE - 1) / WAVE;
  const bool marked = per <= 64 * WAVE;
  int lower = 0, own = 0;
  uint64_t hits = 0;
  if (marked) {
    int k = 0;
    for_ids(ids, first, last, lane, [&](int, int id) {
      const int b = bucket_of(id);
      lower += b < bucket;
      hits |= (uint64_t)(b == bucket) << k++;
    });
    own = __popcll(hits);
  } else {
    for_ids(ids, first, last, lane, [&](int, int id) {
      const int b = bucket_of(id);
      lower += b < bucket;
      own += b == bucket;
    });
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) { lower += __shfl_xor(lower, off, WAVE); own += __shfl_xor(own, off, WAVE); }
  if (lane == 0) { below[wave] = lower; mine[wave] = own; }
  __syncthreads();
  int base = 0, total = 0, at = 0;
#pragma unroll
  for (int w = 0; w < GROUP_WAVES; ++w) {
    base += below[w];
    if (w == wave) at = total;
    total += mine[w];
  }
  if (bucket == BUCKETS - 1 && threadIdx.x == 0) *g.count = base + total;
  if (total == 0) return;
  // f(place, index) for the marked ones, in order
  auto collect = [&](auto f) {
    int to = at;
    for (int k = 0; k < steps; ++k) {
      const bool hit = (hits >> k) & 1;
      const uint64_t m = __ballot(hit);
      if (hit) f(to + __popcll(m & lower_lanes), first + k * WAVE + lane);
      to += __popcll(m);
    }
  };
  const bool held = marked && total <= HELD;
  if (held) {
    collect([&](int to, int i) { rows[to] = i; });
    __syncthreads();
    // (fetched where they are collected, a wavefront would wait for every 64 of them)
    for (int t = threadIdx.x; t < total; t += GROUP_THREADS) keys[t] = ids[rows[t]];
    if (total <= RANKED) {
      // every token counts those that stand before it, the ones of lower words and the earlier ones of its own;
      // GROUP_THREADS / RANKED threads a token
      int* ranks = &counts[0][0];
      if (threadIdx.x < total) ranks[threadIdx.x] = 0;
      __syncthreads();
      const int t = threadIdx.x % RANKED;
      if (t < total) {
        const int key = keys[t];
        int rank = 0;
#pragma unroll 4
        for (int j = threadIdx.x / RANKED; j < total; j += GROUP_THREADS / RANKED) {
          const int other = keys[j];
          rank += other < key || (other == key && j < t);
        }
        atomicAdd(ranks + t, rank);
      }
      __syncthreads();
      if (threadIdx.x < total) {
        g.word[base + ranks[t]] = keys[t];
        g.pos[base + ranks[t]] = rows[t];
      }
      return;
    }
  }
  // an odd number of passes ends in the other pair of arrays: start so that the last one ends in word/pos
  int32_t *word = (digit_passes & 1 ? g.word2 : g.word) + base, *pos = (digit_passes & 1 ? g.pos2 : g.pos) + base;
  int32_t *word_to = (digit_passes & 1 ? g.word : g.word2) + base, *pos_to = (digit_passes & 1 ? g.pos : g.pos2) + base;
  if (!marked) {
    for_ids(ids, first, last, lane, [&](int i, int id) {
      const bool in = bucket_of(id) == bucket;
      const uint64_t m = __ballot(in);
      if (m == 0) return;
      if (in) {
        const int to = at + __popcll(m & lower_lanes);
        word[to] = id;
        pos[to] = i;
      }
      at += __popcll(m);
    });
  } else if (!held || digit_passes == 0) {
    collect([&](int to, int i) { pos[to] = i; });
    __syncthreads();
    for (int t = threadIdx.x; t < total; t += GROUP_THREADS) word[t] = ids[pos[t]];
  }
  // stable counting sorts by the bits above the bucket's, digit_bits at a time
  const int per_own = share(total);
  const int own_first = min(total, wave * per_own), own_last = min(total, own_first + per_own);
  for (int pass = 0; pass < digit_passes; ++pass) {
    const int shift = BUCKET_BITS + pass * digit_bits, mask = (1 << digit_bits) - 1;
    if ((int)threadIdx.x <= mask)
      for (int w = 0; w < GROUP_WAVES; ++w) counts[w][threadIdx.x] = 0;
    __syncthreads();                                       // (the tokens written above are visible behind it, too)
    const bool from_lds = held && pass == 0;
    // the lanes with the same digit, by its bits; the first of them counts for all
    auto same = [&](bool in, int digit) {
      uint64_t m = __ballot(in);
      for (int b = 0; b < digit_bits; ++b) {
        const uint64_t v = __ballot((digit >> b) & 1);
        m &= (digit >> b) & 1 ? v : ~v;
      }
      return m;
    };
    for (int i = own_first + lane; i - lane < own_last; i += WAVE) {
      const bool in = i < own_last;
      const int digit = in ? ((from_lds ? keys[i] : word[i]) >> shift) & mask : 0;
      const uint64_t m = same(in, digit);
      if (in && (m & lower_lanes) == 0) counts[wave][digit] += __popcll(m);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    // counts -> first places: over the digits, and within one over the wavefronts
    static_assert(DIGITS == GROUP_THREADS, "a thread per digit");
    const bool digit_here = (int)threadIdx.x <= mask;
    int sum = 0;
    if (digit_here) {
#pragma unroll
      for (int w = 0; w < GROUP_WAVES; ++w) sum += counts[w][threadIdx.x];
    }
    int scan = sum;
#pragma unroll
    for (int off = 1; off < WAVE; off <<= 1) {
      const int v = __shfl_up(scan, off, WAVE);
      if (lane >= off) scan += v;
    }
    if (lane == 63) wave_total[wave] = scan;
    __syncthreads();
    int run = scan - sum;
    for (int w = 0; w < wave; ++w) run += wave_total[w];
    if (digit_here) {
#pragma unroll
      for (int w = 0; w < GROUP_WAVES; ++w) {
        const int c = counts[w][threadIdx.x];
        counts[w][threadIdx.x] = run;
        run += c;
      }
    }
    __syncthreads();
    for (int i = own_first + lane; i - lane < own_last; i += WAVE) {
      const bool in = i < own_last;
      const int id = !in ? 0 : from_lds ? keys[i] : word[i], p = !in ? 0 : from_lds ? rows[i] : pos[i];
      const int digit = (id >> shift) & mask;
      const uint64_t m = same(in, digit);
      const int before = __popcll(m & lower_lanes);
      if (in) {
        const int to = counts[wave][digit] + before;
        word_to[to] = id;
        pos_to[to] = p;
      }
      // the lanes of a wavefront have all read the place before the first of them moves it on
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (in && before == 0) counts[wave][digit] += __popcll(m);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    int32_t* t = word; word = word_to; word_to = t;
    t = pos; pos = pos_to; pos_to = t;
  }
}

// ---- sum and fold ---------------------------------------------------------------------------

constexpr int COLS = 8;                       // of a lane
constexpr int SLICE = COLS * WAVE;            // of a wavefront
constexpr int AHEAD = 4;                      // rows in flight

// the columns of a lane as they lie in memory
template <typename T>
struct Cols {
  alignas(16) T v[COLS];
  template <bool VEC> __device__ inline void load(const T* p, int left) {
    if constexpr (VEC) {
      constexpr int W = Elt<T>::VEC;
#pragma unroll
      for (int q = 0; q < COLS; q += W)
        if (q < left) *reinterpret_cast<Vec16<T>*>(v + q) = *reinterpret_cast<const Vec16<T>*>(p + q);
    } else {
#pragma unroll
      for (int e = 0; e < COLS; ++e)
        if (e < left) v[e] = p[e];
    }
  }
  __device__ inline float get(int e) const { return Elt<T>::to_f(v[e]); }
};

template <typename T, bool VEC>
__device__ inline void load_cols(const T* p, int left, float (&v)[COLS]) {
  if constexpr (VEC) {
    constexpr int W = Elt<T>::VEC;
#pragma unroll
    for (int q = 0; q < COLS / W; ++q) {
      float t[W];
      if (q * W < left) load16(p + q * W, t);
#pragma unroll
      for (int e = 0; e < W; ++e) v[q * W + e] = q * W < left ? t[e] : 0.f;
    }
  } else {
#pragma unroll
    for (int e = 0; e < COLS; ++e) v[e] = e < left ? Elt<T>::to_f(p[e]) : 0.f;
  }
}
template <bool VEC>
__device__ inline void store_cols(float* p, int left, const float (&v)[COLS]) {
#pragma unroll
  for (int q = 0; q < COLS; q += 4) {
    if constexpr (VEC) {
      if (q < left) *reinterpret_cast<float4*>(p + q) = float4{v[q], v[q + 1], v[q + 2], v[q + 3]};
    } else {
#pragma unroll
      for (int e = q; e < q + 4; ++e)
        if (e < left) p[e] = v[e];
    }
  }
}

constexpr int CHUNK_MIN = 4, CHUNK_MAX = 60;

// What happens behind the last row of a word in a chunk: added to the table, or kept as a piece of a word that lies in
// several chunks -- piece[2 c] where chunk c starts inside the word, piece[2 c + 1] where it only ends inside it.
enum { GOES_ON = 0, ADD, HEAD, TAIL };


// A wavefront: one chunk of grouped rows, one slice of columns.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void sum_kernel(const T* __restrict__ dy, long ld_dy, Grouped g, int n, int d, int chunk, int chunks,
                                                  int slices, float scale, float* __restrict__ dtable, long ld_dtable,
                                                  float* __restrict__ piece, long ld_piece) {
  const int lane = threadIdx.x & 63;
  const long job = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (int)(job / slices), slice = (int)(job % slices);
  if (c >= chunks) return;
  const int first = c * chunk, col = slice * SLICE + lane * COLS, left = d - col;
  // lane l holds the word and the place of row first + l, lane 63 the word in front of the chunk; the one behind it is row `rows`.
  // (Read next to the number of rows, not behind it.)
  static_assert(CHUNK_MAX + 2 <= WAVE, "a chunk and the rows next to it");
  const int mine = lane == 63 ? first - 1 : first + lane, in = max(0, min(mine, n - 1));
  int my_word = g.word[in], my_pos = g.pos[in];
  const int total = *g.count;
  if (first >= total) return;
  const int rows = min(chunk, total - first);
  if (mine < 0 || mine >= total) my_word = -1;
  const int after = __shfl_down(my_word, 1, WAVE);
  // of the row in this lane: its word ends with it
  const uint64_t ends = __ballot(after != my_word);
  bool inside = __builtin_amdgcn_readlane(my_word, 63) == __builtin_amdgcn_readlane(my_word, 0);   // the current word began in an earlier chunk
  float acc[COLS] = {};
  for (int r0 = 0; r0 < rows; r0 += AHEAD) {
    Cols<T> v[AHEAD];
    float old[AHEAD][COLS];
    int then[AHEAD];
    // what the next rows need of dy and of the table is requested together
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int r = r0 + a;
      then[a] = GOES_ON;
      if (r >= rows) continue;
      const bool end = (ends >> r) & 1;
      if (end) then[a] = inside ? HEAD : ADD;
      else if (r + 1 == rows) then[a] = inside ? HEAD : TAIL;
      if (end) inside = false;
      if (left <= 0) continue;
      v[a].template load<VEC>(dy + (size_t)__builtin_amdgcn_readlane(my_pos, r) * ld_dy + col, left);
      if (then[a] == ADD) load_cols<float, VEC>(dtable + (size_t)__builtin_amdgcn_readlane(my_word, r) * ld_dtable + col, left, old[a]);
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int r = r0 + a;
      if (r >= rows || left <= 0) continue;
#pragma unroll
      for (int e = 0; e < COLS; ++e) acc[e] += v[a].get(e);
      if (then[a] == GOES_ON) continue;
      if (then[a] == ADD) {
#pragma unroll
        for (int e = 0; e < COLS; ++e) old[a][e] = fmaf(scale, acc[e], old[a][e]);
        store_cols<VEC>(dtable + (size_t)__builtin_amdgcn_readlane(my_word, r) * ld_dtable + col, left, old[a]);
      } else {
        store_cols<true>(piece + (2l * c + (then[a] == TAIL)) * ld_piece + col, COLS, acc);
      }
#pragma unroll
      for (int e = 0; e < COLS; ++e) acc[e] = 0.f;
    }
  }
}

// A wavefront: the chunk in which a word begins that later chunks go on with, 256 columns.
constexpr int FOLD_COLS = 4 * WAVE;
template <bool VEC>
__global__ __launch_bounds__(256) void fold_kernel(Grouped g, int n, int d, int chunk, int chunks, int slices, float scale,
                                                   float* __restrict__ dtable, long ld_dtable, const float* __restrict__ piece,
                                                   long ld_piece) {
  const int lane = threadIdx.x & 63;
  const long job = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (int)(job / slices), slice = (int)(job % slices);
  if (c + 1 >= chunks) return;
  const int first = c * chunk, end = first + chunk;          // (end < n: c is not the last chunk)
  // the first word of this lane's chunk, c + 1 + lane; read next to the others, not behind them
  long next = end + (long)lane * chunk;
  int at_next = g.word[min(next, (long)n - 1)];
  const int word = g.word[end - 1], at_first = g.word[first], before = g.word[max(first - 1, 0)];
  const int total = *g.count;
  if (end >= total || (first > 0 && before == word && at_first == word)) return;
  // chunks c + 1 .. c + more hold pieces
  int more = 0;
  for (;;) {
    const uint64_t off = ~__ballot(next < total && at_next == word);
    if (off) { more += __ffsll((unsigned long long)off) - 1; break; }
    more += WAVE;
    next += (long)WAVE * chunk;
    at_next = g.word[min(next, (long)n - 1)];
  }
  const int col = slice * FOLD_COLS + lane * 4, left = d - col;
  if (more == 0 || left <= 0) return;
  float* to_row = dtable + (size_t)word * ld_dtable + col;
  float old[4];
  if constexpr (VEC) {
    const float4 v = *reinterpret_cast<const float4*>(to_row);
    old[0] = v.x; old[1] = v.y; old[2] = v.z; old[3] = v.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) old[e] = e < left ? to_row[e] : 0.f;
  }
  float4 acc = *reinterpret_cast<const float4*>(piece + (2l * c + 1) * ld_piece + col);
  constexpr int FLIGHT = 16;
  for (int k0 = 1; k0 <= more; k0 += FLIGHT) {
    float4 v[FLIGHT];
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k)
      if (k0 + k <= more) v[k] = *reinterpret_cast<const float4*>(piece + 2l * (c + k0 + k) * ld_piece + col);
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k)
      if (k0 + k <= more) { acc.x += v[k].x; acc.y += v[k].y; acc.z += v[k].z; acc.w += v[k].w; }
  }
  const float sum[4] = {acc.x, acc.y, acc.z, acc.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) old[e] = fmaf(scale, sum[e], old[e]);
  if constexpr (VEC) {
    *reinterpret_cast<float4*>(to_row) = float4{old[0], old[1], old[2], old[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) to_row[e] = old[e];
  }
}

// ---- few tokens: one launch -------------------------------------------------------------------------
//
// A workgroup: 64 columns, for which it orders the tokens and adds up the rows of every word by itself.  The order is found again in
// every workgroup, by comparing all with all; that costs less than waiting for another launch: 100 tokens of 4096 columns 6.5 us,
// in three launches 10.5; 128 7.2 and 10.6; 256 12.8 and 11.0.
constexpr int FEW = 128, FEW_THREADS = 1024, FEW_WAVES = FEW_THREADS / WAVE;
template <typename T, bool VEC>
__global__ __launch_bounds__(FEW_THREADS) void few_kernel(const T* __restrict__ dy, long ld_dy, const int32_t* __restrict__ ids, int n, int V,
                                                          int d, float scale, float* __restrict__ dtable, long ld_dtable) {
  __shared__ float vals[FEW][WAVE];
  __shared__ int keys[FEW], ranks[FEW], word[FEW], pos[FEW], starts[FEW + 1], runs_of[FEW / WAVE];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col0 = blockIdx.x * WAVE;
  // ids that are none stand behind all words
  int key = INT32_MAX;
  if (tid < n) {
    const int id = ids[tid];
    if ((uint32_t)id < (uint32_t)V) key = id;
  }
  if (tid < FEW) { keys[tid] = key; ranks[tid] = 0; }
  const int total = __syncthreads_count(key != INT32_MAX);
  if (total == 0) return;
  {
    // FEW_THREADS / FEW threads a token
    const int t = tid % FEW, mine = keys[t];
    int rank = 0;
#pragma unroll 4
    for (int j = tid / FEW; j < n; j += FEW_THREADS / FEW) {
      const int other = keys[j];
      rank += other < mine || (other == mine && j < t);
    }
    if (t < n) atomicAdd(ranks + t, rank);
  }
  __syncthreads();
  if (tid < n) { word[ranks[tid]] = key; pos[ranks[tid]] = tid; }
  __syncthreads();
  // a thread: 8 columns of a row
  constexpr int ROWS = FEW_THREADS / 8;
  const int col = col0 + (tid & 7) * COLS, left = d - col;
  Cols<T> v[FEW / ROWS];
#pragma unroll
  for (int k = 0; k < FEW / ROWS; ++k) {
    const int r = k * ROWS + tid / 8;
    if (r < total && left > 0) v[k].template load<VEC>(dy + (size_t)pos[r] * ld_dy + col, left);
  }
  // where words begin
  const bool begins = tid < total && (tid == 0 || word[tid] != word[tid - 1]);
  const uint64_t m = __ballot(begins);
  if (lane == 0 && wave < FEW / WAVE) runs_of[wave] = __popcll(m);
  __syncthreads();
  int runs = 0, before = 0;
#pragma unroll
  for (int w = 0; w < FEW / WAVE; ++w) {
    if (w < wave) before += runs_of[w];
    runs += runs_of[w];
  }
  if (begins) starts[before + __popcll(m & ((1ull << lane) - 1))] = tid;
  if (tid == 0) starts[runs] = total;
  __syncthreads();
  // a wavefront: every 16th word, a column a lane; the table's rows are requested together
  constexpr int EACH = FEW / FEW_WAVES;
  const bool inside = col0 + lane < d;
  float old[EACH];
#pragma unroll
  for (int k = 0; k < EACH; ++k) {
    const int r = k * FEW_WAVES + wave;
    if (r < runs && inside) old[k] = dtable[(size_t)word[starts[r]] * ld_dtable + col0 + lane];
  }
#pragma unroll
  for (int k = 0; k < FEW / ROWS; ++k) {
    const int r = k * ROWS + tid / 8;
    if (r < total && left > 0) {
#pragma unroll
      for (int e = 0; e < COLS; ++e) vals[r][(tid & 7) * COLS + e] = v[k].get(e);
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < EACH; ++k) {
    const int r = k * FEW_WAVES + wave;
    if (r < runs && inside) {
      const int first = starts[r], last = starts[r + 1];
      float acc = 0.f;
#pragma unroll 8
      for (int i = first; i < last; ++i) acc += vals[i][lane];
      dtable[(size_t)word[first] * ld_dtable + col0 + lane] = fmaf(scale, acc, old[k]);
    }
  }
}

// ---- host -------------------------------------------------------------------------------------

// Rows of a chunk: as many as leave 32 wavefronts for every CU.  Longer chunks leave fewer pieces to the words that occur often
// (32768 tokens of 4096 columns, one word in eleven the same: folding chunks of 16 rows 25 us, of 60 rows 13).
constexpr int SUM_WAVES = 8192;
int chunk_rows(int T, int d) {
  const long rows = (long)T * cdiv(d, SLICE) / SUM_WAVES;
  return (int)std::max((long)CHUNK_MIN, std::min((long)CHUNK_MAX, rows));
}
// chunks of any number of tokens up to T: a step from k to k + 1 rows makes them fewer, and is at its widest behind the shortest
size_t max_chunks(int T, int d) {
  const size_t before = (size_t)(CHUNK_MIN + 1) * SUM_WAVES / cdiv(d, SLICE) / CHUNK_MIN + 2;
  return std::max((size_t)cdiv(T, CHUNK_MAX), std::min((size_t)cdiv(T, CHUNK_MIN), before));
}

constexpr int MAX_TOKENS = 1 << 30, MAX_COLUMNS = 1 << 30;

struct Workspace {
  Grouped g;
  float* piece;
  long ld_piece;
  size_t bytes;
  Workspace(void* scratch, int T, int d) {
    Arena a(scratch);
    const size_t ids = (size_t)T * sizeof(int32_t);
    g.word = a.take<int32_t>(ids); g.pos = a.take<int32_t>(ids);
    g.word2 = a.take<int32_t>(ids); g.pos2 = a.take<int32_t>(ids);
    g.count = a.take<int32_t>(sizeof(int32_t));
    ld_piece = (long)align_up((size_t)d, COLS);
    piece = a.take<float>(2 * max_chunks(T, d) * ld_piece * sizeof(float));
    bytes = a.off;
  }
};

template <typename T>
void launch_embed(const void* table, int ld_table, const int32_t* ids, int rows, int V, int d, float scale, void* y, int ld_y,
                  hipStream_t st) {
  constexpr int W = Elt<T>::VEC;
  const bool vec = d % W == 0 && ld_table % W == 0 && ld_y % W == 0;
  const int chunks = vec ? d / W : d;
  int log_lanes = 0;
  while (log_lanes < 6 && (1 << log_lanes) < chunks) ++log_lanes;
  // (a grid has fewer than 2^32 threads)
  const long most = 1l << (31 - log_lanes);
  for (long first = 0; first < rows; first += most) {
    const int n = (int)std::min(most, rows - first);
    const unsigned blocks = (unsigned)((((long)n << log_lanes) + 255) / 256);
    hipLaunchKernelGGL((vec ? embed_kernel<T, true> : embed_kernel<T, false>), dim3(blocks), dim3(256), 0, st, (const T*)table,
                       (long)ld_table, ids + first, n, V, d, scale, (T*)y + first * ld_y, (long)ld_y, log_lanes);
  }
}

template <typename T, bool VEC>
bm_status launch_sums(const void* dy, int ld_dy, const Workspace& w, int n, int d, float scale, float* dtable, int ld_dtable,
                      hipStream_t st) {
  const int chunk = chunk_rows(n, d), chunks = cdiv(n, chunk), slices = cdiv(d, SLICE);
  const long jobs = (long)chunks * slices;
  hipLaunchKernelGGL((sum_kernel<T, VEC>), dim3((unsigned)((jobs + 3) / 4)), dim3(256), 0, st, (const T*)dy, (long)ld_dy, w.g, n, d,
                     chunk, chunks, slices, scale, dtable, (long)ld_dtable, w.piece, w.ld_piece);
  BM_CHECK_LAUNCH("embedding sums");
  if (chunks > 1) {
    const int parts = cdiv(d, FOLD_COLS);
    hipLaunchKernelGGL((fold_kernel<VEC>), dim3((unsigned)(((long)(chunks - 1) * parts + 3) / 4)), dim3(256), 0, st, w.g, n, d, chunk, chunks,
                       parts, scale, dtable, (long)ld_dtable, w.piece, w.ld_piece);
    BM_CHECK_LAUNCH("embedding fold");
  }
  return BM_OK;
}

bm_status check(const char* name, int32_t dtype, int32_t V, int32_t d, int32_t T, int32_t ld0, int32_t ld1) {
  BM_ARG_CHECK(good_dtype(dtype), "%s: dtype %d", name, dtype);
  BM_ARG_CHECK(V > 0 && d > 0, "%s: V and d must be positive", name);
  BM_ARG_CHECK(d <= MAX_COLUMNS, "%s: %d columns", name, d);
  BM_ARG_CHECK(T >= 0 && T <= MAX_TOKENS, "%s: %d tokens", name, T);
  BM_ARG_CHECK(ld0 >= d && ld1 >= d, "%s: leading dimension too small", name);
  // workgroups of a grid
  BM_ARG_CHECK((long)T * cdiv(d, SLICE) < (1l << 31), "%s: %d tokens of %d columns are too many", name, T, d);
  return BM_OK;
}

}  // namespace
}  // namespace bm

using namespace bm;

extern "C" bm_status bm_embedding_forward(int32_t dtype, int32_t V, int32_t d, const void* table, int32_t ld_table,
                                          const int32_t* ids, int32_t T, float scale, void* y, int32_t ld_y, void* hip_stream) {
  BM_RETURN_IF(check("bm_embedding_forward", dtype, V, d, T, ld_table, ld_y));
  if (T == 0) return BM_OK;
  BM_ARG_CHECK(table && ids && y && aligned16(table) && aligned16(ids) && aligned16(y), "bm_embedding_forward: NULL or misaligned tensor");
  hipStream_t st = (hipStream_t)hip_stream;
  ProfScope prof(PROF_ELEMENTWISE, 2.0 * T * d * elt_size(dtype), st);
  if (dtype == BM_DTYPE_BF16) launch_embed<bf16_t>(table, ld_table, ids, T, V, d, scale, y, ld_y, st);
  else launch_embed<float>(table, ld_table, ids, T, V, d, scale, y, ld_y, st);
  BM_CHECK_LAUNCH("embedding lookup");
  return BM_OK;
}

extern "C" size_t bm_embedding_backward_scratch_bytes(int32_t T, int32_t d) {
  if (T <= 0 || T > MAX_TOKENS || d <= 0 || d > MAX_COLUMNS) return 0;
  return Workspace(nullptr, T, d).bytes;
}

extern "C" bm_status bm_embedding_backward(int32_t dtype, int32_t V, int32_t d, const void* dy, int32_t ld_dy, const int32_t* ids,
                                           int32_t T, float scale, float* dtable, int32_t ld_dtable, void* scratch,
                                           size_t scratch_bytes, void* hip_stream) {
  BM_RETURN_IF(check("bm_embedding_backward", dtype, V, d, T, ld_dy, ld_dtable));
  if (T == 0) return BM_OK;
  BM_ARG_CHECK(dy && ids && dtable && aligned16(dy) && aligned16(ids) && aligned16(dtable) && aligned16(scratch),
               "bm_embedding_backward: NULL or misaligned tensor");
  const Workspace w(scratch, T, d);
  if (!scratch || scratch_bytes < w.bytes) {
    set_error("bm_embedding_backward needs %zu scratch bytes, got %zu", w.bytes, scratch_bytes);
    return BM_ERR_WORKSPACE_TOO_SMALL;
  }
  hipStream_t st = (hipStream_t)hip_stream;
  ProfScope prof(PROF_ELEMENTWISE, (double)T * d * (elt_size(dtype) + 8.0), st);
  const int W = dtype == BM_DTYPE_BF16 ? 8 : 4;
  const bool vec = d % W == 0 && ld_dy % W == 0 && ld_dtable % 4 == 0;
  if (T <= FEW) {
    // (a grid has fewer than 2^32 threads)
    constexpr int MOST = 1 << 27;                           // columns of a launch
    auto few = [&](auto kern, auto* rows) -> bm_status {
      for (int c = 0; c < d; c += std::min(MOST, d - c)) {
        const int n = std::min(MOST, d - c);
        hipLaunchKernelGGL(kern, dim3(cdiv(n, WAVE)), dim3(FEW_THREADS), 0, st, rows + c, (long)ld_dy, ids, T, V, n, scale, dtable + c,
                           (long)ld_dtable);
        BM_CHECK_LAUNCH("embedding gradient of few tokens");
      }
      return BM_OK;
    };
    return dtype == BM_DTYPE_BF16 ? few(vec ? few_kernel<bf16_t, true> : few_kernel<bf16_t, false>, (const bf16_t*)dy)
                                  : few(vec ? few_kernel<float, true> : few_kernel<float, false>, (const float*)dy);
  }
  int bits = 0;                                             // of the ids, above those of the bucket
  while (bits < 31 - BUCKET_BITS && ((V - 1) >> (BUCKET_BITS + bits))) ++bits;
  const int passes = cdiv(bits, DIGIT_BITS);
  hipLaunchKernelGGL(group_kernel, dim3(BUCKETS), dim3(GROUP_THREADS), 0, st, ids, T, V, passes, passes ? cdiv(bits, passes) : 0, w.g);
  BM_CHECK_LAUNCH("embedding group");
  if (dtype == BM_DTYPE_BF16)
    return vec ? launch_sums<bf16_t, true>(dy, ld_dy, w, T, d, scale, dtable, ld_dtable, st)
               : launch_sums<bf16_t, false>(dy, ld_dy, w, T, d, scale, dtable, ld_dtable, st);
  return vec ? launch_sums<float, true>(dy, ld_dy, w, T, d, scale, dtable, ld_dtable, st)
             : launch_sums<float, false>(dy, ld_dy, w, T, d, scale, dtable, ld_dtable, st);
}
