// Parts of kernels whose operands go straight from memory into LDS in slices of 64 k: waits, loads, the LDS layouts and the
// fragments of v_mfma_f32_16x16x32 on 16-bit elements (the element type shows in the MFMA only).
#pragma once
#include "gemm_tile.h"

namespace bm {
namespace {

template <int N> using Int = std::integral_constant<int, N>;

template <int N> __device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }
__device__ inline void wait_fragments() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}
__device__ inline void end_phase() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
}
__device__ inline void load_to_lds(const bf16_t* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(lds), "v"(off), "s"(base) : "memory", "m0");
}

// the source of a row, or that of the first row where there is none (the rows that fill up a group)
__device__ inline int source_row(const int32_t* source, int row, int src_rows) {
  const int s = source[row];
  return (uint32_t)s < (uint32_t)src_rows ? s : min(max(source[0], 0), src_rows - 1);
}

// LDS layouts of a region of R rows x 64 k (the swizzles keep fragment reads free of bank conflicts):
//   k-contiguous operand  [row][64 k]: 16-byte chunk c of row r sits at c ^ ((r >> 1) & 7)
//   transposed operand    [k][R rows]: chunk c of k-row k sits at c ^ ((k & 3) << 2) ^ (((k >> 3) & 1) << 1)
//                         R = 64: c ^ (k & 2) ^ (((k >> 3) & 1) << 2)
// (a transpose read of 32 lanes takes 32 bytes of 8 k rows: k .. k + 3 and 8 rows further on.  Rows of 256 bytes all start in the same
// bank, rows of 128 in two that are half of the banks apart)
// A region is filled in LOADS loads per wavefront of WAVES; load i of wavefront w writes the 1 KiB run i*WAVES + w.
template <int R, bool TR, int WAVES = 8>
struct Region {
  static constexpr int LOADS = R / (8 * WAVES);
  static constexpr uint32_t BYTES = R * BK * 2;
  static constexpr int CPR = TR ? R / 8 : KCH;           // chunks per LDS row
  static constexpr int RPL = 64 / CPR;                   // LDS rows per load
  uint32_t off[LOADS];                                   // byte offset from the slice's base pointer
  // LDS row and global chunk of this lane in load i
  static __device__ inline void place(int i, int wave, int lane, int* row, int* chunk) {
    const int r = (i * WAVES + wave) * RPL + lane / CPR;
    *row = r;
    *chunk = (lane % CPR) ^ (TR ? (R == 64 ? (r & 2) ^ (((r >> 3) & 1) << 2) : ((r & 3) << 2) ^ (((r >> 3) & 1) << 1)) : (r >> 1) & 7);
  }
  // row0: this region's first row in the tile; rows past rows_left (counted from the tile's first row)
  // are clamped into the matrix: their products are never stored.
  // half > 0 (k-contiguous only): rows are gathered from two ranges F rows apart -- within every run of
  // 2*half tile rows the first half come from f0.. and the second from F + f0.. (gate and up rows of a
  // SwiGLU weight); offsets are then relative to the matrix's first row.
  // source (k-contiguous only): where the tile's rows lie in a matrix of src_rows rows; offsets are then relative to its first row
  __device__ inline void init(int ld, int row0, int rows_left, int wave, int lane, int half = 0, int F = 0, int f0 = 0,
                              const int32_t* source = nullptr, int src_rows = 0) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      int r, c;
      place(i, wave, lane, &r, &c);
      if (TR) {
        int row = row0 + c * 8;
        if (row >= rows_left) row = 0;
        off[i] = ((uint32_t)r * (uint32_t)ld + (uint32_t)row) * 2u;
      } else {
        int row = min(row0 + r, rows_left - 1);
        if (half > 0) row = (r / half & 1) * F + f0 + (r / (2 * half)) * half + r % half;
        if (source) row = source_row(source, row, src_rows);
        off[i] = ((uint32_t)row * (uint32_t)ld + (uint32_t)c * 8u) * 2u;
      }
    }
  }
  // k_left < 64: a slice that ends inside the k range; what lies past it is fetched from its last
  // valid k (row or chunk) and zeroed in the fragments
  template <bool CUT, int FIRST = 0, int COUNT = LOADS>
  __device__ inline void load(const bf16_t* base, int ld, int k_left, uint32_t lds, int wave, int lane) const {
#pragma unroll
    for (int i = FIRST; i < FIRST + COUNT; ++i) {
      uint32_t o = off[i];
      if (CUT && k_left < BK) {
        int r, c;
        place(i, wave, lane, &r, &c);
        if (TR) { if (r >= k_left) o -= (uint32_t)(r - (k_left - 1)) * (uint32_t)ld * 2u; }
        else if (c * 8 >= k_left) o -= (uint32_t)(c * 8 - (k_left - 8)) * 2u;
      }
      load_to_lds(base, o, lds + (i * WAVES + wave) * 1024);
    }
  }
};

// 16(row) x 32(k) fragments of v_mfma_f32_16x16x32_bf16 from a region of R rows: lane l holds row l%16
// and k = (l/16)*8 .. +7.  NB blocks of 16 rows from row0 on; block q, k-step ks.
template <int R, bool TR, int NB>
struct Fragments {
  static constexpr int NA = TR ? NB : 2;
  uint32_t addr[NA];
  __device__ inline void init(int row0, int lane) {
    const int gi = lane >> 4, s = lane & 15;
#pragma unroll
    for (int q = 0; q < NA; ++q) {
      if (TR) {
        // the 16 lanes of group gi read a 4(k) x 16(row) block, 8 bytes each; the transpose read
        // hands lane s row s with 4 consecutive k; two reads give 8 k
        const int k = gi * 8 + (s >> 2);
        const int c = R == 64 ? (row0 / 8 + q * 2 + ((s & 3) >> 1)) ^ ((s >> 2) & 2) ^ ((gi & 1) << 2)
                              : (row0 / 8 + q * 2 + ((s & 3) >> 1)) ^ ((s >> 2) << 2) ^ ((gi & 1) << 1);
        addr[q] = k * (R * 2) + c * 16 + (s & 1) * 8;
      } else {
        addr[q] = (row0 + s) * (BK * 2) + ((q * 4 + gi) ^ (s >> 1)) * 16;
      }
    }
  }
  __device__ inline bf16x8 read(const unsigned char* smem, int q, int ks, uint32_t base) const {
    if (TR) {
      const unsigned char* p = smem + addr[q] + base + ks * (32 * R * 2);
      s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)p);
      s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p + 4 * R * 2));
      union { struct { s16x4 a, b; } s; bf16x8 v; } u;
      u.s.a = lo; u.s.b = hi;
      return u.v;
    }
    return *reinterpret_cast<const bf16x8*>(smem + addr[ks] + base + q * (16 * BK * 2));
  }
};

}  // namespace
}  // namespace bm
