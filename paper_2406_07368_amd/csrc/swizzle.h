// Rows of D bf16 in LDS without padding, read without bank conflicts both by rows (16 bytes a lane, 32 rows) and by the
// transpose reads (4 rows of 64 bytes a half wave).
//
// LDS has 64 banks of 4 bytes; a 16-byte read is served 16 lanes at a time, whose rows are distinct modulo 16, an 8-byte
// read 32 lanes at a time.  A row's 16-byte piece c lies at place c ^ f(row): f takes all values over the 16 rows (for
// D = 64, where a row is half as long as the banks are wide, over the 8 rows of a parity), and the bits of f that choose
// 64 bytes differ over 4 consecutive rows.
#pragma once
#include "mfma_util.h"

namespace linattn {

template <int D>
struct Swizzled {
  static_assert(D == 64 || D == 128, "");
  __device__ __forceinline__ static int f(int row) { return D == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : ((row & 2) << 1) | ((row >> 2) & 3); }
  // element offset of piece c of a row
  __device__ __forceinline__ static int piece(int row, int c) { return row * D + ((c ^ f(row)) << 3); }

  int row, tr;   // this lane's: of row operands, of transposed operands
  // order: how a transposed operand's registers count the rows -- 4 as an accumulator does (see tr_operand_acc_order), 8 in
  // sequence.  crossed: its lanes 4..7 and 8..11 of every 16 change places.  An accumulator whose rows are such lanes holds
  // rows 8 (lane / 32) + 0..7 of every 16 in registers 0..7 and 8..15: packed, it goes with a row operand as rows() reads it.
  __device__ __forceinline__ Swizzled(int lane, int order, bool crossed = false) {
    const int l32 = lane & 31, hi = lane >> 5, j = lane & 15;
    row = piece(l32, hi);
    const int r = order * hi + (j >> 2), c4 = crossed ? ((j & 1) << 1) | ((j >> 1) & 1) : j & 3;
    tr = piece(r, 2 * ((lane >> 4) & 1) + (c4 >> 1)) + 4 * (c4 & 1);
  }
  // From here on the compiler does not know the offsets: it makes the addresses that hang on them anew where they are used
  // instead of keeping them in registers over a loop.
  __device__ __forceinline__ void forget_rows() { asm volatile("" : "+v"(row)); }
  __device__ __forceinline__ void forget_cols() { asm volatile("" : "+v"(tr)); }
  // lanes <-> rows row0 + 0..31 (a multiple of 32), registers <-> elements 16 ks + 8 (lane / 32) + 0..7
  __device__ __forceinline__ bf16x8 rows(const uint16_t* base, int row0, int ks) const { return lds_row8(base + row0 * D + (row ^ (ks << 4))); }
  // lanes <-> elements 32 ct + lane % 32, registers <-> rows row0 + 0..15 (a multiple of 16) in an accumulator's order ...
  __device__ __forceinline__ bf16x8 cols_acc(const uint16_t* base, int row0, int ct) const {
    const uint16_t* p = base + row0 * D;
    const int o = tr ^ (ct << 5);
    return cat4(lds_tr4(p + o), lds_tr4(p + 8 * D + (o ^ 16)));
  }
  // ... and in sequence
  __device__ __forceinline__ bf16x8 cols(const uint16_t* base, int row0, int ct) const {
    const uint16_t* p = base + row0 * D;
    const int o = tr ^ (ct << 5);
    return cat4(lds_tr4(p + o), lds_tr4(p + 4 * D + (o ^ 8)));
  }
};

// For a run of N products whose operands (R LDS reads for every M of them) the compiler would fetch one by one, each product
// waiting for its own: A reads first, then M products and R reads in turn.
template <int A, int R, int M, int N>
__device__ __forceinline__ void read_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, A, 0);      // LDS reads
  constexpr int turns = (N / M * R - A + R - 1) / R;
#pragma unroll
  for (int i = 0; i < turns; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, M, 0);    // MFMA
    __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, N - turns * M, 0);
}

// ROWS rows of D bf16 from memory straight into LDS, NT threads: a wave's request fills 1 KB in the order of its lanes, so a
// lane asks for the piece that belongs at its place.  `rows` of them are there: the others re-read row 0 and are overwritten
// with zeros (by the thread that asked for them) once they are in.
// The caller waits: arrived(), then a barrier.  Between a request and that the compiler must know that what the code reads by
// transposed operands and what it writes is not what is under way, or it waits there and then: the buffers are __restrict
// parameters of whatever holds both.
template <int D, int ROWS = 64, int NT = 256>
struct Fetch {
  static constexpr int PPR = D / 8, NP = ROWS * PPR / NT, RP = NT / PPR;   // (RP rows on: the same permutation)
  typedef const __attribute__((address_space(1))) void* global_ptr;
  typedef __attribute__((address_space(3))) void* lds_ptr;
  uint32_t row, piece;
  int wave;
  __device__ __forceinline__ explicit Fetch(int tid)
      : row(tid / PPR), piece(((tid % PPR) ^ Swizzled<D>::f(tid / PPR)) * 8), wave(__builtin_amdgcn_readfirstlane(tid >> 6)) {}
  // BACKWARDS: the first of them is the last in memory; row0 is the first in memory either way
  template <bool BACKWARDS = false>
  __device__ __forceinline__ void request(uint16_t* lds, const uint16_t* row0, int64_t stride, int rows) const {
    const uint32_t st = (uint32_t)stride;                 // (at most 2^22: a tile's offsets fit 32 bits)
    const char* base = reinterpret_cast<const char*>(row0);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      uint32_t r = row + RP * i;
      if (BACKWARDS) r = (uint32_t)(rows < ROWS ? rows : ROWS) - 1 - r;   // (wraps where there is no such row)
      if (rows < ROWS) r = r < (uint32_t)rows ? r : 0;
      __builtin_amdgcn_global_load_lds((global_ptr)(base + (r * st + piece) * 2), (lds_ptr)(lds + (i * NT + wave * 64) * 8), 16, 0, 0);
    }
  }
  // behind arrived()
  __device__ __forceinline__ void trim(uint16_t* lds, int rows, int tid) const {
    if (rows < ROWS) {
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if ((int)row + RP * i >= rows) *reinterpret_cast<u32x4*>(lds + (i * NT + tid) * 8) = u32x4{0u, 0u, 0u, 0u};
    }
  }
  // this wave's requests are in LDS (a barrier makes them everybody's)
  static __device__ __forceinline__ void arrived() { __builtin_amdgcn_s_waitcnt(0x0f70); }
};

}  // namespace linattn
