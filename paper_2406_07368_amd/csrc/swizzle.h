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
  // `order`: how a transposed operand's registers count the rows -- 4 as an accumulator does (see tr_operand_acc_order), 8 in sequence
  __device__ __forceinline__ Swizzled(int lane, int order) {
    const int l32 = lane & 31, hi = lane >> 5, j = lane & 15;
    row = piece(l32, hi);
    const int r = order * hi + (j >> 2);
    tr = piece(r, 2 * ((lane >> 4) & 1) + ((j & 3) >> 1)) + 4 * (j & 1);
  }
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

}  // namespace linattn
