// Where the kernels of the 4-bit cache (mra_layer.h) put and find things, as plain functions: of a page of one head, of the
// lanes that write, read and convert it, and of the values' transposition in LDS. All are constexpr, so they serve
// device code and, with no other header, a test on the host.
#pragma once

namespace mra {

// Offsets in bytes within a page of one head, of `size` tokens; x = 0: keys, 1: values.
template <int D>
struct Fp4Page {
  static constexpr int NB = D / 32;                // blocks, and step bytes, of a token
  static constexpr int codes(int x, int size) { return x * size * (D / 2); }
  static constexpr int steps(int x, int size) { return size * (D + x * NB); }
};

// Writing and reading back: a workgroup takes kFp4RowTokens neighbouring tokens (aligned) of one head.
constexpr int kFp4RowTokens = 64;

// Tiles that n neighbouring tokens can touch.
constexpr int fp4_row_tiles(int n) { return (n + kFp4RowTokens - 2) / kFp4RowTokens + 1; }

// Unit `unit` of a tile whose lanes take C channels each: keys or values, token of the tile, and chunk of C channels.
template <int D, int C>
struct Fp4RowUnit {
  static constexpr int CPR = D / C, kUnits = 2 * kFp4RowTokens * CPR;
  int value, r, c;
  constexpr explicit Fp4RowUnit(int unit)
      : value(unit / (kFp4RowTokens * CPR)), r(unit / CPR % kFp4RowTokens), c(unit % CPR) {}
  // of its codes (C / 2 bytes) and its block's step in a page, for a token at place `slot`
  constexpr int codes_at(int slot, int size) const { return Fp4Page<D>::codes(value, size) + slot * (D / 2) + c * (C / 2); }
  constexpr int step_at(int slot, int size) const {
    return Fp4Page<D>::steps(value, size) + slot * Fp4Page<D>::NB + c / (32 / C);
  }
};

// Attention, many rows: unit n of thread tid of T converts 16 bytes of codes, a block, of a stage's 64 tokens; with fewer
// threads than blocks a thread has keys and values. 16 lanes' stores of a chunk reach every bank of LDS once: neighbouring tokens are
// four units apart (in their order: 4-way conflicts).
template <int D, int T>
struct Fp4StageUnit {
  static constexpr int U = 2 * D, N = 2 * U > T ? 2 : 1;
  static_assert(N == 1 || U == T, "a lane has one unit of either, or of one of them");
  int x, r, blk;                                   // keys or values (2: no unit), token, block
  constexpr Fp4StageUnit(int n, int tid)
      : x(N == 2 ? n : tid / U),
        r((tid % U / Fp4Page<D>::NB & 48) | (tid % U / Fp4Page<D>::NB & 3) << 2 | (tid % U / Fp4Page<D>::NB >> 2 & 3)),
        blk(tid % U % Fp4Page<D>::NB) {}
};

// Attention, few rows: the token, of a tile's 32, that lane (lane / 16, i = lane % 16) has as its part x = 0, 1 of
// the keys (register r of the scores of x is key 8 (lane / 16) + 4 x + r) or of the values.
constexpr int fp4_tile_row(int value, int x, int i) { return value ? 16 * x + i : 8 * (i >> 2) + 4 * x + (i & 3); }

// A wave's 32 values of D channels in LDS, rows of bfloat16: the byte of channel c (a multiple of 4) of row r. A row's blocks
// of 16 channels, and the halves of a block, are exchanged by row so that neither the stores of 8 rows at a time nor the
// transposing reads of 4 or 8 meet in a bank (none counted at d = 128; at d = 64 32 cycles a tile are, of 96, whatever of the rows'
// bits decides, and cost no time).
template <int D>
constexpr int fp4_value_place(int r, int c) {
  return r * 2 * D +
         (((c >> 4) ^ (D == 128 ? (r & 3) | (r >> 3 & 1) << 2 : D == 64 ? (r >> 1 & 1) | (r >> 3 & 1) << 1 : r >> 3 & 1)) << 5) +
         (((c >> 3 & 1) ^ (r >> 2 & 1)) << 4) + (c & 4) * 2;
}

}  // namespace mra
