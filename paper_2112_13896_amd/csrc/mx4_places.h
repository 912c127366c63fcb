// Where the operands of mx4_many lie in LDS: what a lane writes and what a lane
// reads, in bytes.  Plain arithmetic, compiled for the host too (a test checks on
// the CPU that every chunk is read where it was written, and that the lanes that
// are served together meet all banks).
//
// 64 keys a step: their codes as in the cache, [64][DT / 2] bytes, and values in
// bf16, transposed, [DT][64].  Rows are cut into chunks of 16 bytes, and a
// chunk's place in its row is turned (xor) by the row's number.  Of the 32 lanes
// that read a column of chunks, a row each, lanes 0-3, 12-15 and 20-27 are served
// together, and the others.
#pragma once

#include "q8_places.h"

namespace cs {

template <int DT>
struct Mx4Places {
  static constexpr int KC = DT / 32;                       // chunks of a key: 32 channels each
  static constexpr int key_bytes = 64 * DT / 2, value_bytes = DT * 128;
  // a key's scale bytes, four groups to a dword: [words][64] dwords
  static constexpr int words = DT == 256 ? 2 : 1;

  static constexpr int key_turn(int key) {
    return DT == 64 ? key >> 3 & 1 : DT == 128 ? key >> 2 & 3 : chunk_turn(key);
  }
  // Keys: piece of 16 bytes t of the step's 64 * KC, in the cache's order.
  static constexpr int piece_key(int t) { return t / KC; }
  static constexpr int piece_put(int t) {
    return t / KC * (DT / 2) + (t % KC ^ key_turn(t / KC)) * 16;
  }
  // Lane 32 h + r, channels 64 k + 32 h .. of key 32 u + r.
  static constexpr int key_column(int r, int h, int k) {
    return r * (DT / 2) + ((2 * k + h) ^ key_turn(r)) * 16;
  }
  static constexpr int key_at(int column, int u) { return column + 32 * u * (DT / 2); }

  // Values: unit t of DT has eight channels of a chunk's eight keys.
  static constexpr int value_turn(int ch) { return (ch ^ ch >> 3) & 7; }
  static constexpr int unit_channels(int t) { return t % (DT / 8); }   // which eight
  static constexpr int unit_chunk(int t) { return t / (DT / 8); }
  // where the unit's channel c (of eight) goes: the turn of its row is that of the first, xor c
  static constexpr int unit_row(int t) { return unit_channels(t) * 8 * 128; }
  static constexpr int unit_bits(int t) {
    return 16 * (unit_chunk(t) ^ value_turn(unit_channels(t) * 8));
  }
  static constexpr int value_put(int row, int bits, int c) {
    return row + c * 128 + (bits ^ 16 * c);
  }
  // key of the step's 64 whose value a chunk's half `i` (of 8) is
  static constexpr int value_key(int chunk, int i) {
    return chunk / 2 * 16 + chunk % 2 * 4 + i / 4 * 8 + i % 4;
  }
  // Lane 32 h + r, channel 32 ct + r at the keys of weights 8 v .. +7: rows 32 ct .. are turned
  // by 4 more where ct is odd, which makes the column of v that of v xor 2.
  static constexpr int value_column(int r, int h, int v) {
    return r * 128 + ((2 * v + h) ^ value_turn(r)) * 16;
  }
  static constexpr int column_of(int v, int ct) { return ct % 2 ? v ^ 2 : v; }
  static constexpr int value_at(int column, int ct) { return column + ct * 32 * 128; }
  // key of a lane's logit i of 32
  static constexpr int logit_key(int h, int i) { return 8 * (i / 4) + 4 * h + i % 4; }
};

}  // namespace cs
