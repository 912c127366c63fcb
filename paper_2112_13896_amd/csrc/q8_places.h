// Where the 8-bit kernels' operands lie in LDS: what a lane writes and what a
// lane reads, in bytes.  Plain arithmetic, compiled for the host too (a test
// checks on the CPU that every chunk is read where it was written).
//
// Rows are cut into chunks of 16 bytes, and a chunk's place in its row is turned
// (xor) by the row's number, so that the lanes that are served together when a
// column of chunks is read meet all banks.
#pragma once

namespace cs {

// LDS rows of 128 bytes, read in columns of 16-byte chunks by 32 lanes, a row
// each: chunk c of a row lies at c ^ chunk_turn(row).  (row and row / 8: lanes
// 0-3, 12-15, 20-27 of 32 are served together, and the others.)
constexpr int chunk_turn(int row) { return (row ^ (row >> 3 & 3)) & 7; }

// linear_q8_tile: rows of 128 codes.  LDS receives a wavefront's loads in lane
// order, so the turn is made in the addresses that it loads from.
struct TilePlaces {
  static constexpr int row(int piece) { return piece >> 3; }         // of a 16-byte piece of LDS
  static constexpr int chunk(int piece) { return (piece ^ chunk_turn(row(piece))) & 7; }
  // codes 32 s + 16 h .. of row r (of 32)
  static constexpr int at(int r, int s, int h) {
    return r * 128 + ((2 * s + h) ^ chunk_turn(r)) * 16;
  }
};

// attention_many: 64 keys a step in halves, keys [64][DT], values transposed
// [DT][64].  Two wavefronts bring the keys, two the values, `half` of the step's
// keys each, in blocks of 16.
template <int DT>
struct ManyPlaces {
  static constexpr int buffer = 64 * DT * 2;               // bytes of keys or values
  static constexpr int KB = DT / 64;                       // keys: loads a block, 16 bytes a lane
  static constexpr int PR = DT / 16;                       // lanes to a key
  static constexpr int VD = DT / 64;                       // dwords a lane and value row
  static constexpr int KA = DT == 64 ? 4 : 8;              // columns of chunks that turn together

  static constexpr int key_turn(int key) { return DT == 64 ? chunk_turn(key) : key & 15; }

  // Keys: a lane's first key of its half and its channels; load p brings those of
  // the key key_step(p) further on.
  static constexpr int key(int lane) { return lane / PR; }
  static constexpr int key_channel(int lane) { return lane % PR * 16; }
  static constexpr int key_step(int p) { return p / KB * 16 + p % KB * (64 / PR); }
  static constexpr int key_row(int half, int lane) { return (32 * half + key(lane)) * DT * 2; }
  static constexpr int key_bits(int half, int lane) {
    return 16 * (key_channel(lane) / 8 ^ key_turn(32 * half + key(lane)));
  }
  // chunk i (of two) of load p's 16 channels
  static constexpr int key_put(int row, int bits, int p, int i) {
    return row + key_step(p) * DT * 2 + (bits ^ 16 * key_turn(key_step(p)) ^ 16 * i);
  }

  // Values: 32 lanes to a block, 16 to each half of its keys (a chunk of LDS), DT / 16 channels.
  static constexpr int value_channel(int lane) { return lane % 16 * 4 * VD; }
  static constexpr int value_chunk(int half, int lane) { return 4 * half + lane / 16; }
  static constexpr int value_row(int lane) { return value_channel(lane) * 128; }
  static constexpr int value_bits(int half, int lane) {
    return 16 * (value_chunk(half, lane) ^ chunk_turn(value_channel(lane)));
  }
  // the lane's channel c (of 4 VD)
  static constexpr int value_put(int row, int bits, int c) {
    return row + c * 128 + (bits ^ 16 * chunk_turn(c));
  }
  // key of the step's 64 whose value a chunk's half `i` (of 8) is
  static constexpr int value_key(int chunk, int i) {
    return chunk / 2 * 16 + chunk % 2 * 4 + i / 4 * 8 + i % 4;
  }

  // Reads, lane = 32 h + r.  Products k = 0 .. DT / 16 - 1 of keys 32 u .. +31:
  // channels 16 k + 8 h ..
  static constexpr int key_column(int r, int h, int k) {                // k < KA
    return r * DT * 2 + ((2 * k + h) ^ key_turn(r)) * 16;
  }
  static constexpr int key_at(int column, int u, int k) {
    return column + 32 * u * DT * 2 + k / KA * 256;
  }
  // values 32 ct .. +31 at the keys of logits 8 v .. +7
  static constexpr int value_column(int r, int h, int v) {
    return r * 128 + ((2 * v + h) ^ chunk_turn(r)) * 16;
  }
  static constexpr int value_at(int column, int ct) { return column + ct * 32 * 128; }
  // key of a lane's logit i of 32
  static constexpr int logit_key(int h, int i) { return 8 * (i / 4) + 4 * h + i % 4; }
};

}  // namespace cs
