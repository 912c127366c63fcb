// Prints what the kernels' address functions say, for test_q8_places_cpu.py: lines of a name and
// numbers.
#include <cstdio>

#include "q8_places.h"

using cs::TilePlaces;

template <int DT>
void many() {
  using P = cs::ManyPlaces<DT>;
  std::printf("many %d %d %d\n", DT, P::buffer, P::KA);
  for (int half = 0; half < 2; ++half)
    for (int lane = 0; lane < 64; ++lane) {
      // key_put: byte, key, chunk of eight channels
      for (int p = 0; p < 2 * P::KB; ++p)
        for (int i = 0; i < 2; ++i)
          std::printf("key_put %d %d %d\n",
                      P::key_put(P::key_row(half, lane), P::key_bits(half, lane), p, i),
                      32 * half + P::key(lane) + P::key_step(p), P::key_channel(lane) / 8 + i);
      // value_put: byte, channel, chunk of eight keys
      for (int c = 0; c < 4 * P::VD; ++c)
        std::printf("value_put %d %d %d\n",
                    P::value_put(P::value_row(lane), P::value_bits(half, lane), c),
                    P::value_channel(lane) + c, P::value_chunk(half, lane));
    }
  for (int h = 0; h < 2; ++h)
    for (int r = 0; r < 32; ++r) {
      for (int k = 0; k < DT / 16; ++k)
        for (int u = 0; u < 2; ++u)
          std::printf("key_at %d %d %d\n", P::key_at(P::key_column(r, h, k % P::KA), u, k), 32 * u + r,
                      2 * k + h);
      for (int v = 0; v < 4; ++v)
        for (int ct = 0; ct < DT / 32; ++ct)
          std::printf("value_at %d %d %d\n", P::value_at(P::value_column(r, h, v), ct), 32 * ct + r,
                      2 * v + h);
    }
  for (int chunk = 0; chunk < 8; ++chunk)
    for (int i = 0; i < 8; ++i)
      std::printf("pair %d %d\n", P::value_key(chunk, i), P::logit_key(chunk % 2, chunk / 2 * 8 + i));
}

int main() {
  std::printf("tile\n");
  for (int piece = 0; piece < 256 * 8; ++piece)
    std::printf("piece %d %d %d\n", piece * 16, TilePlaces::row(piece), TilePlaces::chunk(piece));
  for (int first = 0; first < 256; first += 32)
    for (int s = 0; s < 4; ++s)
      for (int h = 0; h < 2; ++h)
        for (int r = 0; r < 32; ++r)
          std::printf("at %d %d %d\n", first * 128 + TilePlaces::at(r, s, h), first + r, 2 * s + h);
  many<64>();
  many<128>();
  many<256>();
}
