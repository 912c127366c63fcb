// Prints the places of mx4_places.h as tables: DT, name, arguments, byte.
#include <cstdio>

#include "mx4_places.h"

template <int DT>
void print() {
  using P = cs::Mx4Places<DT>;
  for (int t = 0; t < 64 * P::KC; ++t)
    std::printf("%d piece %d %d %d\n", DT, t, P::piece_key(t), P::piece_put(t));
  for (int r = 0; r < 32; ++r)
    for (int h = 0; h < 2; ++h) {
      for (int u = 0; u < 2; ++u)
        for (int k = 0; k < DT / 64; ++k)
          std::printf("%d key %d %d %d %d %d\n", DT, r, h, u, k,
                      P::key_at(P::key_column(r, h, k), u));
      for (int v = 0; v < 4; ++v)
        for (int ct = 0; ct < DT / 32; ++ct)
          std::printf("%d value_at %d %d %d %d %d\n", DT, r, h, v, ct,
                      P::value_at(P::value_column(r, h, P::column_of(v, ct)), ct));
    }
  for (int t = 0; t < DT; ++t)
    for (int c = 0; c < 8; ++c)
      std::printf("%d value_put %d %d %d %d %d\n", DT, t, c, P::unit_channels(t) * 8 + c,
                  P::unit_chunk(t), P::value_put(P::unit_row(t), P::unit_bits(t), c));
  for (int g = 0; g < 8; ++g)
    for (int i = 0; i < 8; ++i) std::printf("%d value_key %d %d %d\n", DT, g, i, P::value_key(g, i));
  for (int h = 0; h < 2; ++h)
    for (int i = 0; i < 32; ++i)
      std::printf("%d logit %d %d %d\n", DT, h, i, P::logit_key(h, i));
}

int main() {
  print<64>();
  print<128>();
  print<256>();
  return 0;
}
