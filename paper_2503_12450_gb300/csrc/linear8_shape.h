// Host only: how lazymar_block8_linear above the few-row kernel cuts a product
// into tiles, and which rows its epilogue takes by whole accesses (k_linear8.cu).
#pragma once

#include <cstdint>

namespace lm {
namespace l8 {

constexpr int kSplitCtas = 128;  // most CTAs of a launch that splits K

// Tiles of 256 x 256 on pairs, of 128 x 128 on single CTAs, or of the latter with K
// in parts, by the time that was measured (us): a pair's round 2.5 and 0.45 for each
// 128 of K, a single CTA's 1 and 0.33 up to 12 of them, 0.65 after that (its ring then
// waits for memory), a launch 4 and 5; parts cost 1 and 0.2 for each row a warp.
// (Measured, pairs : single, N 4096, K 1024: M = 300 11.0 : 9.9, 1000 12.2 : 14.0, 2000 18.7 :
// 21.5; N = K = 1280: 300 10.3 : 8.9 and 7.9 in four parts, 2000 11.0 : 13.0; N 1024, K 4096, M
// = 300: 20.9 in one part, 10.6 in four.)
struct Shape {
  bool pair;
  int parts;
  long long tiles;
};
inline Shape choose(int sms, int M, int N, int K) {
  const long long pair_tiles = (long long)((M + 255) / 256) * ((N + 255) / 256);
  const long long tiles = (long long)((M + 127) / 128) * ((N + 127) / 128);
  const int kb = (K + 127) / 128;
  const auto rounds = [](long long t, int slots) { return (double)((t + slots - 1) / slots); };
  const auto single = [](double k) { return k <= 12 ? 0.33 * k : 4.0 + 0.65 * (k - 12); };
  Shape best{true, 1, pair_tiles};
  double least = 4.0 + rounds(pair_tiles, sms / 2) * (2.5 + 0.45 * kb);
  const double one = 5.0 + rounds(tiles, sms) * (1.0 + single(kb));
  if (one < least) {
    least = one;
    best = Shape{false, 1, tiles};
  }
  // parts of two blocks at least, one tile a cluster, and every cluster finds its
  // SMs at once (a GPC holds two clusters of eight)
  const int most = sms < kSplitCtas ? sms : kSplitCtas;
  for (int parts = 2; parts <= 8 && tiles * parts <= most && kb >= 2 * parts; parts *= 2) {
    const double us = 5.0 + 2.0 + 0.2 * (16 / parts) + single((double)kb / parts);
    if (us < least) {
      least = us;
      best = Shape{false, parts, tiles};
    }
  }
  return best;
}

// Rows on boundaries of four elements (those of an absent tensor are, whatever its
// stride says).
inline bool rows_on_four(const void* p, int ld, int elem_bytes) {
  return !p || (ld % 4 == 0 && reinterpret_cast<uintptr_t>(p) % (4u * (unsigned)elem_bytes) == 0);
}

}  // namespace l8
}  // namespace lm
