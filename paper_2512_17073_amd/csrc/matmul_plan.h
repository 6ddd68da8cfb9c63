// Which kernel a product of matmul_fp8.hip takes, and in how many splits of the sum.
#pragma once
#include <algorithm>
#include <cmath>

namespace lrc {

enum MmKind { kNarrow1, kNarrow2, kNarrow4, kSmall2, kSmall4, kWide4, kTile, kLarge };
struct MmPlan { MmKind kind; int splits; };
constexpr int kMmTileM[] = {16, 32, 64, 32, 64, 64, 128, 256}, kMmTileN[] = {16, 16, 16, 32, 32, 64, 128, 256};
// By an estimate of the time in us, fitted to the times of all kernels and splits on 695 shapes (M 1 to 4096, K 512 to 14336, N 512 to 28672, weights
// from memory).  A small tile:
// 1.8 us for each workgroup of a CU, one after the other, and 11 to 22 ns for each KB of operands, all of them together at 16 TB/s from the
// L2s and the weights at 5.5 TB/s from memory.  A 128 x 128 tile 0.65 to 0.8 us, a 256 x 256 tile 1.4 to 1.8 us for a block of the sum.
// Splits are joined by a second launch.
// Measured anew on 668 shapes (M 1 to 2048), the chosen one takes 2.4% longer than the fastest of these kernels on average, 50% at worst (100 x 14336 x
// 2816, 32.5 / 21.6).  That compares them with one another only: of the shapes whose floor is 8 us or more the median is 1.3 times the floor for M
// up to 8, 1.5 to 1.7 for 16 to 64, 1.9 to 2.6 (at most 3.7) for 100 to 512, 1.75 for 1024 and 2048.
// Without one of them the fastest of the others takes longer on average by 2.0% (16 x 16), 0.9 (32 x 16), 0.2 (64 x 16), 0.5 (32 x 32), 1.6 (64 x 32),
// 0.9 (64 x 64), 7.1 (128 x 128), 0.9 (256 x 256), and by 4 to 34% where it is the fastest itself (tokens x columns).
// Chosen / next best, us: 1 x 14336 x 4096 13.3 (16 x 16) / 15.0 (32 x 32, two splits); 1 x 4096 x 28672 23.6 (16 x 16) / 25.7 (32 x 32); 64 x 4096
// x 4096 8.9 (32 x 32) / 8.8 (64 x 16); 64 x 4096 x 28672 31.4 (64 x 64) / 31.6 (128 x 128, two splits); 333 x 1408 x 2048 8.5 (64 x 64) / 8.3
// (64 x 32); 512 x 4096 x 28672 58.6 (256 x 256) / 74.5 (128 x 128); 2048 x 2048 x 2816 20.4 (128 x 128) / 28.6 (64 x 64).
inline MmPlan mm_plan(int M, int K, int N) {
  constexpr float kNsPerKb[] = {11.f, 12.f, 12.f, 13.f, 16.f, 22.f};
  const int kb = (K + 127) / 128;
  const float weights = float(N) * float(K);
  MmPlan best{kLarge, 1};
  float least = 1e30f;
  for (int kind = kNarrow1; kind <= kLarge; ++kind) {
    const float tiles = float((M + kMmTileM[kind] - 1) / kMmTileM[kind]) * float((N + kMmTileN[kind] - 1) / kMmTileN[kind]);
    for (int splits = 1; splits <= (kind == kLarge ? 1 : 16); splits *= 2) {
      if (splits > 1 && (kb < 4 * splits || tiles * (splits / 2) > 512.f)) break;
      const float per_cu = tiles * splits / 256.f, blocks = float((kb + splits - 1) / splits);
      float us;
      if (kind <= kWide4) {
        const float kbytes = float(kMmTileM[kind] + kMmTileN[kind]) / 8.f;
        const float read = (float(M) * std::ceil(float(N) / kMmTileN[kind]) + float(N) * std::ceil(float(M) / kMmTileM[kind])) * float(K);
        us = 3.7f + std::max(1.8f * (std::ceil(per_cu) - 1.f) + std::max(1.f, per_cu) * blocks * kbytes * kNsPerKb[kind] * 1e-3f,
                             std::max(weights / 5.5e6f, read / 16e6f));
      } else if (kind == kTile) {
        us = 4.f + std::max(blocks * std::max(0.8f, 0.65f * per_cu), weights / 5.5e6f);
      } else {
        us = 6.f + std::max(blocks * std::max(1.4f, 1.8f * per_cu), weights / 5.5e6f);
      }
      if (splits > 1) us += 2.f + float(splits + 1) * M * float(N) * 4.f / 2.2e6f;
      if (us < least) { least = us; best = {MmKind(kind), splits}; }
    }
  }
  return best;
}

}  // namespace lrc
