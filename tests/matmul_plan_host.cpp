// The kernel and the splits that a product takes: for the shapes whose times stand beside the rule, and over many sizes what the launch
// relies on.
#include "../paper_2512_17073_amd/csrc/matmul_plan.h"

#include <cstdio>

using namespace lrc;

int main() {
  const struct { int M, K, N; MmKind kind; int splits; } quoted[] = {
      {1, 14336, 4096, kNarrow1, 1}, {1, 4096, 28672, kNarrow1, 1},   {64, 4096, 4096, kSmall2, 1},  {64, 4096, 28672, kWide4, 1},
      {64, 14336, 4096, kSmall4, 2}, {333, 1408, 2048, kWide4, 1},    {512, 4096, 28672, kLarge, 1}, {2048, 2048, 2816, kTile, 1},
      {2048, 4096, 28672, kLarge, 1}, {100, 14336, 2816, kSmall2, 1}};
  int wrong = 0;
  for (const auto& q : quoted) {
    const MmPlan p = mm_plan(q.M, q.K, q.N);
    if (p.kind != q.kind || p.splits != q.splits) {
      ++wrong;
      std::printf("%d x %d x %d: kernel %d in %d splits, not %d in %d\n", q.M, q.K, q.N, p.kind, p.splits, q.kind, q.splits);
    }
  }
  for (int M = 1; M <= 1 << 22; M += M / 3 + 1)
    for (int K = 16; K <= 1 << 20; K += K / 3 / 16 * 16 + 16)
      for (int N = 1; N <= 1 << 22; N += N / 2 + 1) {
        const MmPlan p = mm_plan(M, K, N);
        const int kb = (K + 127) / 128;
        // (every split has a block of its own; a sum in parts stays within a workspace of a few launches' outputs)
        const bool fine = p.splits >= 1 && p.splits <= 16 && (p.splits == 1 || (kb >= 4 * p.splits && p.kind != kLarge));
        if (!fine) {
          ++wrong;
          std::printf("%d x %d x %d: kernel %d in %d splits\n", M, K, N, p.kind, p.splits);
        }
      }
  return wrong != 0;
}
