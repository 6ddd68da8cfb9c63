// The token norm that bounds the scored routing's first products is at least the norm, whatever the sums of squares lose:
// summed up in fp32 in shares as the kernel has them, every sum cut instead of rounded, numbers below 2^-126 lost.
#include "../paper_2512_17073_amd/csrc/route_bounds.h"

#include <cstdint>
#include <cstdio>
#include <cstring>
#include <random>

namespace {
float cut(double v) {                                      // to fp32 towards zero, none below 2^-126
  if (v < 0x1p-126) return 0.f;
  float f = float(v);
  if (double(f) > v) {
    uint32_t u;
    std::memcpy(&u, &f, 4);
    --u;
    std::memcpy(&f, &u, 4);
  }
  return f;
}
float bf16(float v) {
  uint32_t u;
  std::memcpy(&u, &v, 4);
  u &= 0xffff0000u;
  std::memcpy(&v, &u, 4);
  return v;
}
}  // namespace

int main() {
  std::mt19937 gen(1);
  std::uniform_real_distribution<float> one(1.f, 2.f), unit(0.f, 1.f);
  int checked = 0, wrong = 0;
  for (int H : {64, 320, 2048, 7168, lrc::kNormValues})
    for (int e = -75; e <= 40; ++e)
      for (int kind = 0; kind < 3; ++kind) {               // equal values, values within a factor of two, a few among many far smaller ones
        const float base = kind == 0 ? 1.9921875f : 1.f;
        double exact = 0.0;
        float share[16] = {};
        for (int i = 0; i < H; i += 2) {
          double pair = 0.0;
          for (int j = 0; j < 2; ++j) {
            const float v = bf16(ldexpf(kind == 0 ? base : one(gen), e - (kind == 2 && unit(gen) > 0.01f ? 12 : 0)));
            exact += double(v) * v;
            pair += cut(double(v) * v);
          }
          share[(i / 2) % 16] = cut(share[(i / 2) % 16] + cut(pair));
        }
        float sum = 0.f;
        for (float s : share) sum = cut(double(sum) + s);
        ++checked;
        if (double(lrc::norm_above(sum)) < std::sqrt(exact)) {
          ++wrong;
          if (wrong < 5) std::printf("H %d, 2^%d, kind %d: %a below %a\n", H, e, kind, lrc::norm_above(sum), std::sqrt(exact));
        }
      }
  std::printf("%d of %d bounds too low\n", wrong, checked);
  return wrong != 0;
}
