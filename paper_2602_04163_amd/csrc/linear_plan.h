// Which kernel of the product on stored planes (linear.h) a call takes.
#pragma once
#include <initializer_list>

namespace bpdq {

constexpr int kLinRowsMost = 32;                           // tokens of the kernel without an ordering of X

// The kernel of a call: the one whose estimate is the least.  A work-group takes a CU, so the time is the rounds of 256 of them times a
// work-group's, which was measured alone on the chip (two planes, us):
//   few tokens (R row tiles, 16 or 32 tokens), per 3584 columns: 5.4 + 1.6 R, 8 + 2.2 R, and half of that at the least: with 512 columns a round
//   of R = 5 and 32 tokens takes 9.5, not the 2.7 of its share.  (Of eight shapes up to 800 columns whose kernel this changes seven take
//   0.26 to 0.94 of the time, 257 x 160 -> 20480 88 us and now 23; 1484 x 800 -> 587 takes 25 in place of 23.)
//   tiles, per 64 columns: 256 x 256 1.25, 256 x 128 0.9, 128 x 128 in two parts 1.15 / 2, 128 x 64 in four 1.85 / 4; 8 for the order of X
//   (256 x 256 counts 1.45: two of the others share a CU and their rounds run into one another.  Fp16, two planes in groups of 128, with it and with
//   256 x 128, which its estimate then takes: 512 x 3584 -> 37888 194 us and 160, 1024 x 3584 -> 18944 195 and 162, 700 x 8192 -> 29568 402 and 368, 3000 x 8192 -> 8192 427
//   and 417; at three planes in groups of 32 1024 x 3584 -> 18944 291 and 280, at four in groups of 128 230 and 240.  2048 x 3584 -> 37888 keeps
//   it: 530 and 554.)
// (One, three and four planes are taken like two.)
// 64 x 8192 -> 8192: R = 5, 2 x 16 tokens 43 us, tiles of 128 x 64 48, of 256 x 256 160; 2048 x 8192 -> 8192: 256 x 256 263, 128 x 64 432;
// 333 x 3584 -> 18944: 256 x 128 62, 128 x 128 72, 256 x 256 86.
enum LinearKernel { kRows1, kRows2, kTile256, kTile256x128, kTile128, kTile128x64 };
struct LinearPlan {
  int kernel, r;
};
static inline LinearPlan linear_plan(int n_tok, int d_in, int d_out) {
  LinearPlan best = {kRows1, 1};
  float least = 0.f;
  auto offer = [&](int kernel, int r, int rows, int toks, float each, float once) {
    const long groups = ((long)d_out + rows - 1) / rows * (((long)n_tok + toks - 1) / toks);
    const float t = (float)((groups + 255) / 256) * each + once;
    if (least == 0.f || t < least) {
      least = t;
      best = {kernel, r};
    }
  };
  const float wide = d_in > 1792 ? d_in / 3584.f : 0.5f;
  for (int r : {1, 2, 3, 5, 8}) {
    offer(kRows1, r, 16 * r, 16, (5.4f + 1.6f * r) * wide, 0.f);
    if (n_tok > 16 && r > 1 && r < 8) offer(kRows2, r, 16 * r, 32, (8.f + 2.2f * r) * wide, 0.f);
  }
  // offsets inside a row tile's planes, inside a token tile of the ordered X and so on are 32 bits in the tile kernels
  if (n_tok > kLinRowsMost && d_in <= 1 << 20) {
    const float stages = 4.f * ((d_in + 255) / 256);
    offer(kTile256, 0, 256, 256, 1.45f * stages, 8.f);
    offer(kTile256x128, 0, 256, 128, 0.9f * stages, 8.f);
    offer(kTile128, 0, 128, 128, 1.15f / 2 * stages, 8.f);
    offer(kTile128x64, 0, 128, 64, 1.85f / 4 * stages, 8.f);
  }
  return best;
}

}  // namespace bpdq
