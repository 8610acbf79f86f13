// Which form a product in four bits takes: host arithmetic on its sizes alone, without CUDA.
#pragma once
#include <cstdint>

namespace ssdi8 {

// Few rows (fp4_few_kernel): shared memory of a CTA
struct Fp4Few {
  static constexpr int kMaxStages = 10;
  static constexpr uint32_t kRow = 128, kW = 128 * kRow;   // bytes of a stage's row (256 columns) and of its rows of w
  // the ring, two CTAs on an SM or one; the accumulator's image of [n][128] goes over it
  static constexpr uint32_t kSmall = 101376, kLarge = 221184;
  // 128 rows' scales of a stage, and the stage: n rows of x and 128 of w
  static constexpr uint32_t scales(int block) { return 256u / (uint32_t)block / 4u * 512u; }
  static constexpr uint32_t stage(int n, int block) { return (kW + (uint32_t)n * kRow + (n <= 128 ? 2u : 3u) * scales(block) + 1023u) & ~1023u; }
};

struct Fp4Form {
  bool pair;            // tiles of 256 x 256 on pairs of SMs; else few rows:
  int n, split;         // tokens of a tile (to 16), CTAs that share K
  uint32_t ring;        // bytes of the ring
  int stages;
};

// What is done sooner, in cycles (the figures are measured ones).  Few rows: 5000 for the call, and for each wave 2200 to the first operands, 46 bytes of
// operands a cycle and SM, or where the ring does not hold all of a CTA's stages their latency of 1400 over those that it holds; the
// accumulator's way out, the parts' meeting, the tokens.  A wave behind another takes 12000 at least.
// Pairs: 10000 for the call, the first operands and the last tile's way out, 600 for 256 of K where no epilogue is beside them and 760 where one is, 1700
// from one tile to the next, 5000 at least.  (us, few rows and pairs: 64 x 10576 x 2560 6.9, 9.9; 64 x 10576 x 768 4.7, 6.3; 250 x 2000 x 1024 9.0, 6.0;
// 256 x 4096 x 8192 12.8, 15.7; 512 x 2560 x 5120 12.5, 10.7; 700 x 5000 x 256 7.0, 5.9; 3439 x 16472 x 512 77, 35.)
// vec_out: out's rows lie on 16 bytes.
inline Fp4Form fp4_form(int rows, int outs, int width, int block, bool vec_out, int sms) {
  const int kblocks = (width + 255) / 256;
  const int64_t mt = (outs + 127ll) / 128;
  Fp4Form f = {};
  double best = 0.0;
  for (int n = rows <= 256 ? (rows + 15) / 16 * 16 : 128; n <= 256; n += rows <= 256 ? 256 : 128) {
    const int64_t tiles = mt * ((rows + n - 1ll) / n);
    const uint32_t bytes = Fp4Few::stage(n, block);
    for (int per_sm = n <= 128 ? 2 : 1; per_sm >= 1; --per_sm) {
      const int ring = (int)(per_sm == 2 ? Fp4Few::kSmall : Fp4Few::kLarge), stages = ring / (int)bytes < Fp4Few::kMaxStages ? ring / (int)bytes : Fp4Few::kMaxStages;
      // (clusters of four take 7 of 8 SMs at best, 16 of a GPC's 18; of eight fewer: 64 x 2560 x 5120 8 us with four, 19 to 22 with eight)
      for (int split = 1; split <= 4 && split <= kblocks; split *= 2) {
        const int64_t places = (int64_t)(split == 4 ? sms - sms / 8 : sms) * per_sm;
        const double ctas = (double)tiles * split, waves = (double)((tiles * split + places - 1) / places), share = ctas <= sms ? 1.0 : (double)per_sm;
        const int kb = (kblocks + split - 1) / split;
        const double port = kb * (double)bytes * share / 46.0, latency = kb > stages ? (kb - stages) * 1400.0 / stages : 0.0;
        const double wave = 2200.0 + (port > latency ? port : latency) + n * 8.0 + n / split * 20.0 + (split > 1 ? 1300.0 + n * 25.0 : 0.0);
        const double cycles = 5000.0 + (waves == 1.0 ? wave : waves * (wave > 12000.0 ? wave : 12000.0));
        if (best == 0.0 || cycles < best) {
          best = cycles;
          f.n = n;
          f.split = split;
          f.ring = (uint32_t)ring;
          f.stages = stages;
        }
      }
    }
  }
  const int64_t ptiles = (int64_t)((rows + 255ll) / 256) * ((outs + 255ll) / 256), pairs = sms / 2;
  const double each = 760.0 * kblocks + 1700.0;
  // (where rows lie on no 16-byte boundary the last columns go out by elements: 134 x 115 x 256 10.6, few rows 6.8)
  const double ragged = !vec_out && outs % 64 ? 6000.0 : 0.0;
  f.pair = pairs > 0 && 10000.0 + ragged + 600.0 * kblocks + (double)((ptiles + pairs - 1) / pairs - 1) * (each > 5000.0 ? each : 5000.0) < best;
  return f;
}

}  // namespace ssdi8
