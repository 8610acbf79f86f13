// The slots of the 8-bit state cache as the kernels see them.
#pragma once
#include "block.cuh"

namespace ssdi8 {

constexpr int kWin = SSDI8_CACHE_WINDOW;

struct CacheView {
  int nslots;
  int8_t* codes;    // [nslots][H][P][N]
  float* scales;    // [nslots][H][P]
  int8_t* xwin;     // [nslots][H][kWin][P]
  int8_t* Bwin;     // [nslots][G][kWin][N]
  float* dtwin;     // [nslots][H][kWin]
  int32_t* start;   // [nslots]
};
inline CacheView view_of(const ssdi8_cache_t& c) { return {c.nslots, c.codes, c.scales, c.xwin, c.Bwin, c.dtwin, c.start}; }

// Waiting tokens of one head, by the 16 lanes of a half-warp (lane j: row j of the window; the warp's other half repeats them):
// dt is the row's time step, 0 where none waits; `order` counts the rows from the first waiting token's.  The time behind a token
// up to the last one, and all of it.
struct Waiting {
  double behind, all;
};
__device__ __forceinline__ Waiting waiting_of(float dt, int order) {
  // inclusive sum over the tokens in their order: the scan runs over rotated lanes
  const int lane = threadIdx.x & 31;
  Waiting w;
  double sum = (double)dt;
#pragma unroll
  for (int o = 1; o < kWin; o <<= 1) {
    const double other = __shfl_sync(0xffffffffu, sum, (lane & 16) | ((lane - o) & 15));
    if (order >= o) sum += other;
  }
  const int last = (lane & 16) | ((lane - order + 15) & 15);   // the lane whose order is 15
  w.all = __shfl_sync(0xffffffffu, sum, last);
  w.behind = w.all - sum;
  return w;
}

}  // namespace ssdi8
