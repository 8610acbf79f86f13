// Product of two matrices in four bits: out = act(step_x step_w (x w^T) + bias) + residual, on tcgen05.mma with block scales (e2m1 operands, fp32
// accumulators in tensor memory).  Products of codes and scales are exact, sums are the tensor core's binary32.
//
// Operands come by TMA in rows of 128 bytes (256 columns) with the 128-byte swizzle, scales as they stand in memory: their tiles of
// 128 rows x 4 blocks are what tcgen05.cp spreads over tensor memory (32 lanes of four words, the same for every quarter of the lanes), from where
// the MMA takes them.  Two forms: persistent tiles of 256 x 256 on pairs of SMs, and for few rows a tile of 128 x up to 256 a CTA with K shared out.
//
// What bounds it.  The pipe does 64 columns of a pair's tile in 148 cycles on resident operands and scales (8.2 PFLOP/s at 1965 MHz, with the scales'
// copies between them: N 256 alone hides those, N 128 takes 76 without and 88 with).  16384 x 2560 x 5120 with bias and residual (34 us of
// bytes, 52 of operations at that rate) takes 97 to 108 us on the device: the clock falls to 1.4 to 1.65 GHz under the power limit, at which a tile's 20 stages
// take 13300 cycles where the pipe alone would take 11900 (89 %), and 0.9 us pass from one tile to the next: the accumulators share 48 columns.
// 3439 x 16472 x 1248, fp16, residual (37 us of bytes) 72 to 76, 53 to 57 without the residual: five stages a tile, and operands and results
// share the way between L2 and the SMs (459 MB, 8.7 TB/s; 36 us without the stores, whatever the epilogue does); 16470 columns, rows on words, 98; 16471, odd ones, 146; in
// binary32 (72) 112, 161 and 163.
// 64 x 10576 x 2560 (2.6 us of bytes) 6.9 us from L2 and 8.8 from DRAM, one row 5.9 and 6.8: launch and first operands 1.0, ten stages' MMAs and
// scale copies of a lone CTA 2.5 (issued without checks; 3.5 with them), the accumulator's way out and the tokens 1.5.
#include "fp4.cuh"
#include "fp4_form.h"
#include "kernels.h"
#include "linear.cuh"

namespace ssdi8 {
namespace {

using namespace sm100;

constexpr int BK = 256, ROW = 128;   // columns of a stage, and their bytes

struct Fp4Params {
  const float *s_row, *s_w, *bias;
  const void* residual; i64 res_stride;
  void* out; i64 out_stride;
  int32_t* status;
  int T, O, steps, kblocks, tiles, mtiles, ntiles, act, vec_out, vec_res;   // steps: of 64 columns; tiles: of scales beside one another
};

// Instruction descriptor: e2m1 operands, K-major; scales e4m3 (blocks of 16) or e8m0 (32; bits 4 and 29: the
// word's byte that a step's first scale is in)
__host__ __device__ constexpr uint32_t idesc_fp4(int M, int N, int block) {
  return (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | (block == 32 ? 1u << 23 : 0u) | ((uint32_t)(M >> 4) << 24);
}
template <int CTAS, int BLOCK>
__device__ __forceinline__ void mma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
#define SSDI8_MMA_FP4(WHAT)                                                                                                    \
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\ttcgen05.mma." WHAT " [%0], %1, %2, %3, [%4], [%5], p;\n\t}"     \
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)                                         \
               : "memory")
  if (CTAS == 1 && BLOCK == 16) SSDI8_MMA_FP4("cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X");
  if (CTAS == 1 && BLOCK == 32) SSDI8_MMA_FP4("cta_group::1.kind::mxf4.block_scale.scale_vec::2X");
  if (CTAS == 2 && BLOCK == 16) SSDI8_MMA_FP4("cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X");
  if (CTAS == 2 && BLOCK == 32) SSDI8_MMA_FP4("cta_group::2.kind::mxf4.block_scale.scale_vec::2X");
#undef SSDI8_MMA_FP4
}
// a tile of scales (512 bytes) into four columns, for all quarters of the lanes; both CTAs' from the same place in each for a pair
template <int CTAS>
__device__ __forceinline__ void scales_in(uint32_t taddr, uint32_t saddr) {
  const uint64_t desc = smem_desc(saddr, 16, 128, SWZ_NONE);
  if (CTAS == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

// A stage: rows of a and b, then their scales, a's tiles and those of each 128 rows of b.
template <int BLOCK>
struct Scales {
  static constexpr int kTiles = BK / BLOCK / 4;                       // beside one another in a stage
  static constexpr uint32_t kBytes = kTiles * (uint32_t)kTileBytes;   // of 128 rows
};

// The MMAs of a stage, by one thread: `steps` of 64 columns, four (FULL) but in the last stage.  ts: columns for scales, 4 for each tile of a's and of
// b's.  Copies and MMAs of one thread are carried out in their order, so a tile's columns are free when the next stage's copies come.
template <int CTAS, int BLOCK, int BGROUPS, bool FULL>
__device__ __forceinline__ void issue_steps(uint32_t acc, uint32_t ts, uint32_t a, uint32_t b, uint32_t sa, uint32_t idesc, int steps, bool first) {
  typedef Scales<BLOCK> S;
#pragma unroll
  for (int tile = 0; tile < S::kTiles; ++tile) {
    if (FULL || tile * BLOCK < 16 * steps) {
      const uint32_t ca = ts + 4 * tile, cb = ts + 4 * S::kTiles + 4 * BGROUPS * tile, at = sa + tile * kTileBytes;
      scales_in<CTAS>(ca, at);
      scales_in<CTAS>(cb, at + S::kBytes);
      if (BGROUPS == 2) scales_in<CTAS>(cb + 4, at + 2 * S::kBytes);
    }
  }
  const uint64_t da = tile_desc(a, ROW), db = tile_desc(b, ROW);
#pragma unroll
  for (int k = 0; k < BK / 64; ++k) {
    if (FULL || k < steps) {
      const int tile = BLOCK == 16 ? k : k >> 1, id = BLOCK == 16 ? 0 : 2 * (k & 1);
      mma_fp4<CTAS, BLOCK>(acc, da + 2 * k, db + 2 * k, idesc | (uint32_t)id << 4 | (uint32_t)id << 29, ts + 4 * tile,
                           ts + 4 * S::kTiles + 4 * BGROUPS * tile, !first || k > 0);
    }
  }
}
template <int CTAS, int BLOCK, int BGROUPS>
__device__ __forceinline__ void issue_stage(uint32_t acc, uint32_t ts, uint32_t a, uint32_t b, uint32_t sa, uint32_t idesc, int steps, bool first) {
  if (steps >= BK / 64) issue_steps<CTAS, BLOCK, BGROUPS, true>(acc, ts, a, b, sa, idesc, steps, first);
  else issue_steps<CTAS, BLOCK, BGROUPS, false>(acc, ts, a, b, sa, idesc, steps, first);
}

// ------------------------------------------------------------------------------------------------ pairs of SMs
// Tiles of 256 x 256 for two SMs (cta_group::2), persistent: each CTA of a pair loads 128 rows of x, 128 of w and the scales of its rows of x and of all
// 256 of w, the first one issues the MMAs, and each drains its 128 rows of the accumulator while the next tile's is formed.  Two accumulators
// of 256 columns would be all of tensor memory: they share 48 columns, which the scales take at its end, and an epilogue reads
// the shared ones first.  (Four stages of 38 KB and two slabs to an epilogue warp; five stages and one slab: 100 us where these take 97.  Rows
// stored by their lanes, without slabs: 124.  Sixteen epilogue warps of 64 columns: 116, no gain where the epilogue is waited for.)
constexpr int PBN = 256, PT = 384, kShared = 48;
struct PairLayout {
  static constexpr int kStages = 4;
  static constexpr uint32_t kA = 128 * ROW, kScales = 2 * kA, kStage = kScales + 3 * Scales<16>::kBytes;
  static constexpr uint32_t kSlabs = kStages * kStage;           // of each epilogue warp: twice 32 rows of 128 bytes on their way out
  static constexpr uint32_t kCols = kSlabs + 8 * 2 * 4096;       // step sizes and biases of two tiles' columns
  static constexpr uint32_t kBars = kCols + 2 * 2 * PBN * 4;
  static constexpr uint32_t kAlloc = kBars + 256;
};
static_assert(PairLayout::kStage % 1024 == 0 && PairLayout::kAlloc <= 232448, "tiles start on 1024 bytes, and there are 227 KB");

__device__ __forceinline__ void tma_store_wait_read_but_one() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }
// (relaxed: what it says is that reads of tensor memory are over, which they are before it is issued; a release would wait for stores)
__device__ __forceinline__ void arrive_relaxed_at(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// One epilogue warp: a quarter's 32 rows (lanes) of 128 columns of an accumulator, in units of 128 bytes of out's rows (64 columns, or 32 of
// binary32), each through one of the warp's two slabs in shared memory.  Where out's rows (and the residual's) lie on 16-byte boundaries TMA brings the
// residual of a unit into its slab, a unit ahead, and takes the unit from there; it leaves out what is beyond the last row and column.  Other rows
// are read back from the slabs as binary32, a row at a time by lanes that stand beside one another in it, and stored in words of
// four bytes: in an odd row, one of 16-bit elements that starts in the middle of a word, lane j has elements 2 j - 1 and 2 j, and the
// row's own lane stores both ends.  (The residual's words, of this unit and the next, are 64 of the 168 registers: 8 bytes spill, 112 in binary32.)
enum { ROWS_VECTORS = 0, ROWS_WORDS = 1, ROWS_ODD = 2 };   // out's rows (and the residual's) on 16 bytes, on words (binary32: elements), on 16-bit elements
template <typename T, int ROWS>
struct Epilogue {
  static constexpr bool vectors = ROWS == ROWS_VECTORS;
  static constexpr int U = 128 / sizeof(T);   // columns of a unit
  typedef typename std::conditional<sizeof(T) == 4, uint32_t, uint16_t>::type Bits;

  const Fp4Params& p;
  const CUtensorMap *tout, *tres;
  uint8_t* slab;
  uint64_t* bar;         // of each slab's residual
  const int lane;
  uint32_t phase = 0;    // of the barriers, a bit each
  int t0, n0, end;       // the tile's first row of the warp, its first column, where its columns end
  float sr;
  // rows on other boundaries: the residual of a unit, this lane's word of each of 32 rows, and both ends of its own; the next unit's on its way in the
  // other half, so the halves are named where they are used
  uint32_t res[2][32], ends[2];
  float head, tail;         // ends of this lane's row

  __device__ __forceinline__ Epilogue(const Fp4Params& p_, const CUtensorMap* tout_, const CUtensorMap* tres_, uint8_t* slab_, uint64_t* bar_)
      : p(p_), tout(tout_), tres(tres_), slab(slab_), bar(bar_), lane(threadIdx.x & 31) {}

  __device__ __forceinline__ void tile(int t_first, int n_first) {
    t0 = t_first;
    n0 = n_first;
    end = min(n0 + 128, p.O);
    sr = t0 + lane < p.T ? (p.s_row ? p.s_row[t0 + lane] : 1.0f) : 0.f;
  }
  static __device__ __forceinline__ int odd_row(const void* q) { return (int)(reinterpret_cast<uintptr_t>(q) >> 1 & 1); }

  // the first column of a tile's i-th unit
  static __device__ __forceinline__ int column_of(int i, bool down) { return (i * U) ^ (down ? 64 : 0); }
  // the residual of the unit at (t, o) on its way into a slab, by one lane
  __device__ __forceinline__ void request(int slot, int t, int o) {
    if (t < p.T && o < p.O) {
      mbar_expect_tx(&bar[slot], 4096);
      tma_load_2d(slab + slot * 4096, tres, &bar[slot], o, t);
    }
  }
  // ahead of the first tile: its first unit's
  __device__ __forceinline__ void begin(int t, int n, bool down) {
    if (vectors && p.residual && lane == 0) request(0, t, n + column_of(0, down));
    fetch<0>(t, n + column_of(0, down));
  }
  // rows on other boundaries: the residual of the tile at (t, n) into L2, a tile ahead
  __device__ __forceinline__ void ahead(int t, int n) {
    if (!vectors && p.residual && t + lane < p.T && n < p.O) {
      const uint8_t* const at = reinterpret_cast<const uint8_t*>(static_cast<const T*>(p.residual) + (t + lane) * p.res_stride + n);
      const int bytes = min(128, p.O - n) * (int)sizeof(T);
      for (int o = 0; o < bytes; o += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(at + o));
      asm volatile("prefetch.global.L2 [%0];" ::"l"(at + bytes - 1));
    }
  }
  // rows on other boundaries: whole units are read and written without a check
  __device__ __forceinline__ bool whole(int t, int o) const { return t + 32 <= p.T && o + U <= p.O; }
  template <int SLOT>
  __device__ __forceinline__ void fetch(int t, int o) {
    if (vectors || !p.residual || !whole(t, o)) return;
    const Bits* at = static_cast<const Bits*>(p.residual) + t * p.res_stride + o;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int r = 0; r < 32; ++r, at += p.res_stride) res[SLOT][r] = at[lane];
    } else if constexpr (ROWS == ROWS_WORDS) {
#pragma unroll
      for (int r = 0; r < 32; ++r, at += p.res_stride) res[SLOT][r] = reinterpret_cast<const uint32_t*>(at)[lane];
    } else {
      const int odd0 = odd_row(static_cast<const T*>(p.out) + t * p.out_stride + o), odd1 = odd0 ^ (int)(p.out_stride & 1);   // of every other row
      const uint16_t* const own = at + lane * p.res_stride;
      ends[SLOT] = (uint32_t)own[0] | (uint32_t)own[63] << 16;
      if (odd_row(at) == odd0 && ((p.out_stride ^ p.res_stride) & 1) == 0) {
        // (lane 0's word of an odd row is the one that the row begins in: an element of the row before, or of the word ahead of a tensor that begins
        // in the middle of one, comes with it and is not used)
#pragma unroll
        for (int r = 0; r < 32; ++r, at += p.res_stride) res[SLOT][r] = *reinterpret_cast<const uint32_t*>(at - (r & 1 ? odd1 : odd0) + 2 * lane);
      } else {
#pragma unroll
        for (int r = 0; r < 32; ++r, at += p.res_stride) {
          const int first = 2 * lane - (r & 1 ? odd1 : odd0);
          res[SLOT][r] = (uint32_t)at[max(first, 0)] | (uint32_t)at[first + 1] << 16;
        }
      }
    }
  }
  // 32 columns of the accumulator, in pairs; one loop for each activation
  __device__ __forceinline__ void values(const int (&v)[32], const float* cw, const float* cb, float2 (&f)[16]) const {
    const float2 s2 = make_float2(sr, sr);
#pragma unroll
    for (int c = 0; c < 16; c += 2) {
      const float4 w = *reinterpret_cast<const float4*>(cw + 2 * c), b = *reinterpret_cast<const float4*>(cb + 2 * c);
      f[c] = __ffma2_rn(__fmul2_rn(make_float2(__int_as_float(v[2 * c]), __int_as_float(v[2 * c + 1])), s2), make_float2(w.x, w.y), make_float2(b.x, b.y));
      f[c + 1] = __ffma2_rn(__fmul2_rn(make_float2(__int_as_float(v[2 * c + 2]), __int_as_float(v[2 * c + 3])), s2), make_float2(w.z, w.w),
                            make_float2(b.z, b.w));
    }
    if (p.act == SSDI8_ACT_SILU) {
#pragma unroll
      for (int c = 0; c < 16; ++c) f[c] = make_float2(activate(f[c].x, SSDI8_ACT_SILU), activate(f[c].y, SSDI8_ACT_SILU));
    } else if (p.act == SSDI8_ACT_RELU2) {
#pragma unroll
      for (int c = 0; c < 16; ++c) f[c] = make_float2(activate(f[c].x, SSDI8_ACT_RELU2), activate(f[c].y, SSDI8_ACT_RELU2));
    }
  }
  // 32 columns, the first or second half of a unit of 16-bit elements, or all of one of binary32, into a slab
  __device__ __forceinline__ void into(float2 (&f)[16], int slot, int half) {
    if (vectors) {   // 16-byte chunks of a row of 128 bytes, as the 128-byte swizzle has them
      uint8_t* const to = slab + slot * 4096;
#pragma unroll
      for (int i = 0; i < 32 / (16 / (int)sizeof(T)); ++i) {
        uint4* const at = reinterpret_cast<uint4*>(to + swz_off(lane, (sizeof(T) == 4 ? 0 : 4 * half) + i, 128));
        if constexpr (sizeof(T) == 4) {
          float2 x = f[2 * i], y = f[2 * i + 1];
          if (p.residual) {
            const float4 r = *reinterpret_cast<const float4*>(at);
            x = __fadd2_rn(x, make_float2(r.x, r.y));
            y = __fadd2_rn(y, make_float2(r.z, r.w));
          }
          *at = make_uint4(__float_as_uint(x.x), __float_as_uint(x.y), __float_as_uint(y.x), __float_as_uint(y.y));
        } else {
          if (p.residual) {
            const uint4 r = *at;
            const float4 a = Elem<T>::cvt(make_uint2(r.x, r.y)), b = Elem<T>::cvt(make_uint2(r.z, r.w));
            f[4 * i] = __fadd2_rn(f[4 * i], make_float2(a.x, a.y));
            f[4 * i + 1] = __fadd2_rn(f[4 * i + 1], make_float2(a.z, a.w));
            f[4 * i + 2] = __fadd2_rn(f[4 * i + 2], make_float2(b.x, b.y));
            f[4 * i + 3] = __fadd2_rn(f[4 * i + 3], make_float2(b.z, b.w));
          }
          const uint2 a = Elem<T>::pack(make_float4(f[4 * i].x, f[4 * i].y, f[4 * i + 1].x, f[4 * i + 1].y));
          const uint2 b = Elem<T>::pack(make_float4(f[4 * i + 2].x, f[4 * i + 2].y, f[4 * i + 3].x, f[4 * i + 3].y));
          *at = make_uint4(a.x, a.y, b.x, b.y);
        }
      }
    } else {   // pairs of columns, at a place that depends on the row: no two lanes of a row or of a column meet in a bank
      constexpr int pairs = U / 2;
      if (half == 0) head = f[0].x;
      tail = f[15].y;
      float2* const to = reinterpret_cast<float2*>(slab) + lane * pairs;
#pragma unroll
      for (int c = 0; c < 16; ++c) to[((sizeof(T) == 4 ? 0 : 16 * half) + c) ^ (lane & (pairs - 1))] = f[c];
    }
  }
  // the slab is there for a unit: with the residual in it, or its last store, two units ago, read
  __device__ __forceinline__ void take(int slot, int c0) {
    if (!vectors) return;
    if (!p.residual) {
      if (lane == 0) tma_store_wait_read_but_one();
      __syncwarp();
    } else if (n0 + c0 < end && t0 < p.T) {
      mbar_wait(&bar[slot], phase >> slot & 1u, p.status);
      phase ^= 1u << slot;
    }
  }
  // a unit out of its slab; (t, o): the unit that comes next, whose residual may follow as soon as the other slab's store has been read
  template <int SLOT>
  __device__ __forceinline__ void leave(int c0, int t, int o) {
    constexpr int slot = SLOT;
    const int o0 = n0 + c0;
    if (vectors) {
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        if (p.residual) {
          tma_store_wait_read();
          request(slot ^ 1, t, o);
        }
        if (o0 < end && t0 < p.T) tma_store_2d(tout, slab + slot * 4096, o0, t0);
        tma_store_commit();
      }
      return;
    }
    fetch<SLOT ^ 1>(t, o);
    __syncwarp();
    constexpr int pairs = U / 2;
    const float* const turn = reinterpret_cast<const float*>(slab);
    auto column = [&](int r, int c) { return turn[r * U + (((c >> 1) ^ (r & (pairs - 1))) << 1) + (c & 1)]; };
    T* at = static_cast<T*>(p.out) + t0 * p.out_stride + o0;
    if (whole(t0, o0)) {
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int r = 0; r < 32; ++r, at += p.out_stride) {
          const float x = column(r, lane);
          at[lane] = p.residual ? x + __uint_as_float(res[SLOT][r]) : x;
        }
      } else {
        T* const own = at + lane * p.out_stride;
        const int odd0 = odd_row(at), odd1 = odd0 ^ (int)(p.out_stride & 1);
        if constexpr (ROWS == ROWS_WORDS) {
#pragma unroll
          for (int r = 0; r < 32; ++r, at += p.out_stride) {
            float2 x = reinterpret_cast<const float2*>(turn)[r * pairs + (lane ^ r)];
            if (p.residual) {
              const T* const m = reinterpret_cast<const T*>(&res[SLOT][r]);
              x = __fadd2_rn(x, make_float2(Elem<T>::get(m[0]), Elem<T>::get(m[1])));
            }
            reinterpret_cast<uint32_t*>(at)[lane] = Elem<T>::pack(make_float4(x.x, x.y, 0.f, 0.f)).x;
          }
        } else {
#pragma unroll
          for (int r = 0; r < 32; ++r, at += p.out_stride) {
            const int odd = r & 1 ? odd1 : odd0;
            float2 x = reinterpret_cast<const float2*>(turn)[r * pairs + (lane ^ r)];
            if (odd) x = make_float2(__shfl_up_sync(0xffffffffu, x.y, 1), x.x);
            if (p.residual) {
              const T* const m = reinterpret_cast<const T*>(&res[SLOT][r]);
              x = __fadd2_rn(x, make_float2(Elem<T>::get(m[0]), Elem<T>::get(m[1])));
            }
            if (lane > 0 || !odd) *reinterpret_cast<uint32_t*>(at - odd + 2 * lane) = Elem<T>::pack(make_float4(x.x, x.y, 0.f, 0.f)).x;
          }
          if (odd_row(own)) {
            const T* const m = reinterpret_cast<const T*>(&ends[SLOT]);
            own[0] = Elem<T>::put(p.residual ? head + Elem<T>::get(m[0]) : head);
            own[63] = Elem<T>::put(p.residual ? tail + Elem<T>::get(m[1]) : tail);
          }
        }
      }
    } else if (o0 < end) {
      // the last rows and columns, by elements, sixteen rows at a time
      constexpr int E = U / 32;
      const T* rat = static_cast<const T*>(p.residual) + t0 * p.res_stride + o0;
      const int rows = p.T - t0;
#pragma unroll 1
      for (int r0 = 0; r0 < 32 && r0 < rows; r0 += 16) {
        float x[16][E];
#pragma unroll
        for (int i = 0; i < 16; ++i, rat += p.res_stride)
#pragma unroll
          for (int e = 0; e < E; ++e)
            x[i][e] = p.residual && r0 + i < rows && o0 + lane + 32 * e < end ? Elem<T>::get(rat[lane + 32 * e]) : 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i, at += p.out_stride)
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (r0 + i < rows && o0 + lane + 32 * e < end) {
              const float y = column(r0 + i, lane + 32 * e);
              at[lane + 32 * e] = Elem<T>::put(p.residual ? y + x[i][e] : y);
            }
      }
    }
    __syncwarp();
  }
  // all 128 columns, the halves from the first or from the last on (down); `ready` waits for the accumulator, `drained` is called once the first half is
  // in registers; (t, n): the next tile, which goes the other way (t = p.T: none)
  template <typename R, typename F>
  __device__ __forceinline__ void run(uint32_t tmem, bool down, const float* cw, const float* cb, int t, int n, R ready, F drained) {
    ready();
    auto half = [&](auto which) {
      constexpr int i = decltype(which)::value;
      const int c0 = column_of(i * (64 / U), down);
      int v[32], u[32];
      tmem_ld32(tmem + c0, v);
      tmem_ld32(tmem + c0 + 32, u);
      tmem_ld_wait();
      if (i == 0) {
        tc_fence_before();
        drained();
      }
      const int tn = i == 0 ? t0 : t, on = i == 0 ? n0 + (c0 ^ 64) : n + column_of(0, !down);   // the first unit behind these
      float2 f[16];
      values(v, cw + c0, cb + c0, f);
      if constexpr (sizeof(T) == 4) {
        take(0, c0);
        into(f, 0, 0);
        leave<0>(c0, t0, n0 + c0 + 32);
        values(u, cw + c0 + 32, cb + c0 + 32, f);
        take(1, c0 + 32);
        into(f, 1, 0);
        leave<1>(c0 + 32, tn, on);
      } else {
        take(i, c0);
        into(f, i, 0);
        values(u, cw + c0 + 32, cb + c0 + 32, f);
        into(f, i, 1);
        leave<i>(c0, tn, on);
      }
    };
    half(std::integral_constant<int, 0>());
    half(std::integral_constant<int, 1>());
  }
};

template <typename T, int BLOCK, int ROWS>
__global__ void __launch_bounds__(PT, 1) fp4_pair_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ CUtensorMap tw,
                                                         const __grid_constant__ CUtensorMap tsx, const __grid_constant__ CUtensorMap tsw,
                                                         const __grid_constant__ CUtensorMap tout, const __grid_constant__ CUtensorMap tres,
                                                         const __grid_constant__ Fp4Params p) {
  typedef PairLayout S;
  constexpr uint32_t kSc = Scales<BLOCK>::kBytes;
  extern __shared__ __align__(1024) uint8_t smem[];   // (there is no static part: the window's base is on 1024 bytes)
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kBars);   // (waited for in the first CTA; the second's loads arrive there too)
  uint64_t* empty = full + S::kStages;
  uint64_t* acc_full = empty + S::kStages;
  uint64_t* acc_free = acc_full + 2;                               // (waited for in the first CTA)
  uint64_t* res_full = acc_free + 2;                               // of the epilogue warps' slabs
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(res_full + 16);
  float* cols = reinterpret_cast<float*>(smem + S::kCols);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = blockIdx.x & 1, pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  if (tid == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_free[i], 16);   // the epilogue warps of both
    }
    for (int i = 0; i < 16; ++i) mbar_init(&res_full[i], 1);
    fence_mbar_init();
    tma_prefetch_desc(&tx);
    tma_prefetch_desc(&tw);
    tma_prefetch_desc(&tsx);
    tma_prefetch_desc(&tsw);
    tma_prefetch_desc(&tout);
    tma_prefetch_desc(&tres);
  }
  __syncthreads();
  cluster_sync();   // (the other CTA's barriers are there)
  pdl_wait();
  const uint32_t tmem = warp == 0 ? 0u : allocated<2>(tmem_slot, 512, warp, PT);
  const int ntotal = p.mtiles * p.ntiles;
  if (warp == 0) {
    int it = 0;
    for (int tile = pair; tile < ntotal; tile += npairs) {
      int m, n;
      tile_of<8>(tile, p.mtiles, p.ntiles, &m, &n);
      for (int kb = 0; kb < p.kblocks; ++kb, ++it) {
        const int s = it % S::kStages;
        if (it >= S::kStages) mbar_wait(&empty[s], (it / S::kStages - 1) & 1, p.status);
        if (elect_one()) {
          if (rank == 0) mbar_expect_tx(&full[s], 2 * (2 * S::kA + 3 * kSc));
          const uint32_t bar = in_first(&full[s]);
          uint8_t* const at = smem + s * S::kStage;
          pair_load(at, &tx, bar, kb * ROW, m * 256 + rank * 128);
          pair_load(at + S::kA, &tw, bar, kb * ROW, n * PBN + rank * 128);
          const int tile4 = kb * Scales<BLOCK>::kTiles * 4;
          pair_load(at + S::kScales, &tsx, bar, 0, (m * 2 + rank) * p.tiles * 4 + tile4);
          pair_load(at + S::kScales + kSc, &tsw, bar, 0, n * 2 * p.tiles * 4 + tile4);
          pair_load(at + S::kScales + 2 * kSc, &tsw, bar, 0, (n * 2 + 1) * p.tiles * 4 + tile4);
        }
        __syncwarp();
      }
    }
    // (the last commits have arrived here before this CTA ends)
    for (int k = it > S::kStages ? it - S::kStages : 0; k < it; ++k) mbar_wait(&empty[k % S::kStages], (k / S::kStages) & 1, p.status);
  } else if (warp == 1 && rank == 0) {
    int it = 0, at = 0;
    for (int tile = pair; tile < ntotal; tile += npairs, ++at) {
      const int buf = at & 1;
      // (the tile before has left the shared columns, and so the one before it all of its)
      if (at >= 1) mbar_wait(&acc_free[buf ^ 1], ((at - 1) >> 1) & 1, p.status);
      tc_fence_after();
      for (int kb = 0; kb < p.kblocks; ++kb, ++it) {
        const int s = it % S::kStages;
        mbar_wait(&full[s], (it / S::kStages) & 1, p.status);
        tc_fence_after();
        if (elect_one()) {
          const uint32_t a = smem_u32(smem + s * S::kStage);
          issue_stage<2, BLOCK, 2>(tmem + buf * (PBN - kShared), tmem + 2 * PBN - kShared, a, a + S::kA, a + S::kScales, idesc_fp4(256, PBN, BLOCK),
                                   p.steps - kb * (BK / 64), kb == 0);
          pair_commit(&empty[s]);
          if (kb + 1 == p.kblocks) pair_commit(&acc_full[buf]);
        }
        __syncwarp();
      }
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3, upper = (warp - 4) >> 2, et = tid & 127;   // eight warps: a quarter of the rows, half of the columns
    Epilogue<T, ROWS> ep(p, &tout, &tres, smem + S::kSlabs + (warp - 4) * 2 * 4096, res_full + (warp - 4) * 2);
    // a column's step size and bias, a tile ahead
    float w = 0.f, b = 0.f;
    auto column = [&](int n) {
      const int o = n * PBN + upper * 128 + et;
      w = o < p.O ? (p.s_w ? p.s_w[o] : 1.0f) : 0.f;
      b = o < p.O && p.bias ? p.bias[o] : 0.f;
    };
    int at = 0, m, n;
    tile_of<8>(pair, p.mtiles, p.ntiles, &m, &n);
    column(n);
    ep.ahead(m * 256 + rank * 128 + quarter * 32, n * PBN + upper * 128);
    ep.begin(m * 256 + rank * 128 + quarter * 32, n * PBN + upper * 128, true);
    for (int tile = pair; tile < ntotal; tile += npairs, ++at) {
      const int buf = at & 1;
      float* const cw = cols + (buf * 2 + upper) * 256;
      cw[et] = w;
      cw[128 + et] = b;
      ep.tile(m * 256 + rank * 128 + quarter * 32, n * PBN + upper * 128);
      if (tile + npairs < ntotal) {
        tile_of<8>(tile + npairs, p.mtiles, p.ntiles, &m, &n);
        column(n);
        ep.ahead(m * 256 + rank * 128 + quarter * 32, n * PBN + upper * 128);
      }
      named_bar_sync(3 + upper, 128);   // the four warps of these columns (nobody is still reading those of the tile before the last)
      // The shared columns are the last of the first accumulator and the first of the second: the upper half's or the lower's.  The warps of the other
      // half have nothing there; what they say is that they are through with the tile before, which had the accumulator that the next tile gets.
      const bool shared = upper != buf;
      auto free = [&] {
        __syncwarp();
        if (lane == 0) arrive_relaxed_at(in_first(&acc_free[buf]));
      };
      if (!shared) free();
      ep.run(tmem + ((uint32_t)(quarter * 32) << 16) + buf * (PBN - kShared) + upper * 128, buf == 0, cw, cw + 128,
             tile + npairs < ntotal ? m * 256 + rank * 128 + quarter * 32 : p.T, n * PBN + upper * 128,
             [&] { mbar_wait(&acc_full[buf], (at >> 1) & 1, p.status); tc_fence_after(); }, [&] {
               if (shared) free();
             });
      tc_fence_before();   // (what the next tile's arrival vouches for)
    }
    if (lane == 0) tma_store_wait_read();
  }
  tc_fence_before();
  __syncthreads();
  drain_after_timeout(p.status);
  cluster_sync();   // (nothing of the other CTA's is on its way here any more: its commits and arrivals have been waited for or precede this)
  if (warp == 2) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------ few rows
// The weight's rows are the accumulator's 128 lanes and up to 256 tokens its columns, a tile to a CTA, and K is shared out among the CTAs of a cluster
// until the SMs are all at it.  The parts of a tile meet in shared memory, added in the order of their CTAs, each CTA finishing some tokens.
constexpr int FT = 256;
struct FewLayout : Fp4Few {
  static constexpr uint32_t kRows = 256, kTail = kRows + 256 * 4 + 1024;   // barriers, step sizes of rows; the tiles start on 1024 bytes
};
static_assert(2 * (FewLayout::kSmall + FewLayout::kTail + 1024) <= 233472 && FewLayout::kLarge + FewLayout::kTail <= 232448, "");
static_assert(FewLayout::kRow == ROW && FewLayout::scales(16) == Scales<16>::kBytes && FewLayout::scales(32) == Scales<32>::kBytes, "");
struct FewParams {
  Fp4Params l;
  int n, bgroups, split, stages;   // columns of the accumulator (tokens, to 16), their 128s, CTAs of a cluster
  uint32_t ring, columns;          // bytes; of tensor memory
};

__device__ __forceinline__ float4 ld_from(const float* p, int rank) {   // the same place in another CTA of the cluster
  uint32_t a;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}
// (relaxed: nothing was written for the others, and what was read of theirs has been used; a release would wait for stores to out)
__device__ __forceinline__ void cluster_leave() {
  asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
  cluster_wait();
}

// A CTA's tokens, every split-th one, a warp to a token and four outputs to a lane: the parts of four tokens and their residuals on their way at a time
template <typename T, int ACT>
__device__ __forceinline__ void few_out(const FewParams& f, const float* part, const float* s_row, int rank, int tok0, int ntok, int o, int no,
                                        const float (&sw)[4], const float (&bias)[4]) {
  const Fp4Params& p = f.l;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, step = f.split * (FT / 32), first = rank + f.split * warp;
  const bool vector = no == 4 && p.vec_out && (!p.residual || p.vec_res);
  T* dst = static_cast<T*>(p.out) + (i64)(tok0 + first) * p.out_stride + o;
  const T* res = static_cast<const T*>(p.residual) + (i64)(tok0 + first) * p.res_stride + o;
  const i64 dstep = (i64)step * p.out_stride, rstep = (i64)step * p.res_stride;
  const float2 w0 = make_float2(sw[0], sw[1]), w1 = make_float2(sw[2], sw[3]), b0 = make_float2(bias[0], bias[1]), b1 = make_float2(bias[2], bias[3]);
#pragma unroll 1
  for (int t0 = first; t0 < ntok; t0 += 4 * step, dst += 4 * dstep, res += 4 * rstep) {
    float4 acc[4] = {};
    typename Elem<T>::raw4 q[4];
    if (p.residual) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (t0 + u * step >= ntok) break;
        const T* const r = res + u * rstep;
        if (vector) {
          q[u] = *reinterpret_cast<const typename Elem<T>::raw4*>(r);
        } else {
          T* const e4 = reinterpret_cast<T*>(&q[u]);
#pragma unroll
          for (int e = 0; e < 4; ++e) e4[e] = e < no ? r[e] : Elem<T>::put(0.f);
        }
      }
    }
    const auto parts = [&](auto all) {
      // (of the others' none behind the last token: a read that nothing uses could still be on its way when the CTA that it goes to has left)
      const auto read = [&](int u, int r) { return ld_from(part + (t0 + u * step) * 128 + 4 * lane, r); };
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (decltype(all)::value || t0 + u * step < ntok) acc[u] = read(u, 0);
      for (int r = 1; r < f.split; ++r) {
        float4 v[4] = {};
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (decltype(all)::value || t0 + u * step < ntok) v[u] = read(u, r);
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[u] = make_float4(acc[u].x + v[u].x, acc[u].y + v[u].y, acc[u].z + v[u].z, acc[u].w + v[u].w);
      }
    };
    if (f.split == 1) {
#pragma unroll
      for (int u = 0; u < 4; ++u) acc[u] = *reinterpret_cast<const float4*>(part + min(t0 + u * step, ntok - 1) * 128 + 4 * lane);
    } else if (t0 + 3 * step < ntok) {
      parts(std::true_type());
    } else {
      parts(std::false_type());
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (t0 + u * step >= ntok) break;
      const float sr = s_row[t0 + u * step];
      float2 x = __ffma2_rn(__fmul2_rn(make_float2(acc[u].x, acc[u].y), make_float2(sr, sr)), w0, b0);
      float2 y = __ffma2_rn(__fmul2_rn(make_float2(acc[u].z, acc[u].w), make_float2(sr, sr)), w1, b1);
      x = make_float2(activate(x.x, ACT), activate(x.y, ACT));
      y = make_float2(activate(y.x, ACT), activate(y.y, ACT));
      if (p.residual) {
        const float4 r = Elem<T>::cvt(q[u]);
        x = __fadd2_rn(x, make_float2(r.x, r.y));
        y = __fadd2_rn(y, make_float2(r.z, r.w));
      }
      if (vector) {
        *reinterpret_cast<typename Elem<T>::raw4*>(dst + u * dstep) = Elem<T>::pack(make_float4(x.x, x.y, y.x, y.y));
      } else if (sizeof(T) == 2 && no == 4) {   // words where the row's boundary allows
        const typename Elem<T>::raw4 w4 = Elem<T>::pack(make_float4(x.x, x.y, y.x, y.y));
        const uint32_t* const w = reinterpret_cast<const uint32_t*>(&w4);
        uint16_t* const d = reinterpret_cast<uint16_t*>(dst + u * dstep);
        if ((reinterpret_cast<uintptr_t>(d) & 2) == 0) {
          reinterpret_cast<uint32_t*>(d)[0] = w[0];
          reinterpret_cast<uint32_t*>(d)[1] = w[1];
        } else {
          d[0] = (uint16_t)w[0];
          *reinterpret_cast<uint32_t*>(d + 1) = __byte_perm(w[0], w[1], 0x5432);
          d[3] = (uint16_t)(w[1] >> 16);
        }
      } else {
        const float v[4] = {x.x, x.y, y.x, y.y};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < no) dst[u * dstep + e] = Elem<T>::put(v[e]);
      }
    }
  }
}

template <typename T, int BLOCK>
__global__ void __launch_bounds__(FT, 2) fp4_few_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ CUtensorMap tw,
                                                        const __grid_constant__ CUtensorMap tsx, const __grid_constant__ CUtensorMap tsw,
                                                        const __grid_constant__ FewParams f) {
  typedef FewLayout S;
  constexpr uint32_t kSc = Scales<BLOCK>::kBytes;
  const Fp4Params& p = f.l;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + f.ring);
  uint64_t* empty = full + S::kMaxStages;
  uint64_t* acc_full = empty + S::kMaxStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_full + 1);
  float* s_row = reinterpret_cast<float*>(smem + f.ring + S::kRows);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < S::kMaxStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    mbar_init(acc_full, 1);
    fence_mbar_init();
    tma_prefetch_desc(&tx);
    tma_prefetch_desc(&tw);
    tma_prefetch_desc(&tsx);
    tma_prefetch_desc(&tsw);
  }
  __syncthreads();
  pdl_wait();
  if (warp != 0) allocated<1>(tmem_slot, f.columns, warp, FT);
  // CTAs of a cluster, then the tiles of tokens, then those of the weight (which their CTAs share in L2)
  const int rank = blockIdx.x % f.split, tile = blockIdx.x / f.split, m = tile / p.ntiles, n = tile % p.ntiles;
  const int o0 = m * 128, tok0 = n * f.n, ntok = min(f.n, p.T - tok0);
  const int kb0 = (int)((i64)p.kblocks * rank / f.split), kb1 = (int)((i64)p.kblocks * (rank + 1) / f.split);
  // (n % 16 = 0: codes and scales start on 1024 bytes)
  const uint32_t scales = S::kW + f.n * ROW, stage = (scales + (1 + f.bgroups) * kSc + 1023) & ~1023u;   // (as S::stage has it on the host)
  if (warp == 0) {
    int s = 0, round = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (round > 0) mbar_wait(&empty[s], (round - 1) & 1, p.status);
      if (elect_one()) {
        uint8_t* const at = smem + s * stage;
        const int tile4 = kb * Scales<BLOCK>::kTiles * 4;
        mbar_expect_tx(&full[s], scales + (1 + f.bgroups) * kSc);
        tma_load_2d(at, &tw, &full[s], kb * ROW, o0);
        tma_load_2d(at + scales, &tsw, &full[s], 0, m * p.tiles * 4 + tile4);
        tma_load_2d(at + S::kW, &tx, &full[s], kb * ROW, tok0);
        for (int g = 0; g < f.bgroups; ++g) tma_load_2d(at + scales + (1 + g) * kSc, &tsx, &full[s], 0, ((tok0 >> 7) + g) * p.tiles * 4 + tile4);
      }
      __syncwarp();
      if (++s == f.stages) { s = 0; ++round; }
    }
  } else if (warp == 1) {
    const uint32_t tmem = *tmem_slot, idesc = idesc_fp4(128, f.n, BLOCK), base = smem_u32(smem);
    const auto issue = [&](auto groups) {
      int s = 0, round = 0;
      for (int kb = kb0; kb < kb1; ++kb) {
        mbar_wait(&full[s], round & 1, p.status);
        tc_fence_after();
        if (elect_one()) {
          const uint32_t a = base + s * stage;
          issue_stage<1, BLOCK, decltype(groups)::value>(tmem, tmem + f.n, a, a + S::kW, a + scales, idesc, p.steps - kb * (BK / 64), kb == kb0);
          mma_commit(&empty[s]);
          if (kb + 1 == kb1) mma_commit(acc_full);
        }
        __syncwarp();
        if (++s == f.stages) { s = 0; ++round; }
      }
    };
    if (f.bgroups == 1) issue(std::integral_constant<int, 1>());
    else issue(std::integral_constant<int, 2>());
  } else if (warp == 3) {
    for (int i = lane; i < ntok; i += 32) s_row[i] = p.s_row ? p.s_row[tok0 + i] : 1.0f;
  }
  // a warp per token in the end, four outputs per lane
  const int o = o0 + 4 * lane, no = min(p.O - o, 4);
  float sw[4], bias[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    sw[e] = e < no ? (p.s_w ? p.s_w[o + e] : 1.0f) : 0.f;
    bias[e] = e < no && p.bias ? p.bias[o + e] : 0.f;
  }
  float* const part = reinterpret_cast<float*>(smem);   // [n][128]
  __syncthreads();
  {
    // the accumulator over the ring: every load has been consumed by an MMA that is complete.  Two warps to a quarter of the lanes.
    const int quarter = warp & 3;
    mbar_wait(acc_full, 0, p.status);
    tc_fence_after();
    const uint32_t at = *tmem_slot + ((uint32_t)(quarter * 32) << 16);
    float* const to = part + quarter * 32 + lane;
    for (int c0 = warp >> 2 << 4; c0 < f.n; c0 += 32) {
      int v[16];
      tmem_ld8(at + c0, reinterpret_cast<int(&)[8]>(v[0]));
      tmem_ld8(at + c0 + 8, reinterpret_cast<int(&)[8]>(v[8]));
      tmem_ld_wait();
#pragma unroll
      for (int c = 0; c < 16; ++c) to[(c0 + c) * 128] = __int_as_float(v[c]);
    }
    tc_fence_before();
  }
  __syncthreads();
  if (f.split > 1) cluster_sync();
  if (no > 0) {
    const auto finish = [&](auto act) { few_out<T, decltype(act)::value>(f, part, s_row, rank, tok0, ntok, o, no, sw, bias); };
    if (p.act == SSDI8_ACT_SILU) finish(std::integral_constant<int, SSDI8_ACT_SILU>());
    else if (p.act == SSDI8_ACT_RELU2) finish(std::integral_constant<int, SSDI8_ACT_RELU2>());
    else finish(std::integral_constant<int, SSDI8_ACT_NONE>());
  }
  drain_after_timeout(p.status);
  if (f.split > 1) cluster_leave();   // (the others have read this CTA's part)
  else __syncthreads();
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(*tmem_slot, f.columns);
  }
}

template <typename T, int BLOCK>
ssdi8_status_t launch(const ssdi8_fp4_linear_args_t& a, cudaStream_t st) {
  const i64 e = sizeof(T);
  const ssdi8_fp4_t &x = *a.x, &w = *a.w;
  Fp4Params p = {};
  p.s_row = x.step; p.s_w = w.step; p.bias = a.bias;
  p.residual = a.residual; p.res_stride = a.stride_residual; p.out = a.out; p.out_stride = a.stride_out;
  p.status = a.status;
  p.T = x.rows; p.O = w.rows; p.act = a.act;
  p.steps = (x.width + 63) / 64;
  p.kblocks = (x.width + BK - 1) / BK;
  p.tiles = fp4_tiles(x.width, BLOCK);
  auto vec = [e](const void* q, i64 stride) { return reinterpret_cast<uintptr_t>(q) % 16 == 0 && stride * e % 16 == 0; };
  p.vec_out = vec(a.out, a.stride_out);
  p.vec_res = vec(a.residual, a.stride_residual);
  const int sms = sm_count();
  if (sms <= 0) return SSDI8_ERR_CUDA;
  CUtensorMap tx, tw, tsx, tsw;
  auto codes = [&](CUtensorMap* tm, const ssdi8_fp4_t& q, uint32_t rows) {
    const uint64_t dims[2] = {(uint64_t)q.width / 2, (uint64_t)q.rows}, stride[1] = {(uint64_t)q.width / 2};
    const uint32_t box[2] = {ROW, rows};
    return encode_tensor_map(tm, q.codes, 1, 2, dims, stride, box, 128);
  };
  // tiles of scales as rows of 128 bytes, four to a tile (what lies beyond the last one of a row block is the next one's: no step reads it)
  auto scales = [&](CUtensorMap* tm, const ssdi8_fp4_t& q) {
    const uint64_t dims[2] = {32, (uint64_t)((q.rows + 127ll) / 128 * p.tiles * 4)}, stride[1] = {128};
    const uint32_t box[2] = {32, 4 * Scales<BLOCK>::kTiles};
    return encode_tensor_map(tm, q.scales, 4, 2, dims, stride, box, 0);
  };
  if (!scales(&tsx, x) || !scales(&tsw, w)) return SSDI8_ERR_CUDA;
  const Fp4Form form = fp4_form(x.rows, w.rows, x.width, BLOCK, p.vec_out, sms);
  const i64 mt = (w.rows + 127ll) / 128, ptiles = (i64)((x.rows + 255ll) / 256) * ((w.rows + PBN - 1ll) / PBN), pairs = sms / 2;
  if (form.pair) {
    if (ptiles > 0x3fffffff) return SSDI8_ERR_SHAPE;
    p.mtiles = (int)((x.rows + 255ll) / 256);
    p.ntiles = (int)((w.rows + PBN - 1ll) / PBN);
    if (!codes(&tx, x, 128) || !codes(&tw, w, 128)) return SSDI8_ERR_CUDA;
    // (a map's rows lie behind one another: a residual whose rows overlap, one row for all among them, is read by the lanes, and a lone row of
    // out, which may have any stride, written by them.  Where rows are not on 16 bytes the maps are not used)
    CUtensorMap tout = tx;
    const uint64_t dims[2] = {(uint64_t)p.O, (uint64_t)p.T}, stride[1] = {(uint64_t)(a.stride_out * e)};
    const uint32_t box[2] = {(uint32_t)(128 / e), 32};
    if (p.vec_out && (a.stride_out < w.rows || !encode_tensor_map(&tout, a.out, (int)e, 2, dims, stride, box, 128))) p.vec_out = 0;
    CUtensorMap tres = tx;
    const uint64_t rstride[1] = {(uint64_t)(a.stride_residual * e)};
    if (a.residual && p.vec_res && (a.stride_residual < w.rows || !encode_tensor_map(&tres, a.residual, (int)e, 2, dims, rstride, box, 128))) p.vec_res = 0;
    auto go = [&](auto rows) {
      return launch_any(fp4_pair_kernel<T, BLOCK, decltype(rows)::value>, dim3((unsigned)(2 * (ptiles < pairs ? ptiles : pairs))), 2, dim3(PT), PairLayout::kAlloc,
                        PairLayout::kAlloc, -1, true, st, tx, tw, tsx, tsw, tout, tres, p);
    };
    if (p.vec_out && (!a.residual || p.vec_res)) return go(std::integral_constant<int, ROWS_VECTORS>());
    auto words = [](const void* q, i64 stride) { return reinterpret_cast<uintptr_t>(q) % 4 == 0 && stride % 2 == 0; };
    if (sizeof(T) == 4 || (words(a.out, a.stride_out) && (!a.residual || words(a.residual, a.stride_residual)))) return go(std::integral_constant<int, ROWS_WORDS>());
    if constexpr (sizeof(T) == 2) return go(std::integral_constant<int, ROWS_ODD>());
  }
  FewParams f = {};
  f.n = form.n;
  f.split = form.split;
  f.ring = form.ring;
  f.stages = form.stages;
  f.l = p;
  f.l.mtiles = (int)mt;
  f.l.ntiles = (int)((x.rows + f.n - 1ll) / f.n);
  f.bgroups = f.n <= 128 ? 1 : 2;
  const int need = f.n + 4 * Scales<BLOCK>::kTiles * (1 + f.bgroups);
  f.columns = need <= 64 ? 64 : need <= 128 ? 128 : need <= 256 ? 256 : 512;
  const i64 grid = (i64)f.l.mtiles * f.l.ntiles * f.split;
  if (grid > 0x7fffffff) return SSDI8_ERR_SHAPE;
  if (!codes(&tx, x, f.n) || !codes(&tw, w, 128)) return SSDI8_ERR_CUDA;
  return launch_any(fp4_few_kernel<T, BLOCK>, dim3((unsigned)grid), f.split, dim3(FT), f.ring + FewLayout::kTail, FewLayout::kLarge + FewLayout::kTail, -1,
                    false, st, tx, tw, tsx, tsw, f);
}

}  // namespace

ssdi8_status_t launch_fp4_linear(const ssdi8_fp4_linear_args_t& a, int dtype, cudaStream_t st) {
  if (a.x->block == 16)
    return dtype == 0 ? launch<float, 16>(a, st) : dtype == 1 ? launch<__half, 16>(a, st) : launch<__nv_bfloat16, 16>(a, st);
  return dtype == 0 ? launch<float, 32>(a, st) : dtype == 1 ? launch<__half, 32>(a, st) : launch<__nv_bfloat16, 32>(a, st);
}

}  // namespace ssdi8
