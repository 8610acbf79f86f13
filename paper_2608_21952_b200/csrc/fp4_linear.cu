// Product of two matrices in four bits: out = act(step_x step_w (x w^T) + bias) + residual, on tcgen05.mma with block scales (e2m1 operands, fp32
// accumulators in tensor memory).  Products of codes and scales are exact, sums are the tensor core's binary32.
//
// Operands come by TMA in rows of 128 bytes (256 columns) with the 128-byte swizzle, scales as they stand in memory: their tiles of
// 128 rows x 4 blocks are what tcgen05.cp spreads over tensor memory (32 lanes of four words, the same for every quarter of the lanes), from where
// the MMA takes them.  Two forms: pairs of SMs, and up to a few tiles a CTA with K shared out.
#include "fp4.cuh"
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

// Instruction descriptor: e2m1 operands, K-major; scales e4m3 (blocks of 16) or e8m0 (32), whose byte of the word `id` names
__host__ __device__ constexpr uint32_t idesc_fp4(int M, int N, int block, int id) {
  return (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | (block == 32 ? 1u << 23 : 0u) | ((uint32_t)(M >> 4) << 24) |
         ((uint32_t)id << 4) | ((uint32_t)id << 29);
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

// The MMAs of a stage (up to four steps of 64 columns), by one thread.  ts: columns for scales, 4 for each tile of a's and of b's.
// Copies and MMAs of one thread are carried out in their order, so a tile's columns are free when the next stage's copies come.
template <int CTAS, int BLOCK>
__device__ __forceinline__ void issue_stage(uint32_t acc, uint32_t ts, uint32_t a, uint32_t b, uint32_t sa, uint32_t sb, int bgroups, int steps, int M, int N,
                                            bool first) {
  typedef Scales<BLOCK> S;
  const uint64_t da = tile_desc(a, ROW), db = tile_desc(b, ROW);
#pragma unroll
  for (int tile = 0; tile < S::kTiles; ++tile) {
    if (tile * BLOCK < 16 * steps) {
      const uint32_t ca = ts + 4 * tile, cb = ts + 4 * S::kTiles + 4 * bgroups * tile;
      scales_in<CTAS>(ca, sa + tile * kTileBytes);
      scales_in<CTAS>(cb, sb + tile * kTileBytes);
      if (bgroups == 2) scales_in<CTAS>(cb + 4, sb + S::kBytes + tile * kTileBytes);
    }
  }
#pragma unroll
  for (int k = 0; k < BK / 64; ++k) {
    if (k < steps) {
      const int tile = BLOCK == 16 ? k : k >> 1, id = BLOCK == 16 ? 0 : 2 * (k & 1);
      const uint32_t ca = ts + 4 * tile, cb = ts + 4 * S::kTiles + 4 * bgroups * tile;
      mma_fp4<CTAS, BLOCK>(acc, da + 2 * k, db + 2 * k, idesc_fp4(M, N, BLOCK, id), ca, cb, !first || k > 0);
    }
  }
}

// ------------------------------------------------------------------------------------------------ pairs of SMs
// Tiles of 256 x 256 for two SMs (cta_group::2), persistent: each CTA of a pair loads 128 rows of x, 128 of w and the scales of its rows of x and of all
// 256 of w, the first one issues the MMAs, and each drains its 128 rows of the accumulator while the next tile's is formed.  Two accumulators
// of 256 columns would be all of tensor memory: they share 48 columns, which the scales take at its end, and an epilogue reads
// the shared ones first.
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

// One epilogue warp: a quarter's 32 rows (lanes) of 128 columns of an accumulator.  It works in units of 128 bytes of out's rows (64 columns, or 32 of
// binary32), whose residual is on its way while the unit before is finished, and leaves them in one of its two slabs in shared memory.  Where out's rows
// (and the residual's) lie on 16-byte boundaries a slab goes out by TMA, which leaves out what is beyond the last row and column.  Other
// rows are read back from it as binary32, a row at a time by lanes that stand beside one another in it, and stored in words of four bytes: in
// an odd row, one of 16-bit elements that starts in the middle of a word, lane j has elements 2 j + 1 and 2 j + 2, and the last lane both ends.
template <typename T>
struct Epilogue {
  static constexpr int U = 128 / sizeof(T);   // columns of a unit
  typedef typename std::conditional<sizeof(T) == 4, uint32_t, uint16_t>::type Bits;

  const Fp4Params& p;
  const CUtensorMap* tout;
  uint8_t* slab;
  const int lane;
  const bool vectors;
  int slot = 0;
  int t0, n0, end;       // the tile's first row of the warp, its first column, where its columns end
  float sr;
  uint32_t res[32];      // residual of a unit: this lane's row, or its word (two words' halves) of each of 32 rows

  __device__ __forceinline__ Epilogue(const Fp4Params& p_, const CUtensorMap* tout_, uint8_t* slab_)
      : p(p_), tout(tout_), slab(slab_), lane(threadIdx.x & 31), vectors(p_.vec_out && (!p_.residual || p_.vec_res)) {}

  static __device__ __forceinline__ int odd_row(const void* q) { return (int)(reinterpret_cast<uintptr_t>(q) >> 1 & 1); }
  // the residual of a tile into L2, ahead of its turn
  __device__ __forceinline__ void prefetch(int t_first, int n_first) const {
    const int t = t_first + lane;
    if (!p.residual || t >= p.T || n_first >= p.O) return;
    const uint8_t* const at = reinterpret_cast<const uint8_t*>(static_cast<const T*>(p.residual) + t * p.res_stride + n_first);
    const int bytes = min(128, p.O - n_first) * (int)sizeof(T);
    for (int o = 0; o < bytes; o += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(at + o));
    asm volatile("prefetch.global.L2 [%0];" ::"l"(at + bytes - 1));
  }
  __device__ __forceinline__ void tile(int t_first, int n_first) {
    t0 = t_first;
    n0 = n_first;
    end = min(n0 + 128, p.O);
    sr = t0 + lane < p.T ? (p.s_row ? p.s_row[t0 + lane] : 1.0f) : 0.f;
  }
  __device__ __forceinline__ void fetch(int c0) {
    const int o0 = n0 + c0;
    if (!p.residual || o0 >= end) return;
    const T* const residual = static_cast<const T*>(p.residual);
    if (vectors) {
      if (t0 + lane >= p.T) return;
      const T* const at = residual + (t0 + lane) * p.res_stride + o0;
      if (o0 + U <= end) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint4 q = reinterpret_cast<const uint4*>(at)[i];
          res[4 * i] = q.x; res[4 * i + 1] = q.y; res[4 * i + 2] = q.z; res[4 * i + 3] = q.w;
        }
      } else {
        const Bits* const e = reinterpret_cast<const Bits*>(at);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          constexpr int n = 4 / (int)sizeof(T);
          uint32_t w = o0 + n * i < end ? (uint32_t)e[n * i] : 0u;
          if (n == 2 && o0 + 2 * i + 1 < end) w |= (uint32_t)e[2 * i + 1] << 16;
          res[i] = w;
        }
      }
      return;
    }
    const Bits* at = reinterpret_cast<const Bits*>(residual) + t0 * p.res_stride + o0;
    const T* to = static_cast<const T*>(p.out) + t0 * p.out_stride + o0;
    const int rows = min(32, p.T - t0);
#pragma unroll
    for (int r = 0; r < 32; ++r, at += p.res_stride, to += p.out_stride) {
      if (r >= rows) break;
      if constexpr (sizeof(T) == 4) {
        if (o0 + lane < end) res[r] = at[lane];
      } else {
        const int odd = odd_row(to), a = 2 * lane + odd, b = (a + 1) & 63;
        if (odd_row(at + odd) == 0 && b > a && o0 + b < end) res[r] = *reinterpret_cast<const uint32_t*>(at + a);
        else res[r] = (o0 + a < end ? (uint32_t)at[a] : 0u) | (o0 + b < end ? (uint32_t)at[b] << 16 : 0u);
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
  __device__ __forceinline__ void into(float2 (&f)[16], int half) {
    if (vectors) {   // 16-byte chunks of a row of 128 bytes, as the 128-byte swizzle has them
      uint8_t* const to = slab + slot * 4096;
      if (p.residual) {
#pragma unroll
        for (int c = 0; c < 16; ++c) {
          if constexpr (sizeof(T) == 4) {
            f[c] = __fadd2_rn(f[c], make_float2(__uint_as_float(res[2 * c]), __uint_as_float(res[2 * c + 1])));
          } else {
            const T* const r = reinterpret_cast<const T*>(&res[16 * half + c]);
            f[c] = __fadd2_rn(f[c], make_float2(Elem<T>::get(r[0]), Elem<T>::get(r[1])));
          }
        }
      }
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *reinterpret_cast<uint4*>(to + swz_off(lane, i, 128)) = make_uint4(__float_as_uint(f[2 * i].x), __float_as_uint(f[2 * i].y),
                                                                              __float_as_uint(f[2 * i + 1].x), __float_as_uint(f[2 * i + 1].y));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint2 a = Elem<T>::pack(make_float4(f[4 * i].x, f[4 * i].y, f[4 * i + 1].x, f[4 * i + 1].y));
          const uint2 b = Elem<T>::pack(make_float4(f[4 * i + 2].x, f[4 * i + 2].y, f[4 * i + 3].x, f[4 * i + 3].y));
          *reinterpret_cast<uint4*>(to + swz_off(lane, 4 * half + i, 128)) = make_uint4(a.x, a.y, b.x, b.y);
        }
      }
    } else {   // pairs of columns, at a place that depends on the row: no two lanes of a row or of a column meet in a bank
      constexpr int pairs = U / 2;
      float2* const to = reinterpret_cast<float2*>(slab) + lane * pairs;
#pragma unroll
      for (int c = 0; c < 16; ++c) to[(16 * half + c) ^ (lane & (pairs - 1))] = f[c];
    }
  }
  __device__ __forceinline__ void take() {   // the slab's last store has been read
    if (vectors) {
      if (lane == 0) tma_store_wait_read_but_one();
      __syncwarp();
    }
  }
  __device__ __forceinline__ void leave(int c0) {
    const int o0 = n0 + c0;
    if (vectors) {
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        if (o0 < end && t0 < p.T) tma_store_2d(tout, slab + slot * 4096, o0, t0);
        tma_store_commit();
      }
      slot ^= 1;
      return;
    }
    __syncwarp();
    if (o0 < end) {
      constexpr int pairs = U / 2;
      const float* const turn = reinterpret_cast<const float*>(slab);
      T* at = static_cast<T*>(p.out) + t0 * p.out_stride + o0;
      const int rows = min(32, p.T - t0);
      auto column = [&](int r, int c) { return turn[r * U + (((c >> 1) ^ (r & (pairs - 1))) << 1) + (c & 1)]; };
#pragma unroll
      for (int r = 0; r < 32; ++r, at += p.out_stride) {
        if (r >= rows) break;
        if constexpr (sizeof(T) == 4) {
          const float x = column(r, lane);
          if (o0 + lane < end) at[lane] = p.residual ? x + __uint_as_float(res[r]) : x;
        } else {
          const int odd = odd_row(at), a = 2 * lane + odd, b = (a + 1) & 63;
          float2 x;
          if (odd) x = make_float2(column(r, a), column(r, b));
          else x = reinterpret_cast<const float2*>(turn)[r * pairs + (lane ^ r)];
          if (p.residual) {
            const T* const m = reinterpret_cast<const T*>(&res[r]);
            x = __fadd2_rn(x, make_float2(Elem<T>::get(m[0]), Elem<T>::get(m[1])));
          }
          const uint32_t w = Elem<T>::pack(make_float4(x.x, x.y, 0.f, 0.f)).x;
          if (b > a && o0 + b < end) {
            *reinterpret_cast<uint32_t*>(at + a) = w;
          } else {
            if (o0 + a < end) reinterpret_cast<uint16_t*>(at)[a] = (uint16_t)w;
            if (o0 + b < end) reinterpret_cast<uint16_t*>(at)[b] = (uint16_t)(w >> 16);
          }
        }
      }
    }
    __syncwarp();
  }
  // all 128 columns, the halves from the first or from the last on (down); `ready` waits for the accumulator, `drained` is called once the first half is
  // in registers
  template <typename R, typename F>
  __device__ __forceinline__ void run(uint32_t tmem, bool down, const float* cw, const float* cb, R ready, F drained) {
    int c0 = down ? 64 : 0;
    fetch(c0);
    ready();
#pragma unroll 1
    for (int i = 0; i < 2; ++i, c0 ^= 64) {
      int v[32], u[32];
      tmem_ld32(tmem + c0, v);
      tmem_ld32(tmem + c0 + 32, u);
      tmem_ld_wait();
      if (i == 0) {
        tc_fence_before();
        drained();
      }
      float2 f[16];
      take();
      values(v, cw + c0, cb + c0, f);
      into(f, 0);
      if constexpr (sizeof(T) == 4) {
        leave(c0);
        fetch(c0 + 32);
        take();
      }
      values(u, cw + c0 + 32, cb + c0 + 32, f);
      into(f, sizeof(T) == 4 ? 0 : 1);
      leave(sizeof(T) == 4 ? c0 + 32 : c0);
      if (i == 0) fetch(c0 ^ 64);
    }
  }
};

template <typename T, int BLOCK>
__global__ void __launch_bounds__(PT, 1) fp4_pair_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ CUtensorMap tw,
                                                         const __grid_constant__ CUtensorMap tsx, const __grid_constant__ CUtensorMap tsw,
                                                         const __grid_constant__ CUtensorMap tout, const __grid_constant__ Fp4Params p) {
  typedef PairLayout S;
  constexpr uint32_t kSc = Scales<BLOCK>::kBytes;
  extern __shared__ __align__(1024) uint8_t smem[];   // (there is no static part: the window's base is on 1024 bytes)
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kBars);   // (waited for in the first CTA; the second's loads arrive there too)
  uint64_t* empty = full + S::kStages;
  uint64_t* acc_full = empty + S::kStages;
  uint64_t* acc_free = acc_full + 2;                               // (waited for in the first CTA)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_free + 2);
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
    fence_mbar_init();
    tma_prefetch_desc(&tx);
    tma_prefetch_desc(&tw);
    tma_prefetch_desc(&tsx);
    tma_prefetch_desc(&tsw);
    tma_prefetch_desc(&tout);
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
          issue_stage<2, BLOCK>(tmem + buf * (PBN - kShared), tmem + 2 * PBN - kShared, a, a + S::kA, a + S::kScales, a + S::kScales + kSc, 2,
                                p.steps - kb * (BK / 64), 256, PBN, kb == 0);
          pair_commit(&empty[s]);
          if (kb + 1 == p.kblocks) pair_commit(&acc_full[buf]);
        }
        __syncwarp();
      }
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3, upper = (warp - 4) >> 2, et = tid & 127;   // eight warps: a quarter of the rows, half of the columns
    Epilogue<T> ep(p, &tout, smem + S::kSlabs + (warp - 4) * 2 * 4096);
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
    ep.prefetch(m * 256 + rank * 128 + quarter * 32, n * PBN + upper * 128);
    for (int tile = pair; tile < ntotal; tile += npairs, ++at) {
      const int buf = at & 1;
      float* const cw = cols + (buf * 2 + upper) * 256;
      cw[et] = w;
      cw[128 + et] = b;
      ep.tile(m * 256 + rank * 128 + quarter * 32, n * PBN + upper * 128);
      if (tile + npairs < ntotal) {
        tile_of<8>(tile + npairs, p.mtiles, p.ntiles, &m, &n);
        column(n);
        ep.prefetch(m * 256 + rank * 128 + quarter * 32, n * PBN + upper * 128);
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
// The weight's rows are the accumulator's 128 lanes and up to 256 tokens its columns, and K is shared out among the CTAs of a cluster until the SMs
// are all at it.  The parts of a tile meet in shared memory, added in the order of their CTAs, each CTA finishing some tokens.
constexpr int FT = 256;
struct FewLayout {
  static constexpr int kMaxStages = 5;
  static constexpr uint32_t kW = 128 * ROW;
  static constexpr uint32_t kSmall = 101376, kLarge = 221184;    // the ring, two CTAs on an SM or one; the accumulator's image of [n][128] goes over it
  static constexpr uint32_t kTail = 256 + 1024;                  // barriers; the tiles start on 1024 bytes
};
static_assert(2 * (FewLayout::kSmall + FewLayout::kTail + 1024) <= 233472 && FewLayout::kLarge + FewLayout::kTail <= 232448, "");
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
  const uint32_t tmem = warp == 0 ? 0u : allocated<1>(tmem_slot, f.columns, warp, FT);
  // CTAs of a cluster, then the tiles of tokens, then those of the weight (which their CTAs share in L2)
  const int rank = blockIdx.x % f.split, tile = blockIdx.x / f.split, m = tile / p.ntiles, n = tile % p.ntiles;
  const int o0 = m * 128, tok0 = n * f.n, ntok = min(f.n, p.T - tok0);
  const int kb0 = (int)((i64)p.kblocks * rank / f.split), kb1 = (int)((i64)p.kblocks * (rank + 1) / f.split);
  // a warp per token in the end, four outputs per lane
  const int o = o0 + 4 * lane, no = min(p.O - o, 4), step = f.split * (FT / 32);
  float sw[4], bias[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    sw[e] = e < no ? (p.s_w ? p.s_w[o + e] : 1.0f) : 0.f;
    bias[e] = e < no && p.bias ? p.bias[o + e] : 0.f;
  }
  // (n % 16 = 0: codes and scales start on 1024 bytes)
  const uint32_t scales = S::kW + f.n * ROW, stage = (scales + (1 + f.bgroups) * kSc + 1023) & ~1023u;
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
    int s = 0, round = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      mbar_wait(&full[s], round & 1, p.status);
      tc_fence_after();
      if (elect_one()) {
        const uint32_t a = smem_u32(smem + s * stage);
        issue_stage<1, BLOCK>(tmem, tmem + f.n, a, a + S::kW, a + scales, a + scales + kSc, f.bgroups, p.steps - kb * (BK / 64), 128, f.n, kb == kb0);
        mma_commit(&empty[s]);
        if (kb + 1 == kb1) mma_commit(acc_full);
      }
      __syncwarp();
      if (++s == f.stages) { s = 0; ++round; }
    }
  }
  float* const part = reinterpret_cast<float*>(smem);   // [n][128]
  if (warp >= 4) {
    // the accumulator over the ring: every load has been consumed by an MMA that is complete
    const int quarter = warp & 3;
    mbar_wait(acc_full, 0, p.status);
    tc_fence_after();
    for (int c0 = 0; c0 < f.n; c0 += 16) {
      int v[16];
      tmem_ld8(tmem + ((uint32_t)(quarter * 32) << 16) + c0, reinterpret_cast<int(&)[8]>(v[0]));
      tmem_ld8(tmem + ((uint32_t)(quarter * 32) << 16) + c0 + 8, reinterpret_cast<int(&)[8]>(v[8]));
      tmem_ld_wait();
#pragma unroll
      for (int c = 0; c < 16; ++c) part[(c0 + c) * 128 + quarter * 32 + lane] = __int_as_float(v[c]);
    }
    tc_fence_before();
  }
  __syncthreads();
  if (f.split > 1) cluster_sync();
  // (the parts of four tokens on their way at a time)
  for (int t0 = rank + f.split * warp; t0 < ntok; t0 += 4 * step) {
    float4 acc[4];
    float srs[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      acc[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      srs[u] = p.s_row && t0 + u * step < ntok ? p.s_row[tok0 + t0 + u * step] : 1.0f;
    }
    for (int r = 0; r < f.split; ++r)
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (t0 + u * step < ntok) {
          const float* const at = part + (t0 + u * step) * 128 + 4 * lane;
          const float4 v = f.split == 1 ? *reinterpret_cast<const float4*>(at) : ld_from(at, r);
          acc[u] = make_float4(acc[u].x + v.x, acc[u].y + v.y, acc[u].z + v.z, acc[u].w + v.w);
        }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (t0 + u * step >= ntok || no <= 0) continue;
      const i64 t = tok0 + t0 + u * step;
      const float a4[4] = {acc[u].x, acc[u].y, acc[u].z, acc[u].w};
      const T* const res = p.residual ? static_cast<const T*>(p.residual) + t * p.res_stride + o : nullptr;
      T* const dst = static_cast<T*>(p.out) + t * p.out_stride + o;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = activate(fmaf(a4[e] * srs[u], sw[e], bias[e]), p.act);
      if (no == 4 && p.vec_out && (!res || p.vec_res)) {
        if (res) {
          const float4 q = Elem<T>::cvt(*reinterpret_cast<const typename Elem<T>::raw4*>(res));
          v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w;
        }
        *reinterpret_cast<typename Elem<T>::raw4*>(dst) = Elem<T>::pack(make_float4(v[0], v[1], v[2], v[3]));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < no) dst[e] = Elem<T>::put(res ? v[e] + Elem<T>::get(res[e]) : v[e]);
      }
    }
  }
  drain_after_timeout(p.status);
  if (f.split > 1) cluster_sync();   // (the others have read this CTA's part)
  else __syncthreads();
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, f.columns);
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
  // What is done sooner, in cycles: an SM takes 60 bytes of operands a cycle.
  const i64 mt = (w.rows + 127ll) / 128;
  FewParams f = {};
  double best = 0.0;
  for (int n = x.rows <= 256 ? (x.rows + 15) / 16 * 16 : 128; n <= 256; n += x.rows <= 256 ? 256 : 128) {
    const i64 tiles = mt * ((x.rows + n - 1ll) / n);
    const int per_sm = n <= 128 ? 2 : 1;
    const double bytes = FewLayout::kW + n * ROW + (n <= 128 ? 2 : 3) * (double)Scales<BLOCK>::kBytes;
    for (int split = 1; split <= 8 && split <= p.kblocks; split *= 2) {
      const double waves = (double)((tiles * split + sms * per_sm - 1) / (sms * per_sm)), share = tiles * split < sms ? 1.0 : (double)per_sm;
      const double cycles = waves * (share * ((p.kblocks + split - 1) / split * bytes / 60.0 + n * 8.0) + 3000.0 + (split > 1 ? 1000.0 : 0.0));
      if (best == 0.0 || cycles < best) {
        best = cycles;
        f.n = n;
        f.split = split;
      }
    }
  }
  const i64 ptiles = (i64)((x.rows + 255ll) / 256) * ((w.rows + PBN - 1ll) / PBN), pairs = sms / 2;
  const bool pair = pairs > 0 && (double)((ptiles + pairs - 1) / pairs) * (650.0 * p.kblocks + 800.0) + 5000.0 < best;
  if (pair) {
    if (ptiles > 0x3fffffff) return SSDI8_ERR_SHAPE;
    p.mtiles = (int)((x.rows + 255ll) / 256);
    p.ntiles = (int)((w.rows + PBN - 1ll) / PBN);
    if (!codes(&tx, x, 128) || !codes(&tw, w, 128)) return SSDI8_ERR_CUDA;
    CUtensorMap tout = tx;   // (where out's rows are not on 16 bytes it is not used)
    const uint64_t dims[2] = {(uint64_t)p.O, (uint64_t)p.T}, stride[1] = {(uint64_t)(a.stride_out * e)};
    const uint32_t box[2] = {(uint32_t)(128 / e), 32};
    if (p.vec_out && !encode_tensor_map(&tout, a.out, (int)e, 2, dims, stride, box, 128)) p.vec_out = 0;
    return launch_any(fp4_pair_kernel<T, BLOCK>, dim3((unsigned)(2 * (ptiles < pairs ? ptiles : pairs))), 2, dim3(PT), PairLayout::kAlloc, PairLayout::kAlloc,
                      -1, true, st, tx, tw, tsx, tsw, tout, p);
  }
  f.l = p;
  f.l.mtiles = (int)mt;
  f.l.ntiles = (int)((x.rows + f.n - 1ll) / f.n);
  f.bgroups = f.n <= 128 ? 1 : 2;
  f.ring = f.n <= 128 ? FewLayout::kSmall : FewLayout::kLarge;
  const int need = f.n + 4 * Scales<BLOCK>::kTiles * (1 + f.bgroups);
  f.columns = need <= 64 ? 64 : need <= 128 ? 128 : need <= 256 ? 256 : 512;
  const uint32_t stage = (FewLayout::kW + f.n * ROW + (1 + f.bgroups) * Scales<BLOCK>::kBytes + 1023) & ~1023u;
  const int stages = (int)(f.ring / stage);
  f.stages = stages < FewLayout::kMaxStages ? stages : FewLayout::kMaxStages;
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
