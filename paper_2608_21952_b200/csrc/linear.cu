// Int8 projection: out = act(s_row s_w (xq wq^T) + bias) + residual, on tcgen05.mma.kind::i8 with int32 accumulators in tensor memory
// (the integer sums are exact) and everything behind them in the epilogue.  Persistent: a loading warp (TMA, both operands K-major in
// rows of 128 bytes with the 128-byte swizzle), an issuing warp, and epilogue warps that drain one accumulator while the
// next tile's is formed in the other.  Three forms: tiles for pairs of SMs where they are done sooner, lone tiles, and up to 128 rows.
//
// What bounds it: 16384 x 2560 x 5120 with bias and residual (95 us at the 4.5 POPS that the pipe reaches on resident operands, 41 us of bytes)
// takes 145 to 153 us on inputs that stay (3.0 POPS; 135 without the residual) and 177 to 186 on inputs that do not, in a row of calls under the power limit: the
// operands' 64 bytes a cycle and SM from L2, which is what an SM's port gives, and the clock.  64 x 10576 x 2560 (28.5 MB, 4.4 us): 9.0 us, 3.4 of them
// operands from L2 at 11 TB/s (the tokens are read by every tile), then the parts' meeting and the epilogue, 2 us each.
// From 129 to about 1000 rows a lone tile walks all of K on as many CTAs as there are tiles: 250 x 4096 x 8192 (5.8 us of bytes) 18.9 us, 250 x 18560 x
// 4096 (13.4) 24, 600 x 2560 x 5120 (3.5) 15.  Rows of out off 16-byte boundaries leave as single elements: 3439 x 16470 x 1232, fp16, residual (39) 284.
#include "block.cuh"
#include "kernels.h"
#include "sm100.cuh"

namespace ssdi8 {
namespace {

using namespace sm100;

constexpr int LT = 256;      // threads: loader, issuer, tensor-memory allocator, one idle, four epilogue warps (pairs of SMs: eight)
constexpr int BM = 128, BK = 128;

struct LinearParams {
  const float *s_row, *s_w, *bias;
  const void* residual; i64 res_stride;
  void* out; i64 out_stride;
  int32_t* status;
  int T, O, kblocks, mtiles, ntiles, act, vec_out, vec_res;
  int bn, stages;   // lone tiles: columns, stages of the ring
};

// Shared memory of a lone tile's CTA: a ring of stages, 128 rows of x and bn rows of w each.
struct Layout {
  static constexpr int kMaxBN = 256, kMaxStages = 10;
  static constexpr uint32_t kA = BM * BK, kRing = 196608;
  static constexpr uint32_t kBars = kRing;
  static constexpr uint32_t kCols = kBars + 256;                 // s_w and bias of two tiles' columns
  static constexpr uint32_t kTurns = kCols + 2 * 2 * kMaxBN * 4;
  static constexpr uint32_t kAlloc = kTurns + 4 * 32 * 17 * 4 + 1024;   // (the tiles start on 1024 bytes)
};

__device__ __forceinline__ float activate(float v, int act) {
  if (act == SSDI8_ACT_SILU) return v * rcp_approx(1.0f + ex2_approx(v * -1.44269504f));
  if (act == SSDI8_ACT_RELU2) return v < 0.f ? 0.f : v * v;   // (-inf is 0, a NaN stays one)
  return v;
}

// Tensor memory for all warps but the loader's, by warp 2.  Behind the wait for the kernel before and ahead of the trigger for the next
// one: a kernel that held some while it waits, or that still had to ask for some when the next one may be scheduled beside it, could
// leave the two waiting for one another.
template <int GROUP>
__device__ __forceinline__ uint32_t allocated(uint32_t* slot, uint32_t columns, int warp, int threads) {
  if (warp == 2) {
    if (GROUP == 1) {
      tmem_alloc(slot, columns);
    } else {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(columns) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    pdl_launch_dependents();
  }
  tc_fence_before();
  named_bar_sync(2, threads - 32);
  tc_fence_after();
  return *slot;
}

// tile -> (row block, column block): GROUP row blocks at a time, so that the tiles in flight share rows of x and of w in L2
template <int GROUP>
__device__ __forceinline__ void tile_of(int tile, int mtiles, int ntiles, int* m, int* n) {
  const int per = GROUP * ntiles, group = tile / per, rest = tile % per;
  const int rows = min(GROUP, mtiles - group * GROUP);
  *m = group * GROUP + rest % rows;
  *n = rest / rows;
}

// A quarter's 32 rows (lanes) of `ncols` columns of an accumulator: t is this lane's row, n0 the first column, cw and cb the
// columns' step sizes and biases; `drained` is called once the last column has been read.  Rows of out (and residual) on 16-byte
// boundaries are written by their lane, 32 columns at a time; others, and a ragged end, go through `turn` (32 x 17 floats of the
// warp's), 16 columns at a time, so that lanes stand beside one another in a row (3439 x 16470 x 1232, fp16, residual: 985 us one by one, 284).
// The residual of 32 columns is on its way while the 32 before it are finished, the first of them while the accumulator is; `ready` waits
// for that.
constexpr int kTurn = 32 * 17;
template <typename T, typename R, typename F>
__device__ __forceinline__ void epilogue(const LinearParams& p, uint32_t tmem, int t, int n0, int ncols, const float* cw, const float* cb, float* turn,
                                         R ready, F drained) {
  typedef typename std::conditional<sizeof(T) == 4, uint32_t, uint16_t>::type Bits;
  constexpr int V = 16 / sizeof(T), NV = 32 / V;   // elements of a 16-byte vector, vectors of 32 elements
  const int end = min(n0 + ncols, p.O), lane = threadIdx.x & 31;
  const float sr = t < p.T ? (p.s_row ? p.s_row[t] : 1.0f) : 0.f;
  const T* const residual = static_cast<const T*>(p.residual);
  T* const out = static_cast<T*>(p.out);
  const bool vectors = p.vec_out && (!residual || p.vec_res);
  uint32_t res[32];   // this lane's 32 elements as 16-byte vectors, or one element of each 16 columns of 16 rows, twice
  auto fetch = [&](int o0) {
    if (!residual || o0 >= end) return;
    if (vectors && o0 + 32 <= end) {
      if (t < p.T) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const uint4 q = reinterpret_cast<const uint4*>(residual + t * p.res_stride + o0)[i];
          res[4 * i] = q.x; res[4 * i + 1] = q.y; res[4 * i + 2] = q.z; res[4 * i + 3] = q.w;
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < 32; ++k) {
        const int tt = t - lane + 2 * (k & 15) + (lane >> 4), o = o0 + (k & 16) + (lane & 15);
        if (tt < p.T && o < end) res[k] = reinterpret_cast<const Bits*>(residual)[tt * p.res_stride + o];
      }
    }
  };
  fetch(n0);
  ready();
#pragma unroll 1
  for (int c0 = 0; c0 < ncols; c0 += 32) {
    int v[32];
    __syncwarp();   // (lanes beyond the last row skip the stores)
    tmem_ld32(tmem + c0, v);
    tmem_ld_wait();
    if (c0 + 32 >= ncols) {
      tc_fence_before();
      drained();
    }
    const int o0 = n0 + c0;
    if (o0 >= end) continue;
    if (vectors && o0 + 32 <= end) {
      uint32_t mine[NV * 4];
#pragma unroll
      for (int i = 0; i < NV * 4; ++i) mine[i] = res[i];
      fetch(o0 + 32);
      if (t < p.T) {
        T* const dst = out + t * p.out_stride + o0;
#pragma unroll
        for (int c = 0; c < 32; c += 8) {
          float f[8];
          const float4 w0 = *reinterpret_cast<const float4*>(cw + c0 + c), w1 = *reinterpret_cast<const float4*>(cw + c0 + c + 4);
          const float4 b0 = *reinterpret_cast<const float4*>(cb + c0 + c), b1 = *reinterpret_cast<const float4*>(cb + c0 + c + 4);
          const float ws[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w}, bs[8] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = activate(fmaf((float)v[c + e] * sr, ws[e], bs[e]), p.act);
          T* const at = reinterpret_cast<T*>(mine) + c;
          if (residual) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += Elem<T>::get(at[e]);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) at[e] = Elem<T>::put(f[e]);
#pragma unroll
          for (int i = 0; i < 8 / V; ++i) {
            const uint32_t* const w = mine + (c / V + i) * 4;
            reinterpret_cast<uint4*>(dst + c)[i] = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
    } else {
      Bits mine[32];
#pragma unroll
      for (int k = 0; k < 32; ++k) mine[k] = (Bits)res[k];
      fetch(o0 + 32);
#pragma unroll
      for (int h = 0; h < 32; h += 16) {
#pragma unroll
        for (int c = 0; c < 16; ++c) turn[lane * 17 + c] = activate(fmaf((float)v[h + c] * sr, cw[c0 + h + c], cb[c0 + h + c]), p.act);
        __syncwarp();
        const int o = o0 + h + (lane & 15);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int row = 2 * i + (lane >> 4), tt = t - lane + row;
          if (tt < p.T && o < end) {
            float f = turn[row * 17 + (lane & 15)];
            if (residual) f += Elem<T>::get(*reinterpret_cast<const T*>(&mine[h + i]));
            out[tt * p.out_stride + o] = Elem<T>::put(f);
          }
        }
        __syncwarp();
      }
    }
  }
}
// step sizes and biases of a tile's columns into shared memory, by the epilogue threads
__device__ __forceinline__ void columns(const LinearParams& p, int n0, int ncols, float* cw, float* cb, int et, int threads) {
  for (int c = et; c < ncols; c += threads) {
    const int o = n0 + c;
    cw[c] = o < p.O ? p.s_w[o] : 0.f;
    cb[c] = o < p.O && p.bias ? p.bias[o] : 0.f;
  }
}

template <typename T>
__global__ void __launch_bounds__(LT, 1) linear_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ CUtensorMap tw,
                                                       const __grid_constant__ LinearParams p) {
  typedef Layout S;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kBars);
  uint64_t* empty = full + S::kMaxStages;
  uint64_t* acc_full = empty + S::kMaxStages;
  uint64_t* acc_empty = acc_full + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
  float* cols = reinterpret_cast<float*>(smem + S::kCols);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < S::kMaxStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], 128);
    }
    fence_mbar_init();
    tma_prefetch_desc(&tx);
    tma_prefetch_desc(&tw);
  }
  __syncthreads();
  pdl_wait();
  const uint32_t tmem = warp == 0 ? 0u : allocated<1>(tmem_slot, 512, warp, LT);
  const int ntotal = p.mtiles * p.ntiles;
  const uint32_t stage = S::kA + p.bn * BK;   // (bn % 16 = 0: the operands start on 1024 bytes)
  if (warp == 0) {
    int s = 0, round = 0;
    for (int tile = blockIdx.x; tile < ntotal; tile += gridDim.x) {
      int m, n;
      tile_of<8>(tile, p.mtiles, p.ntiles, &m, &n);
      for (int kb = 0; kb < p.kblocks; ++kb) {
        if (round > 0) mbar_wait(&empty[s], (round - 1) & 1, p.status);
        if (elect_one()) {
          mbar_expect_tx(&full[s], (uint32_t)(BM + p.bn) * BK);
          tma_load_2d(smem + s * stage, &tx, &full[s], kb * BK, m * BM);
          tma_load_2d(smem + s * stage + S::kA, &tw, &full[s], kb * BK, n * p.bn);
        }
        __syncwarp();
        if (++s == p.stages) { s = 0; ++round; }
      }
    }
    // the loads in flight land before the block ends: the issuer has waited for each of them
  } else if (warp == 1) {
    const uint32_t idesc = idesc_s8(BM, p.bn, 0, 0);
    int s = 0, round = 0, at = 0;
    for (int tile = blockIdx.x; tile < ntotal; tile += gridDim.x, ++at) {
      const int buf = at & 1;
      if (at >= 2) mbar_wait(&acc_empty[buf], ((at >> 1) - 1) & 1, p.status);
      tc_fence_after();
      for (int kb = 0; kb < p.kblocks; ++kb) {
        mbar_wait(&full[s], round & 1, p.status);
        tc_fence_after();
        if (elect_one()) {
          const uint64_t da = tile_desc(smem_u32(smem + s * stage), 128), db = tile_desc(smem_u32(smem + s * stage + S::kA), 128);
#pragma unroll
          for (int k = 0; k < BK / 32; ++k) mma_s8_ss(tmem + buf * S::kMaxBN, da + 2 * k, db + 2 * k, idesc, kb > 0 || k > 0);
          mma_commit(&empty[s]);
          if (kb + 1 == p.kblocks) mma_commit(&acc_full[buf]);
        }
        __syncwarp();
        if (++s == p.stages) { s = 0; ++round; }
      }
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3;
    int at = 0;
    for (int tile = blockIdx.x; tile < ntotal; tile += gridDim.x, ++at) {
      const int buf = at & 1;
      int m, n;
      tile_of<8>(tile, p.mtiles, p.ntiles, &m, &n);
      float* cw = cols + buf * 2 * S::kMaxBN;
      columns(p, n * p.bn, p.bn, cw, cw + S::kMaxBN, tid - 128, 128);
      named_bar_sync(1, 128);   // (and nobody is still reading the columns of the tile before the last)
      epilogue<T>(p, tmem + ((uint32_t)(quarter * 32) << 16) + buf * S::kMaxBN, m * BM + quarter * 32 + lane, n * p.bn, p.bn, cw, cw + S::kMaxBN,
                  reinterpret_cast<float*>(smem + S::kTurns) + quarter * kTurn,
                  [&] { mbar_wait(&acc_full[buf], (at >> 1) & 1, p.status); tc_fence_after(); }, [&] { mbar_arrive(&acc_empty[buf]); });
    }
  }
  tc_fence_before();
  __syncthreads();
  drain_after_timeout(p.status);
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ------------------------------------------------------------------------------------------------ pairs of SMs
// The same on tiles of 256 x 256 for two SMs (cta_group::2): each CTA of a pair loads 128 rows of x and 128 of w, the first one issues the
// MMAs, and each drains its 128 rows of the accumulator.  32 KB per CTA and 128 of K where a lone tile of 128 x 256 takes 48: what the
// operands' way from L2 bounds (16384 x 2560 x 5120: 238 us with lone tiles, 155 with pairs).
constexpr int PBN = 256, PT = 384;
struct PairLayout {
  static constexpr int kStages = 6;
  static constexpr uint32_t kA = BM * BK, kStage = 2 * kA;
  static constexpr uint32_t kBars = kStages * kStage;
  static constexpr uint32_t kCols = kBars + 256;
  static constexpr uint32_t kTurns = kCols + 2 * 2 * PBN * 4;
  static constexpr uint32_t kAlloc = kTurns + 8 * kTurn * 4 + 1024;
};

__device__ __forceinline__ uint32_t in_first(const void* p) {   // the same place in the pair's first CTA
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(smem_u32(p)));
  return a;
}
__device__ __forceinline__ void pair_load(void* dst, const CUtensorMap* tm, uint32_t bar, int x, int y) {   // bar: of the first CTA
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(smem_u32(dst)), "l"(tm), "r"(bar), "r"(x), "r"(y)
               : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
               : "memory");
}
__device__ __forceinline__ void pair_commit(uint64_t* bar) {   // arrives at this place in both CTAs
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(smem_u32(bar)), "h"((uint16_t)3)
               : "memory");
}
__device__ __forceinline__ void arrive_at(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

template <typename T>
__global__ void __launch_bounds__(PT, 1) linear_pair_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ CUtensorMap tw,
                                                            const __grid_constant__ LinearParams p) {
  typedef PairLayout S;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kBars);   // (waited for in the first CTA; the second's loads arrive there too)
  uint64_t* empty = full + S::kStages;
  uint64_t* acc_full = empty + S::kStages;
  uint64_t* acc_empty = acc_full + 2;                              // (waited for in the first CTA)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
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
      mbar_init(&acc_empty[i], 16);   // the epilogue warps of both
    }
    fence_mbar_init();
    tma_prefetch_desc(&tx);
    tma_prefetch_desc(&tw);
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
          if (rank == 0) mbar_expect_tx(&full[s], 2 * S::kStage);
          const uint32_t bar = in_first(&full[s]);
          pair_load(smem + s * S::kStage, &tx, bar, kb * BK, m * 256 + rank * 128);
          pair_load(smem + s * S::kStage + S::kA, &tw, bar, kb * BK, n * PBN + rank * 128);
        }
        __syncwarp();
      }
    }
    // (the last commits have arrived here before this CTA ends)
    for (int k = it > S::kStages ? it - S::kStages : 0; k < it; ++k) mbar_wait(&empty[k % S::kStages], (k / S::kStages) & 1, p.status);
  } else if (warp == 1 && rank == 0) {
    constexpr uint32_t idesc = idesc_s8(256, PBN, 0, 0);
    int it = 0, at = 0;
    for (int tile = pair; tile < ntotal; tile += npairs, ++at) {
      const int buf = at & 1;
      if (at >= 2) mbar_wait(&acc_empty[buf], ((at >> 1) - 1) & 1, p.status);
      tc_fence_after();
      for (int kb = 0; kb < p.kblocks; ++kb, ++it) {
        const int s = it % S::kStages;
        mbar_wait(&full[s], (it / S::kStages) & 1, p.status);
        tc_fence_after();
        if (elect_one()) {
          const uint64_t da = tile_desc(smem_u32(smem + s * S::kStage), 128), db = tile_desc(smem_u32(smem + s * S::kStage + S::kA), 128);
#pragma unroll
          for (int k = 0; k < BK / 32; ++k) pair_mma(tmem + buf * PBN, da + 2 * k, db + 2 * k, idesc, kb > 0 || k > 0);
          pair_commit(&empty[s]);
          if (kb + 1 == p.kblocks) pair_commit(&acc_full[buf]);
        }
        __syncwarp();
      }
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3, half = (warp - 4) >> 2 << 7;   // eight warps: a quarter of the rows, half of the columns
    int at = 0;
    for (int tile = pair; tile < ntotal; tile += npairs, ++at) {
      const int buf = at & 1;
      int m, n;
      tile_of<8>(tile, p.mtiles, p.ntiles, &m, &n);
      float* cw = cols + buf * 2 * PBN;
      columns(p, n * PBN, PBN, cw, cw + PBN, tid - 128, PT - 128);
      named_bar_sync(1, PT - 128);
      epilogue<T>(p, tmem + ((uint32_t)(quarter * 32) << 16) + buf * PBN + half, m * 256 + rank * 128 + quarter * 32 + lane, n * PBN + half, 128, cw + half,
                  cw + PBN + half, reinterpret_cast<float*>(smem + S::kTurns) + (warp - 4) * kTurn,
                  [&] { mbar_wait(&acc_full[buf], (at >> 1) & 1, p.status); tc_fence_after(); }, [&] {
                    __syncwarp();
                    if (lane == 0) arrive_at(in_first(&acc_empty[buf]));
                  });
    }
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
// Up to 128 rows (decode): the weight is what is read, so its rows are the accumulator's 128 lanes and the tokens its columns (a weight row
// costs the tensor pipe a tenth of what 128 mostly empty token rows cost), and K is shared out among the CTAs of a cluster, two on
// an SM, until they are all at it.  The parts of a tile meet in shared memory (int32: in any order the same), each CTA finishing some tokens.
constexpr int FT = 256, kFewRows = 128;
struct FewLayout {
  static constexpr int kMaxStages = 5;
  static constexpr uint32_t kW = 128 * BK, kRing = 102400;       // (the accumulator's image of [128 tokens][128] goes over the ring: 65536)
  static constexpr uint32_t kBars = kRing;
  static constexpr uint32_t kAlloc = kBars + 256 + 1024;
};
struct FewParams {
  LinearParams l;
  int n, split;   // columns of the accumulator (tokens, to 16), CTAs of a cluster
};

__device__ __forceinline__ int4 ld_from(const int* p, int rank) {   // the same place in another CTA of the cluster
  uint32_t a;
  int4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}

template <typename T>
__global__ void __launch_bounds__(FT, 2) linear_few_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ CUtensorMap tw,
                                                           const __grid_constant__ FewParams f) {
  typedef FewLayout S;
  const LinearParams& p = f.l;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kBars);
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
  }
  __syncthreads();
  pdl_wait();
  const uint32_t tmem = warp == 0 ? 0u : allocated<1>(tmem_slot, 128, warp, FT);
  const int rank = blockIdx.x % f.split, o0 = blockIdx.x / f.split * 128;
  const int kb0 = p.kblocks * rank / f.split, kb1 = p.kblocks * (rank + 1) / f.split;
  // a warp per token in the end, four outputs per lane
  const int o = o0 + 4 * lane, no = min(p.O - o, 4), step = f.split * (FT / 32);
  float sw[4], bias[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    sw[e] = e < no ? p.s_w[o + e] : 0.f;
    bias[e] = e < no && p.bias ? p.bias[o + e] : 0.f;
  }
  const uint32_t stage = S::kW + f.n * BK;   // (n % 16 = 0: the operands start on 1024 bytes)
  if (warp == 0) {
    int s = 0, round = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (round > 0) mbar_wait(&empty[s], (round - 1) & 1, p.status);
      if (elect_one()) {
        mbar_expect_tx(&full[s], stage);
        tma_load_2d(smem + s * stage, &tw, &full[s], kb * BK, o0);
        tma_load_2d(smem + s * stage + S::kW, &tx, &full[s], kb * BK, 0);
      }
      __syncwarp();
      if (++s == p.stages) { s = 0; ++round; }
    }
  } else if (warp == 1) {
    const uint32_t idesc = idesc_s8(128, f.n, 0, 0);
    int s = 0, round = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      mbar_wait(&full[s], round & 1, p.status);
      tc_fence_after();
      if (elect_one()) {
        const uint64_t da = tile_desc(smem_u32(smem + s * stage), 128), db = tile_desc(smem_u32(smem + s * stage + S::kW), 128);
#pragma unroll
        for (int k = 0; k < BK / 32; ++k) mma_s8_ss(tmem, da + 2 * k, db + 2 * k, idesc, kb > kb0 || k > 0);
        mma_commit(&empty[s]);
        if (kb + 1 == kb1) mma_commit(acc_full);
      }
      __syncwarp();
      if (++s == p.stages) { s = 0; ++round; }
    }
  }
  int* const part = reinterpret_cast<int*>(smem);   // [n][128]
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
      for (int c = 0; c < 16; ++c) part[(c0 + c) * 128 + quarter * 32 + lane] = v[c];
    }
    tc_fence_before();
  }
  __syncthreads();
  if (f.split > 1) cluster_sync();
  {
    // (the parts of four tokens on their way at a time)
    for (int t0 = rank + f.split * warp; t0 < p.T; t0 += 4 * step) {
      int4 acc[4];
      float srs[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        acc[u] = make_int4(0, 0, 0, 0);
        srs[u] = p.s_row && t0 + u * step < p.T ? p.s_row[t0 + u * step] : 1.0f;
      }
      for (int r = 0; r < f.split; ++r)
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (t0 + u * step < p.T) {
            const int* const at = part + (t0 + u * step) * 128 + 4 * lane;
            const int4 v = f.split == 1 ? *reinterpret_cast<const int4*>(at) : ld_from(at, r);
            acc[u] = make_int4(acc[u].x + v.x, acc[u].y + v.y, acc[u].z + v.z, acc[u].w + v.w);
          }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int t = t0 + u * step;
        if (t >= p.T || no <= 0) continue;
        const int a4[4] = {acc[u].x, acc[u].y, acc[u].z, acc[u].w};
        const T* const res = p.residual ? static_cast<const T*>(p.residual) + t * p.res_stride + o : nullptr;
        T* const dst = static_cast<T*>(p.out) + t * p.out_stride + o;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = activate(fmaf((float)a4[e] * srs[u], sw[e], bias[e]), p.act);
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
  }
  drain_after_timeout(p.status);
  if (f.split > 1) cluster_sync();   // (the others have read this CTA's part)
  else __syncthreads();
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, 128);
  }
}

}  // namespace

ssdi8_status_t launch_linear(const ssdi8_linear_args_t& a, int dtype, cudaStream_t st) {
  const size_t e = dtype == 0 ? 4 : 2;
  LinearParams p = {};
  p.s_row = a.s_row; p.s_w = a.s_w; p.bias = a.bias;
  p.residual = a.residual; p.res_stride = a.stride_residual; p.out = a.out; p.out_stride = a.stride_out;
  p.status = a.status;
  p.T = a.rows; p.O = a.outs; p.act = a.act;
  p.kblocks = (a.inner + BK - 1) / BK;
  auto vec = [e](const void* q, i64 stride) { return reinterpret_cast<uintptr_t>(q) % 16 == 0 && stride * (i64)e % 16 == 0; };
  p.vec_out = vec(a.out, a.stride_out);
  p.vec_res = vec(a.residual, a.stride_residual);
  const int sms = sm_count();
  if (sms <= 0) return SSDI8_ERR_CUDA;
  auto maps = [&](CUtensorMap* tx, uint32_t xrows, CUtensorMap* tw, uint32_t wrows) {
    const uint64_t dx[2] = {(uint64_t)a.inner, (uint64_t)a.rows}, dw[2] = {(uint64_t)a.inner, (uint64_t)a.outs}, stride[1] = {(uint64_t)a.inner};
    const uint32_t bx[2] = {BK, xrows}, bw[2] = {BK, wrows};
    return encode_tensor_map(tx, a.xq, 1, 2, dx, stride, bx, 128) && encode_tensor_map(tw, a.wq, 1, 2, dw, stride, bw, 128);
  };
  if (a.rows <= kFewRows) {
    FewParams f = {p, (a.rows + 15) / 16 * 16, 1};
    const i64 tiles = ((i64)a.outs + 127) / 128;
    // (a part has at least four blocks of K)
    while (f.split < 8 && tiles * f.split * 2 <= 2 * sms && p.kblocks >= 8 * f.split) f.split *= 2;
    if (tiles * f.split > 0x7fffffff) return SSDI8_ERR_SHAPE;
    const int stages = (int)(FewLayout::kRing / (FewLayout::kW + f.n * BK));
    f.l.stages = stages < FewLayout::kMaxStages ? stages : FewLayout::kMaxStages;
    CUtensorMap tx, tw;
    if (!maps(&tx, f.n, &tw, 128)) return SSDI8_ERR_CUDA;
    auto go = [&](auto kernel) {
      return launch_any(kernel, dim3((unsigned)(tiles * f.split)), f.split, dim3(FT), FewLayout::kAlloc, FewLayout::kAlloc, -1, false, st, tx, tw, f);
    };
    return dtype == 0 ? go(linear_few_kernel<float>) : dtype == 1 ? go(linear_few_kernel<__half>) : go(linear_few_kernel<__nv_bfloat16>);
  }
  // Lone tiles of 128 x bn or, on pairs of SMs, of 256 x 256: what is done sooner, by waves of tiles and cycles per tile (128 of K
  // take the tensor pipe 2 bn cycles of a lone tile, their operands 2 (128 + bn) on the SM's way from L2; a pair's 512 take about 640).
  // bn is a multiple of 32.
  const i64 mt = (a.rows + BM - 1) / BM;
  double best = 0.0;
  for (int bn = 32; bn <= Layout::kMaxBN; bn += 32) {
    const i64 tiles = mt * ((a.outs + bn - 1) / bn);
    const double cycles = (double)((tiles + sms - 1) / sms) * ((double)p.kblocks * 2.0 * (BM + bn) + 1500.0 + 12.0 * bn);
    if (best == 0.0 || cycles < best) {
      best = cycles;
      p.bn = bn;
    }
  }
  const i64 ptiles = (i64)((a.rows + 255) / 256) * ((a.outs + PBN - 1) / PBN), pairs = sms / 2;
  const bool pair = pairs > 0 && (double)((ptiles + pairs - 1) / pairs) * (640.0 * p.kblocks + 4500.0) < best;
  const i64 tiles = pair ? ptiles : mt * ((a.outs + p.bn - 1) / p.bn);
  if (tiles > 0x3fffffff) return SSDI8_ERR_SHAPE;
  p.mtiles = pair ? (a.rows + 255) / 256 : (int)mt;
  p.ntiles = pair ? (a.outs + PBN - 1) / PBN : (a.outs + p.bn - 1) / p.bn;
  CUtensorMap tx, tw;
  if (!(pair ? maps(&tx, 128, &tw, 128) : maps(&tx, BM, &tw, p.bn))) return SSDI8_ERR_CUDA;
  const int stages = (int)(Layout::kRing / (Layout::kA + p.bn * BK));
  p.stages = stages < Layout::kMaxStages ? stages : Layout::kMaxStages;
  auto go = [&](auto lone, auto paired) -> ssdi8_status_t {
    if (pair)
      return launch_any(paired, dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs))), 2, dim3(PT), PairLayout::kAlloc, PairLayout::kAlloc, -1, false, st, tx,
                        tw, p);
    return launch_configured(lone, dim3((unsigned)(tiles < sms ? tiles : sms)), dim3(LT), Layout::kAlloc, -1, false, st, tx, tw, p);
  };
  return dtype == 0 ? go(linear_kernel<float>, linear_pair_kernel<float>)
       : dtype == 1 ? go(linear_kernel<__half>, linear_pair_kernel<__half>)
                    : go(linear_kernel<__nv_bfloat16>, linear_pair_kernel<__nv_bfloat16>);
}

}  // namespace ssdi8
