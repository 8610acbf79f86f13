// Int8 projection: out = act(s_row s_w (xq wq^T) + bias) + residual, on tcgen05.mma.kind::i8 with int32 accumulators in tensor memory
// (the integer sums are exact) and everything behind them in the epilogue.  Persistent: a loading warp (TMA, both operands K-major in
// rows of 128 bytes with the 128-byte swizzle), an issuing warp, and four epilogue warps that drain one accumulator while the
// next tile's is formed in the other.
#include "block.cuh"
#include "kernels.h"
#include "sm100.cuh"

namespace ssdi8 {
namespace {

using namespace sm100;

constexpr int LT = 256;      // threads: loader, issuer, tensor-memory allocator, one idle, four epilogue warps
constexpr int BM = 128, BK = 128;

struct LinearParams {
  const float *s_row, *s_w, *bias;
  const void* residual; i64 res_stride;
  void* out; i64 out_stride;
  int32_t* status;
  int T, O, kblocks, mtiles, ntiles, act, vec_out, vec_res;
};

template <int BN>
struct Layout {
  static constexpr int kStages = BN == 256 ? 4 : 6;
  static constexpr uint32_t kA = BM * BK, kStage = kA + BN * BK;
  static constexpr uint32_t kBars = kStages * kStage;
  static constexpr uint32_t kCols = kBars + 256;                 // s_w and bias of two tiles' columns
  static constexpr uint32_t kBytes = kCols + 2 * 2 * BN * 4;
  static constexpr uint32_t kAlloc = kBytes + 1024;              // (the tiles start on 1024 bytes)
};

__device__ __forceinline__ float activate(float v, int act) {
  if (act == SSDI8_ACT_SILU) return v * rcp_approx(1.0f + ex2_approx(v * -1.44269504f));
  if (act == SSDI8_ACT_RELU2) return v > 0.f ? v * v : 0.f * v;   // (a NaN stays one)
  return v;
}

// tile -> (row block, column block): eight row blocks at a time, so that the tiles in flight share rows of x and of w in L2
__device__ __forceinline__ void tile_of(int tile, int mtiles, int ntiles, int* m, int* n) {
  const int per = 8 * ntiles, group = tile / per, rest = tile % per;
  const int rows = min(8, mtiles - group * 8);
  *m = group * 8 + rest % rows;
  *n = rest / rows;
}

template <typename T, int BN>
__global__ void __launch_bounds__(LT, 1) linear_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ CUtensorMap tw,
                                                       const __grid_constant__ LinearParams p) {
  typedef Layout<BN> S;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kBars);
  uint64_t* empty = full + S::kStages;
  uint64_t* acc_full = empty + S::kStages;
  uint64_t* acc_empty = acc_full + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
  float* cols = reinterpret_cast<float*>(smem + S::kCols);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < S::kStages; ++i) {
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
  if (warp == 2) tmem_alloc(tmem_slot, 2 * BN);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_launch_dependents();
  pdl_wait();
  const int ntotal = p.mtiles * p.ntiles;
  if (warp == 0) {
    int it = 0;
    for (int tile = blockIdx.x; tile < ntotal; tile += gridDim.x) {
      int m, n;
      tile_of(tile, p.mtiles, p.ntiles, &m, &n);
      for (int kb = 0; kb < p.kblocks; ++kb, ++it) {
        const int s = it % S::kStages;
        if (it >= S::kStages) mbar_wait(&empty[s], (it / S::kStages - 1) & 1, p.status);
        if (elect_one()) {
          mbar_expect_tx(&full[s], S::kStage);
          tma_load_2d(smem + s * S::kStage, &tx, &full[s], kb * BK, m * BM);
          tma_load_2d(smem + s * S::kStage + S::kA, &tw, &full[s], kb * BK, n * BN);
        }
        __syncwarp();
      }
    }
    // the loads in flight land before the block ends: the issuer has waited for each of them
  } else if (warp == 1) {
    constexpr uint32_t idesc = idesc_s8(BM, BN, 0, 0);
    int it = 0, at = 0;
    for (int tile = blockIdx.x; tile < ntotal; tile += gridDim.x, ++at) {
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
          for (int k = 0; k < BK / 32; ++k) mma_s8_ss(tmem + buf * BN, da + 2 * k, db + 2 * k, idesc, kb > 0 || k > 0);
          mma_commit(&empty[s]);
          if (kb + 1 == p.kblocks) mma_commit(&acc_full[buf]);
        }
        __syncwarp();
      }
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3, et = tid - 128;
    int at = 0;
    for (int tile = blockIdx.x; tile < ntotal; tile += gridDim.x, ++at) {
      const int buf = at & 1;
      int m, n;
      tile_of(tile, p.mtiles, p.ntiles, &m, &n);
      float* cw = cols + buf * 2 * BN;
      float* cb = cw + BN;
      for (int c = et; c < BN; c += 128) {
        const int o = n * BN + c;
        cw[c] = o < p.O ? p.s_w[o] : 0.f;
        cb[c] = o < p.O && p.bias ? p.bias[o] : 0.f;
      }
      const int t = m * BM + quarter * 32 + lane;
      const float sr = t < p.T ? (p.s_row ? p.s_row[t] : 1.0f) : 0.f;
      named_bar_sync(1, 128);   // (and nobody is still reading the columns of the tile before the last)
      mbar_wait(&acc_full[buf], (at >> 1) & 1, p.status);
      tc_fence_after();
      for (int c0 = 0; c0 < BN; c0 += 32) {
        int v[32];
        tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + buf * BN + c0, v);
        tmem_ld_wait();
        if (c0 + 32 == BN) {
          tc_fence_before();
          mbar_arrive(&acc_empty[buf]);
        }
        const int o0 = n * BN + c0;
        if (t >= p.T || o0 >= p.O) continue;
        T* dst = static_cast<T*>(p.out) + t * p.out_stride + o0;
        const T* res = p.residual ? static_cast<const T*>(p.residual) + t * p.res_stride + o0 : nullptr;
        const bool whole = o0 + 32 <= p.O;
        if (whole && p.vec_out && (!res || p.vec_res)) {
#pragma unroll
          for (int c = 0; c < 32; c += 8) {
            constexpr int V = 16 / sizeof(T), NV = 8 / V;   // elements of a 16-byte vector, vectors of eight elements
            float f[8];
            const float4 w0 = *reinterpret_cast<const float4*>(cw + c0 + c), w1 = *reinterpret_cast<const float4*>(cw + c0 + c + 4);
            const float4 b0 = *reinterpret_cast<const float4*>(cb + c0 + c), b1 = *reinterpret_cast<const float4*>(cb + c0 + c + 4);
            const float ws[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w}, bs[8] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = activate(fmaf((float)v[c + e] * sr, ws[e], bs[e]), p.act);
            uint4 raw[NV];
            if (res) {
#pragma unroll
              for (int i = 0; i < NV; ++i) raw[i] = reinterpret_cast<const uint4*>(res + c)[i];
#pragma unroll
              for (int e = 0; e < 8; ++e) f[e] += Elem<T>::get(reinterpret_cast<const T*>(raw)[e]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) reinterpret_cast<T*>(raw)[e] = Elem<T>::put(f[e]);
#pragma unroll
            for (int i = 0; i < NV; ++i) reinterpret_cast<uint4*>(dst + c)[i] = raw[i];
          }
        } else {
#pragma unroll
          for (int c = 0; c < 32; ++c)
            if (o0 + c < p.O) {
              float f = activate(fmaf((float)v[c] * sr, cw[c0 + c], cb[c0 + c]), p.act);
              if (res) f += Elem<T>::get(res[c]);
              dst[c] = Elem<T>::put(f);
            }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  drain_after_timeout(p.status);
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, 2 * BN);
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
  auto go = [&](auto bn, auto t) -> ssdi8_status_t {
    constexpr int BN = decltype(bn)::value;
    using E = decltype(t);
    p.mtiles = (a.rows + BM - 1) / BM;
    p.ntiles = (a.outs + BN - 1) / BN;
    const i64 tiles = (i64)p.mtiles * p.ntiles;
    if (tiles > 0x3fffffff) return SSDI8_ERR_SHAPE;
    CUtensorMap tx, tw;
    const uint64_t dx[2] = {(uint64_t)a.inner, (uint64_t)a.rows}, dw[2] = {(uint64_t)a.inner, (uint64_t)a.outs}, stride[1] = {(uint64_t)a.inner};
    const uint32_t bx[2] = {BK, BM}, bw[2] = {BK, BN};
    if (!encode_tensor_map(&tx, a.xq, 1, 2, dx, stride, bx, 128) || !encode_tensor_map(&tw, a.wq, 1, 2, dw, stride, bw, 128)) return SSDI8_ERR_CUDA;
    const int sms = sm_count();
    if (sms <= 0) return SSDI8_ERR_CUDA;
    return launch_configured(linear_kernel<E, BN>, dim3((unsigned)(tiles < sms ? tiles : sms)), dim3(LT), Layout<BN>::kAlloc, -1, false, st, tx, tw, p);
  };
  // Tiles of 256 columns where they fill the SMs, else of 128.
  auto pick = [&](auto t) -> ssdi8_status_t {
    const i64 wide = (i64)((a.rows + BM - 1) / BM) * ((a.outs + 255) / 256);
    return wide >= sm_count() ? go(std::integral_constant<int, 256>{}, t) : go(std::integral_constant<int, 128>{}, t);
  };
  return dtype == 0 ? pick(float{}) : dtype == 1 ? pick(__half{}) : pick(__nv_bfloat16{});
}

}  // namespace ssdi8
