// Rows to codes: the residual stream's addition and the RMS norm behind it, h = x + residual, p = h w, ending in int8 codes or in four bits;
// the same without addition and norm (p = x) as the quantiser of matrices in four bits; and the values of such a matrix.
//
// One pass: every thread keeps eight columns of up to four chunks in registers between the row's two reductions (sum of squares in binary64,
// absmax of p; one exchange through shared memory) and the codes.  The norm's factor r never meets a code: it is the same for the row, so it
// goes into the row's step size (with a static step size it does, once per element).  So the sum need not be formed ahead of the codes' arithmetic, and codes
// are functions of p alone.  In binary64 the sum cannot leave its range (a conversion and a fused multiply-add an element, on pipes that nothing else
// uses: 64 cycles for a warp's 256 columns).
//
// What bounds it (device times; in brackets the bytes).  With an fp32 stream the bytes: 16384 x 2560 bf16 to int8 (461 MB, 70 us) 80 us, to four bits (67) 76,
// 4096 x 8192 (56) 61.  With less to move instructions, most of them on the half-rate integer pipe (unpacking, maxima, addresses; 55 % busy): bf16
// stream (45) 56, without one (19) 41, to four bits (41) 61 and (16) 50; the quantiser 137 a warp and 256 columns, 16384 x 5120 bf16 (33) 60, 53 in
// blocks of 32, 10576 x 2560 fp32 (19) 19.  Divisions in place of corrected products took 204 and 86.  Values: 16384 x 5120 to bf16 (33) 39, 60 with
// a division to find a thread's row.  2560 rows of 16384 to int8 (70) 87, to four bits (67) 110: one block of 96 KB a row to an SM.  Rows wider than
// that are read twice in blocks of 16, 2048 x 32768 bf16 (26) 63, fp32 (47) 92, 256 x 131072 (13) 47, and once in blocks of 32, bf16 44.  One row of
// 768: 2.0, where the call itself takes 3.7 from Python.
#include "fp4.cuh"
#include "kernels.h"
#include "sm100.cuh"

#include <type_traits>

namespace ssdi8 {
namespace {

constexpr int kRing = 2;      // rows of a block's ring
constexpr int kChunk = 256;   // columns of a chunk: a warp's lanes have eight each, so that a block of 16 is two lanes and one of 32 four

struct None {};   // no residual stream

struct RowParams {
  const void* x; i64 sx;
  const void* residual; i64 sr;
  void* stream; i64 ss;
  const float* weight;
  const float* static_scale;
  int8_t* xq; float* scale;                  // int8: codes, step sizes (or NULL)
  uint8_t *codes, *scales; float* step;      // four bits
  int32_t* status;
  int D, block, tiles;
  bool vx, vr, vs;                           // rows on 16 bytes (16-bit elements), 16 bytes (fp32)
  float eps;
};

template <typename T>
__device__ __forceinline__ void unpack8(const uint4& q, float (&v)[8]) {   // of 16-bit elements
  const float4 a = Elem<T>::cvt(make_uint2(q.x, q.y)), b = Elem<T>::cvt(make_uint2(q.z, q.w));
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void spread8(const float4& a, const float4& b, float (&v)[8]) {
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, bool aligned, float (&v)[8]) {   // from global memory
  if (aligned) {
    if constexpr (sizeof(T) == 4) spread8(__ldcs(reinterpret_cast<const float4*>(p)), __ldcs(reinterpret_cast<const float4*>(p) + 1), v);
    else unpack8<T>(__ldcs(reinterpret_cast<const uint4*>(p)), v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = Elem<T>::get(p[i]);
  }
}
template <typename T>
__device__ __forceinline__ void load8_shared(const void* p, float (&v)[8]) {   // on 16 bytes
  if constexpr (sizeof(T) == 4) spread8(static_cast<const float4*>(p)[0], static_cast<const float4*>(p)[1], v);
  else unpack8<T>(*static_cast<const uint4*>(p), v);
}
// rounds to T, in place, and stores (p = NULL: does not)
template <typename T>
__device__ __forceinline__ void store8(T* p, bool aligned, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    if (!p) return;
    if (aligned) {
      reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = v[i];
    }
  } else {
    const uint2 a = Elem<T>::pack(make_float4(v[0], v[1], v[2], v[3])), b = Elem<T>::pack(make_float4(v[4], v[5], v[6], v[7]));
    if (!p) {
    } else if (aligned) {
      *reinterpret_cast<uint4*>(p) = make_uint4(a.x, a.y, b.x, b.y);
    } else {
      const uint32_t w[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
      for (int i = 0; i < 8; ++i) reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
    const float4 f = Elem<T>::cvt(a), g = Elem<T>::cvt(b);
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w; v[4] = g.x; v[5] = g.y; v[6] = g.z; v[7] = g.w;
  }
}

__device__ __forceinline__ void bulk_store(void* dst, const void* src, uint32_t bytes) {   // both on 16 bytes
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(sm100::smem_u32(src)), "r"(bytes) : "memory");
}
__device__ __forceinline__ float warp_max(float v) {   // of numbers >= 0; a NaN counts for nothing
  float m;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
  return m;
}
__device__ __forceinline__ float absmax8(const float (&v)[8]) {
  float a, b, c;   // (a NaN counts for nothing)
  asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(a) : "f"(v[0]), "f"(v[1]), "f"(v[2]));
  asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(b) : "f"(v[3]), "f"(v[4]), "f"(v[5]));
  asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(c) : "f"(a), "f"(v[6]), "f"(v[7]));
  return fmaxf(fmaxf(b, c), 0.f);
}

// Codes and scales in four bits of a chunk's eight columns of this lane (`live`: inside the row) into the row's codes and the row's place in the first of
// its tiles; m is their absmax.  All lanes of the warp call it.  Bytes of a tile's blocks behind the row's end are 0.
template <int BLOCK, bool SAFE>
__device__ __forceinline__ void chunk_fp4(uint8_t* codes, uint8_t* scales, int tiles, int chunk, bool live, const float (&v)[8], float m, const Fp4Row& r) {
  const int lane = threadIdx.x & 31;
  constexpr int lanes = BLOCK / 8, shift = BLOCK == 16 ? 3 : 4;   // of a block; of a tile's four blocks (logarithm)
  m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
  if (BLOCK == 32) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
  uint32_t s = BLOCK == 16 ? fp4_scale16<SAFE>(m, r) : fp4_scale32(m);
  const uint32_t c = BLOCK == 16 ? fp4_codes16<SAFE>(v, r, e4m3_to(s)) : fp4_codes32(v, s);
  s = live ? s : 0u;
  uint32_t word = s | __shfl_down_sync(0xffffffffu, s, lanes) << 8;
  word |= __shfl_down_sync(0xffffffffu, word, 2 * lanes) << 16;
  if (live) reinterpret_cast<uint32_t*>(codes)[chunk * 32 + lane] = c;
  const int tile = (chunk << (5 - shift)) + (lane >> shift);
  if ((lane & (4 * lanes - 1)) == 0 && tile < tiles) *reinterpret_cast<uint32_t*>(scales + tile * kTileBytes) = word;
}
template <int BLOCK, bool SAFE, int NCH>
__device__ __forceinline__ void row_fp4(const RowParams& p, i64 row, int c0, const float (&v)[NCH][8], const float (&m)[NCH], const Fp4Row& r) {
  uint8_t* const codes = p.codes + row * (p.D / 2);
  uint8_t* const scales = p.scales + fp4_scale_at(row, 0, p.tiles);
  const int col = (threadIdx.x & 31) * 8;
#pragma unroll
  for (int k = 0; k < NCH; ++k)
    if ((c0 + k) * kChunk < p.D) chunk_fp4<BLOCK, SAFE>(codes, scales, p.tiles, c0 + k, (c0 + k) * kChunk + col < p.D, v[k], m[k], r);
}
template <int NCH>   // rows whose step size is beyond what the corrected products take
__device__ __noinline__ void row_fp4_by_division(const RowParams& p, i64 row, int c0, const float (&v)[NCH][8], const float (&m)[NCH], const Fp4Row& r) {
  row_fp4<16, false, NCH>(p, row, c0, v, m, r);
}

// What a row's threads say to one another; two of each, so that a row's are read while the next one's are written
struct Meeting {
  double sums[2][16];
  float maxima[2][16];
};

// A warp's chunks of a row from their h (v): p = h w, the row's sum of squares and absmax of p (the block's only barrier), step sizes and codes.
// `behind` is called behind that barrier.
template <int NCH, bool NORM, bool FP4, bool RING, typename F>
__device__ __forceinline__ void finish_row(const RowParams& p, Meeting& meet, int turn, i64 row, float (&v)[NCH][8], F behind) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const int c0 = warp * NCH, col0 = c0 * kChunk + lane * 8;
  float m[NCH];
  constexpr int SIDE = NCH == 1 ? 4 : 1;   // sums side by side: their chain is what a short row waits for (two chunks have no registers for it)
  double part[SIDE] = {};
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
    if constexpr (NORM) {
#pragma unroll
      for (int i = 0; i < 8; ++i) part[i % SIDE] = fma((double)v[k][i], (double)v[k][i], part[i % SIDE]);
      if (p.weight && col0 + k * kChunk < p.D) {
        const float4 a = reinterpret_cast<const float4*>(p.weight + col0 + k * kChunk)[0], b = reinterpret_cast<const float4*>(p.weight + col0 + k * kChunk)[1];
        const float w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float2 x = __fmul2_rn(make_float2(v[k][i], v[k][i + 1]), make_float2(w[i], w[i + 1]));
          v[k][i] = x.x;
          v[k][i + 1] = x.y;
        }
      }
    }
    m[k] = absmax8(v[k]);
  }
  float top = 0.f;
  if (NORM || p.block == 16) {
#pragma unroll
    for (int k = 0; k < NCH; ++k) top = fmaxf(top, m[k]);
    top = warp_max(top);
    double ss = part[0];
    if (SIDE == 4) ss = (part[0] + part[1 % SIDE]) + (part[2 % SIDE] + part[3 % SIDE]);
    if constexpr (NORM) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    }
    if (lane == 0) {
      meet.maxima[turn][warp] = top;
      if (NORM) meet.sums[turn][warp] = ss;
    }
  }
  if (NORM || RING || p.block == 16) __syncthreads();
  behind();
  if (NORM || p.block == 16) top = warp_max(lane < nwarps ? meet.maxima[turn][lane] : 0.f);
  // 1 / sqrt(mean + eps), by the threads that need it; 0 for a row of zeros without an eps, whose codes are 0 under a static step too
  auto factor = [&] {
    double s = 0.0;
    for (int i = 0; i < nwarps; ++i) s += meet.sums[turn][i];
    s = s / (double)p.D + (double)p.eps;
    return s == 0.0 ? 0.0 : 1.0 / sqrt(s);
  };
  // the step size of a row whose codes have step a: 1 where they are all 0, but for a row with a NaN in it
  auto step_of = [&](bool some, float a) {
    const double r = factor();
    return some || r != r ? (float)((double)a * r) : 1.0f;
  };
  if constexpr (FP4) {
    Fp4Row r = {1.0f, 6.0f, 0.f, true};
    if (p.block == 16) r = fp4_row(top);
    if (p.step && threadIdx.x == 0) {
      if constexpr (NORM) p.step[row] = step_of(top > 0.f, r.g);
      else p.step[row] = r.g;
    }
    if (p.block == 32) {
      row_fp4<32, true, NCH>(p, row, c0, v, m, r);
    } else if (r.safe) {
      row_fp4<16, true, NCH>(p, row, c0, v, m, r);
    } else {
      float w[NCH][8], n[NCH];   // (copies: the call takes their addresses)
#pragma unroll
      for (int k = 0; k < NCH; ++k) {
        n[k] = m[k];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[k][i] = v[k][i];
      }
      const Fp4Row q = r;
      row_fp4_by_division<NCH>(p, row, c0, w, n, q);
    }
  } else {
    float a;
    if (p.static_scale) {
      const float r = (float)factor();
      a = *p.static_scale;
#pragma unroll
      for (int k = 0; k < NCH; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] = __fmul_rn(v[k][i], r);
    } else {
      // (the product with the rounded reciprocal and one correction: the correctly rounded quotient for all 2^23 significands)
      constexpr float c = 1.0f / 127.0f;
      a = __fmul_rn(top, c);
      a = __fmaf_rn(__fmaf_rn(-a, 127.0f, top), c, a);
      if (!(top >= 1e-25f && top <= 1e25f)) a = __fdiv_rn(top, 127.0f);
      const bool some = a > 0.f;
      a = some ? a : 1.0f;
      if (p.scale && threadIdx.x == 0) p.scale[row] = step_of(some, a);
    }
    const float4 a4 = make_float4(a, a, a, a);
    const Step4 st = step4(a4);
#pragma unroll
    for (int k = 0; k < NCH; ++k)
      if (col0 + k * kChunk < p.D) {
        const float4 lo = make_float4(v[k][0], v[k][1], v[k][2], v[k][3]), hi = make_float4(v[k][4], v[k][5], v[k][6], v[k][7]);
        const uint2 q = st.usable ? make_uint2(code4(lo, st), code4(hi, st)) : make_uint2(code4_by_division(lo, a4), code4_by_division(hi, a4));
        *reinterpret_cast<uint2*>(p.xq + row * p.D + col0 + k * kChunk) = q;
      }
  }
}

// A block has a row, a warp NCH chunks of it, one after the other.  NORM: h, its norm and the weight; else p is x (four bits).
template <typename T, typename R, int NCH, bool NORM, bool FP4>
__global__ void __launch_bounds__(512) row_kernel(const __grid_constant__ RowParams p) {
  __shared__ Meeting meet;
  pdl_launch_dependents();
  pdl_wait();
  const i64 row = blockIdx.x;
  const int col0 = (threadIdx.x >> 5) * NCH * kChunk + (threadIdx.x & 31) * 8;
  float v[NCH][8];
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[k][i] = 0.f;
    if (col0 + k * kChunk < p.D) load8<T>(static_cast<const T*>(p.x) + row * p.sx + col0 + k * kChunk, p.vx, v[k]);
  }
  if constexpr (!std::is_same<R, None>::value) {
    const R* const res = static_cast<const R*>(p.residual);
    R* const out = static_cast<R*>(p.stream);
    float r[NCH][8];
#pragma unroll
    for (int k = 0; k < NCH; ++k)
      if (res && col0 + k * kChunk < p.D) load8<R>(res + row * p.sr + col0 + k * kChunk, p.vr, r[k]);
#pragma unroll
    for (int k = 0; k < NCH; ++k)
      if (col0 + k * kChunk < p.D) {
        if (res) {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[k][i] = __fadd_rn(v[k][i], r[k][i]);
        }
        store8<R>(out ? out + row * p.ss + col0 + k * kChunk : nullptr, p.vs, v[k]);
      }
  }
  finish_row<NCH, NORM, FP4, false>(p, meet, 0, row, v, [] {});
}

// Many rows: a block walks rows a grid apart through a ring in shared memory, the next row's x and residual on their way by bulk copies while one
// is worked on.  The row's barrier (every thread has its elements in registers then) gives its place in the ring to the row after the next; where there is a
// residual stream, h takes the place of the residual, leaves from there, and the next copy waits until it has been read.
template <typename T, typename R, int NCH, bool NORM, bool FP4>
__global__ void __launch_bounds__(512, 2) ring_kernel(const __grid_constant__ RowParams p, int rows) {
  using namespace sm100;
  constexpr bool STREAM = !std::is_same<R, None>::value;
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ Meeting meet;
  __shared__ uint64_t full[kRing];
  const int tid = threadIdx.x, col0 = (tid >> 5) * NCH * kChunk + (tid & 31) * 8;
  typedef typename std::conditional<STREAM, R, T>::type S;
  const uint32_t xbytes = p.D * (uint32_t)sizeof(T), rbytes = STREAM ? p.D * (uint32_t)sizeof(S) : 0u;
  if (tid == 0) {
    for (int i = 0; i < kRing; ++i) mbar_init(&full[i], 1);
    fence_mbar_init();
  }
  __syncthreads();
  pdl_launch_dependents();
  pdl_wait();
  auto request = [&](int s, i64 row) {   // by one thread
    uint8_t* const at = ring + s * (xbytes + rbytes);
    mbar_expect_tx(&full[s], xbytes + (STREAM && p.residual ? rbytes : 0u));
    bulk_load(at, static_cast<const T*>(p.x) + row * p.sx, xbytes, &full[s]);
    if (STREAM && p.residual) bulk_load(at + xbytes, static_cast<const S*>(p.residual) + row * p.sr, rbytes, &full[s]);
  };
  if (tid == 0)
    for (int s = 0; s < kRing && blockIdx.x + (i64)s * gridDim.x < rows; ++s) request(s, blockIdx.x + (i64)s * gridDim.x);
  int s = 0, round = 0, turn = 0;
  bool late = false;
  for (i64 row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
    uint8_t* const at = ring + s * (xbytes + rbytes);
    late |= !mbar_wait_inline<0>(&full[s], round & 1, p.status);
    float v[NCH][8];
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int col = col0 + k * kChunk;
      if (col >= p.D) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] = 0.f;
      } else {
        load8_shared<T>(reinterpret_cast<const T*>(at) + col, v[k]);
        if constexpr (STREAM) {
          S* const h = reinterpret_cast<S*>(at + xbytes) + col;
          if (p.residual) {
            float r[8];
            load8_shared<S>(h, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = __fadd_rn(v[k][i], r[i]);
          }
          store8<S>(h, true, v[k]);
        }
      }
    }
    if (STREAM) fence_async_smem();   // (ahead of the copies from and to the places just written)
    const i64 next = row + (i64)kRing * gridDim.x;
    finish_row<NCH, NORM, FP4, true>(p, meet, turn, row, v, [&] {   // behind the barrier
      if (tid == 0) {
        if (STREAM && p.stream) {
          bulk_store(static_cast<S*>(p.stream) + row * p.ss, at + xbytes, rbytes);
          tma_store_commit();
        }
        if (next < rows) {
          if (STREAM && p.stream) tma_store_wait_read();
          request(s, next);
        }
      }
    });
    if (++s == kRing) { s = 0; ++round; }
  }
  if (STREAM && p.stream && tid == 0) tma_store_wait_read();
  if (late)   // (a copy may still be under way)
    for (int i = 0; i < 50; ++i) __nanosleep(1000);
}

// Rows wider than a block's registers: the row is read twice where its absmax is needed.
template <typename T>
__global__ void __launch_bounds__(512) wide_kernel(const __grid_constant__ RowParams p) {
  __shared__ float maxima[16];
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const i64 row = blockIdx.x;
  const T* const x = static_cast<const T*>(p.x) + row * p.sx;
  float v[8];
  Fp4Row r = {1.0f, 6.0f, 0.f, true};
  if (p.block == 16) {
    float top = 0.f;
    for (int c = threadIdx.x * 8; c < p.D; c += 512 * 8) {
      load8<T>(x + c, p.vx, v);
      top = fmaxf(top, absmax8(v));
    }
    top = warp_max(top);
    if (lane == 0) maxima[warp] = top;
    __syncthreads();
    r = fp4_row(warp_max(lane < 16 ? maxima[lane] : 0.f));
  }
  if (p.step && threadIdx.x == 0) p.step[row] = r.g;
  for (int c = warp; c * kChunk < p.D; c += 16) {
    const int col = c * kChunk + lane * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (col < p.D) load8<T>(x + col, p.vx, v);
    const float w[1][8] = {{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}}, m[1] = {absmax8(v)};
    if (p.block == 32) row_fp4<32, true, 1>(p, row, c, w, m, r);
    else if (r.safe) row_fp4<16, true, 1>(p, row, c, w, m, r);
    else row_fp4<16, false, 1>(p, row, c, w, m, r);
  }
}

// Values of a matrix in four bits: a row is one or more warps', a thread has up to four vectors of 16 bytes of it at a time
template <typename T>
__global__ void __launch_bounds__(256) values_kernel(const uint8_t* codes, const uint8_t* scales, const float* step, T* out, i64 stride, bool aligned,
                                                     int rows, int D, int block, int tiles) {
  constexpr int V = 16 / (int)sizeof(T);
  pdl_launch_dependents();
  pdl_wait();
  const i64 row = blockIdx.x * (i64)blockDim.y + threadIdx.y;
  if (row >= rows) return;
  const uint8_t* const c = codes + row * (D / 2);
  const uint8_t* const sc = scales + fp4_scale_at(row, 0, tiles);
  T* const to = out + row * stride;
  const float f = step ? step[row] : 1.0f;
  const int shift = block == 16 ? 4 : 5;
#pragma unroll 1
  for (int c0 = threadIdx.x * V; c0 < D; c0 += 4 * blockDim.x * V) {
    uint32_t w[4], s[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int col = c0 + k * blockDim.x * V, b = col >> shift;
      w[k] = s[k] = 0;
      if (col < D) {
        w[k] = __ldcs(reinterpret_cast<const uint32_t*>(c) + (col >> 3));   // (binary32: the eight codes that two lanes' vectors are in)
        s[k] = sc[(b >> 2) * kTileBytes + (b & 3)];
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int col = c0 + k * blockDim.x * V;
      if (col >= D) break;
      const float sv = block == 16 ? e4m3_to(s[k]) : e8m0_to(s[k]);
      float v[8];
      e2m1_to8(w[k], v);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = __fmul_rn(__fmul_rn(V == 4 && (col & 4) ? v[4 + (i & 3)] : v[i], sv), f);
      if constexpr (V == 8) {
        store8<T>(to + col, aligned, v);
      } else if (aligned) {
        *reinterpret_cast<float4*>(to + col) = make_float4(v[0], v[1], v[2], v[3]);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) to[col + i] = v[i];
      }
    }
  }
}

// Many rows on 16 bytes go through the ring, with as many blocks as shared memory has room for with two rows each (of narrow rows threads and registers hold fewer at
// a time): what a row waits for is then on its way while the one before
// is worked on (us, direct and ring: 16384 x 2560 bf16 with an fp32 stream to int8 81 and 79, to four bits 87 and 75, bf16 stream 72 and 56;
// 4096 x 8192 75 and 61; quantiser 16384 x 5120 bf16 75 and 56).  Not fp32 rows without a stream, whose 32 bytes a lane meet in shared memory's banks
// (quantiser 10576 x 2560 19 and 24).  A chunk to a warp where rows are short (or few: 300 x 2560 6.0 with two, 4.2),
// two up to 8192 columns; four where the quantiser, which asks less of
// a row's warps, has many rows (16384 x 5120 67 and 56; 64 x 5120 2.2 and 2.8).
template <typename T, typename R, bool NORM, bool FP4>
ssdi8_status_t launch(const RowParams& p, i64 rows, cudaStream_t st) {
  const int chunks = (p.D + kChunk - 1) / kChunk;
  const int sms = sm_count();
  if (sms <= 0) return SSDI8_ERR_CUDA;
  constexpr bool STREAM = !std::is_same<R, None>::value;
  constexpr i64 kShared = 200 * 1024;
  const i64 bytes = (i64)p.D * (sizeof(T) + (STREAM ? sizeof(typename std::conditional<STREAM, R, T>::type) : 0));
  const i64 fit = kShared / (kRing * bytes), blocks = fit < 32 ? fit : 32;   // on an SM
  const bool ring = (STREAM || sizeof(T) == 2) && p.vx && (!p.residual || p.vr) && (!p.stream || p.vs) && blocks > 0 && rows > 2 * sms * blocks;
  auto go = [&](auto n) -> ssdi8_status_t {
    constexpr int NCH = decltype(n)::value;
    const int warps = (chunks + NCH - 1) / NCH;
    if constexpr (STREAM || sizeof(T) == 2) {
      if (ring)
        return launch_sized(ring_kernel<T, R, NCH, NORM, FP4>, dim3((unsigned)(sms * blocks)), dim3(32 * warps), (size_t)(kRing * bytes), (size_t)kShared, -1,
                            false, st, p, (int)rows);
    }
    return launch_configured(row_kernel<T, R, NCH, NORM, FP4>, dim3((unsigned)rows), dim3(32 * warps), 0, -1, false, st, p);
  };
  // (short rows of a ring: without a second warp, or with half as many, a row's meeting is short.  16001 x 320 bf16 21 and 15, 16384 x 1024 to four bits 33 and
  // 29, quantiser 16384 x 768 15 and 12; three chunks of a norm are better off apart: 16384 x 768 26, 28 with two warps, 32 with one)
  if (ring && (chunks == 2 || (NORM && chunks == 4))) return go(std::integral_constant<int, 2>());
  if (ring && !NORM && chunks > 2 && chunks <= 4) return go(std::integral_constant<int, 4>());
  if (chunks <= (rows <= 4 * sms ? 16 : 8)) return go(std::integral_constant<int, 1>());
  if (chunks <= 32 && (NORM || !ring)) return go(std::integral_constant<int, 2>());
  return go(std::integral_constant<int, 4>());
}

template <typename T>
bool rows_aligned(const void* p, i64 stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % (16 / (i64)sizeof(T)) == 0; }

template <typename T, typename R>
ssdi8_status_t norm_of(const ssdi8_add_norm_args_t& a, cudaStream_t st) {
  RowParams p = {};
  p.x = a.x; p.sx = a.stride_x; p.vx = rows_aligned<T>(a.x, a.stride_x);
  if constexpr (!std::is_same<R, None>::value) {
    p.residual = a.residual; p.sr = a.stride_residual; p.vr = rows_aligned<R>(a.residual, a.stride_residual);
    p.stream = a.residual_out; p.ss = a.stride_out; p.vs = rows_aligned<R>(a.residual_out, a.stride_out);
  }
  p.weight = a.weight; p.static_scale = a.static_scale; p.xq = a.xq; p.scale = a.scale;
  p.D = a.width; p.eps = a.eps; p.status = a.status;
  if (!a.fp4) return launch<T, R, true, false>(p, a.rows, st);
  p.codes = a.fp4->codes; p.scales = a.fp4->scales; p.step = a.fp4->step;
  p.block = a.fp4->block; p.tiles = fp4_tiles(p.D, p.block);
  return launch<T, R, true, true>(p, a.rows, st);
}

template <typename T>
ssdi8_status_t quantize_of(const void* x, i64 stride, const ssdi8_fp4_t& q, int32_t* status, cudaStream_t st) {
  RowParams p = {};
  p.x = x; p.sx = stride; p.vx = rows_aligned<T>(x, stride);
  p.codes = q.codes; p.scales = q.scales; p.step = q.step;
  p.status = status;
  p.D = q.width; p.block = q.block; p.tiles = fp4_tiles(q.width, q.block);
  if (q.width <= kMaxNormWidth) return launch<T, None, false, true>(p, q.rows, st);
  return launch_configured(wide_kernel<T>, dim3((unsigned)q.rows), dim3(512), 0, -1, false, st, p);
}

}  // namespace

ssdi8_status_t launch_add_norm(const ssdi8_add_norm_args_t& a, int dtype, int rdtype, cudaStream_t st) {
  if (rdtype < 0)
    return dtype == 0 ? norm_of<float, None>(a, st) : dtype == 1 ? norm_of<__half, None>(a, st) : norm_of<__nv_bfloat16, None>(a, st);
  if (rdtype == 0)
    return dtype == 0 ? norm_of<float, float>(a, st) : dtype == 1 ? norm_of<__half, float>(a, st) : norm_of<__nv_bfloat16, float>(a, st);
  return dtype == 1 ? norm_of<__half, __half>(a, st) : norm_of<__nv_bfloat16, __nv_bfloat16>(a, st);
}

ssdi8_status_t launch_fp4_quantize(const void* x, i64 stride, int dtype, const ssdi8_fp4_t& q, int32_t* status, cudaStream_t st) {
  return dtype == 0 ? quantize_of<float>(x, stride, q, status, st)
       : dtype == 1 ? quantize_of<__half>(x, stride, q, status, st)
                    : quantize_of<__nv_bfloat16>(x, stride, q, status, st);
}

ssdi8_status_t launch_fp4_dequantize(const ssdi8_fp4_t& q, void* out, i64 stride, int dtype, cudaStream_t st) {
  auto go = [&](auto t) -> ssdi8_status_t {
    typedef decltype(t) T;
    // (four vectors a thread where a row has as many)
    const int vectors = q.width / (16 / (int)sizeof(T)), tx = vectors <= 128 ? 32 : vectors <= 1024 ? (vectors / 4 + 31) / 32 * 32 : 256, ty = 256 / tx;
    return launch_configured(values_kernel<T>, dim3((unsigned)((q.rows + (i64)ty - 1) / ty)), dim3(tx, ty), 0, -1, false, st, (const uint8_t*)q.codes,
                             (const uint8_t*)q.scales, (const float*)q.step, static_cast<T*>(out), stride, rows_aligned<T>(out, stride), q.rows, q.width,
                             q.block, fp4_tiles(q.width, q.block));
  };
  return dtype == 0 ? go(float()) : dtype == 1 ? go(__half()) : go(__nv_bfloat16());
}

}  // namespace ssdi8
