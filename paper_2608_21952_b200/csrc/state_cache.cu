// Writing states into the 8-bit cache and reading them back.  Both stream: the fp32 state is 4 of the 5 bytes per element that
// have to move (write: one pass, the row in registers between its absmax and its codes; read: codes in, fp32 out, with the
// waiting tokens as up to 16 rank-one updates in registers).  Write, 8 sequences x 80 heads (26 MB, 4 us at the copy rate): 7.2 us, most of it one
// round trip and the launch.  Read, 37 x 128 heads with half-filled windows (198 MB, 31 us): 47, the chain slot, window, weights, operands ahead of a
// block's stores with 32 warps to an SM (operands written by lanes of one bank 77; eight single loads of x a token where two do 57).
#include "kernels.h"
#include "state_cache.cuh"

namespace ssdi8 {
namespace {

constexpr int SC_T = 256;

// N / 4 lanes per row, four rows of four elements per thread, all in flight; a block has so many rows of a head.  (A whole head
// of N 128 to a block, eight rows per thread and four blocks on an SM: 8 sequences x 80 heads 8.1 us.)
template <int N>
__global__ void __launch_bounds__(SC_T) cache_write_kernel(CacheView c, const int32_t* __restrict__ slots, const int32_t* __restrict__ pos,
                                                           const float4* __restrict__ state, int32_t* status, int H) {
  constexpr int N4 = N / 4, RPP = SC_T / N4, R = 4, SPLIT = 64 / (R * RPP);   // lanes per row, rows per pass, passes, blocks per head
  pdl_launch_dependents();
  pdl_wait();
  const int bh = blockIdx.x / SPLIT, b = bh / H, h = bh % H;
  const int lane = threadIdx.x % N4, p0 = blockIdx.x % SPLIT * R * RPP + threadIdx.x / N4;
  float4 v[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
    v[r] = state ? __ldcs(state + (((i64)b * H + h) * 64 + p0 + r * RPP) * N4 + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
  bool bad;
  const int slot = slot_of(slots, pos, c.nslots, b, &bad);
  if (bad && h == 0 && threadIdx.x == 0) bad_row(status);
  if (slot < 0) return;
  if (h == 0 && p0 == 0 && lane == 0) c.start[slot] = pos ? pos[b] : 0;
  const i64 row0 = ((i64)slot * H + h) * 64 + p0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float m = fmaxf(fmaxf(fmaxf(fabsf(v[r].x), fabsf(v[r].y)), fmaxf(fabsf(v[r].z), fabsf(v[r].w))), 0.f);   // (not NaN)
#pragma unroll
    for (int o = N4 / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    float s = step_of_max(__float_as_uint(m));
    if (s == 0.f) s = 1.f;   // (the quotient underflowed)
    const float4 a = make_float4(s, s, s, s);
    const Step4 st = step4(a);
    const i64 row = row0 + r * RPP;
    reinterpret_cast<uint32_t*>(c.codes)[row * N4 + lane] = st.usable ? code4(v[r], st) : code4_by_division(v[r], a);
    if (lane == 0) c.scales[row] = s;
  }
}

template <int N>
__global__ void __launch_bounds__(SC_T, 4) cache_read_kernel(CacheView c, const int32_t* __restrict__ slots, const int32_t* __restrict__ first,
                                                          const int32_t* __restrict__ pos, const float* __restrict__ A,
                                                          const float* __restrict__ s_x, const float* __restrict__ s_B,
                                                          float4* __restrict__ state, int32_t* status, int H, int G) {
  constexpr int THREADS = SC_T, N4 = N / 4, RPP = THREADS / N4, R = 64 / RPP;
  __shared__ __align__(16) float xw[kWin][64];
  __shared__ float4 Bf[kWin][N4];
  __shared__ float wj[kWin], whole;
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.x / H, h = blockIdx.x % H, g = h / (H / G);
  const int lane = threadIdx.x % N4, p0 = threadIdx.x / N4 * R;   // R rows, one after the other
  bool bad;
  const int slot = slot_of(slots, pos, c.nslots, b, &bad);
  int n = 0, f = 0;
  if (slot >= 0) {
    const int p = pos[b];
    f = first ? first[b] : max(c.start[slot], p - p % kWin);
    bad = f < 0 || f > p || p - f > kWin;
    n = bad ? 0 : p - f;
  }
  if (bad && h == 0 && threadIdx.x == 0) bad_row(status);
  if (slot < 0 || bad) return;
  const i64 sh = (i64)slot * H + h;
  uint32_t q[R];
  float sc[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    q[r] = __ldcs(reinterpret_cast<const uint32_t*>(c.codes) + (sh * 64 + p0 + r) * N4 + lane);
    sc[r] = c.scales[sh * 64 + p0 + r];
  }
  if (n > 0) {
    // x of the waiting tokens with all their factors, [row][p], and B, [row][n]; the weights by one warp, lane j of a half for row j
    const int j = threadIdx.x >> 4, word = threadIdx.x & 15;
    const uint32_t x4 = reinterpret_cast<const uint32_t*>(c.xwin)[(sh * kWin + j) * 16 + word];
    const float4 sx = *reinterpret_cast<const float4*>(s_x + h * 64 + 4 * word);
    uint32_t B4[kWin * N4 / THREADS];
#pragma unroll
    for (int k = 0; k < kWin * N4 / THREADS; ++k)
      B4[k] = reinterpret_cast<const uint32_t*>(c.Bwin)[((i64)slot * G + g) * kWin * N4 + threadIdx.x + k * THREADS];
    if (threadIdx.x < 32) {
      const int row = threadIdx.x & 15, order = (row - f) & (kWin - 1);
      const float dt = order < n ? c.dtwin[sh * kWin + row] : 0.f;
      const Waiting w = waiting_of(dt, order);
      const double e = exp((double)A[h] * (threadIdx.x < 16 ? w.behind : w.all));
      if (threadIdx.x < 16) wj[row] = order < n ? (float)((double)dt * e) * s_B[g] : 0.f;
      if (threadIdx.x == 16) whole = (float)e;
    }
    __syncthreads();
    const float w = wj[j];
    *reinterpret_cast<float4*>(&xw[j][4 * word]) =
        make_float4(w * sx.x * (float)sx8(x4, 0), w * sx.y * (float)sx8(x4, 1), w * sx.z * (float)sx8(x4, 2), w * sx.w * (float)sx8(x4, 3));
#pragma unroll
    for (int k = 0; k < kWin * N4 / THREADS; ++k)
      (&Bf[0][0])[threadIdx.x + k * THREADS] = make_float4((float)sx8(B4[k], 0), (float)sx8(B4[k], 1), (float)sx8(B4[k], 2), (float)sx8(B4[k], 3));
  } else if (threadIdx.x == 0) {
    whole = 1.f;
  }
  __syncthreads();
  float2 v[R][2];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float s = sc[r] * whole;
    const uint32_t w = q[r] ^ 0x80808080u;
    v[r][0] = make_float2(s * s8_to_f32(w, 0), s * s8_to_f32(w, 1));
    v[r][1] = make_float2(s * s8_to_f32(w, 2), s * s8_to_f32(w, 3));
  }
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    const int row = (f + i) & (kWin - 1);
    const float4 B = Bf[row][lane];
    float xr[R];
#pragma unroll
    for (int r = 0; r < R; r += 4) *reinterpret_cast<float4*>(xr + r) = *reinterpret_cast<const float4*>(&xw[row][p0 + r]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float x = xr[r];
      v[r][0] = __ffma2_rn(make_float2(x, x), make_float2(B.x, B.y), v[r][0]);
      v[r][1] = __ffma2_rn(make_float2(x, x), make_float2(B.z, B.w), v[r][1]);
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
    __stcs(state + (((i64)b * H + h) * 64 + p0 + r) * N4 + lane, make_float4(v[r][0].x, v[r][0].y, v[r][1].x, v[r][1].y));
}

}  // namespace

ssdi8_status_t launch_cache_write(const Dims& d, const ssdi8_cache_t& c, const int32_t* slots, const int32_t* pos, const float* state,
                                  int32_t* status, cudaStream_t st) {
  auto go = [&](auto kernel) {
    return launch_configured(kernel, dim3((unsigned)(d.b * d.H * (d.N / 64))), dim3(SC_T), 0, kStreamCarveout, false, st, view_of(c), slots, pos,
                             reinterpret_cast<const float4*>(state), status, d.H);
  };
  return d.N == 128 ? go(cache_write_kernel<128>) : go(cache_write_kernel<64>);
}

ssdi8_status_t launch_cache_read(const Dims& d, const ssdi8_cache_t& c, const int32_t* slots, const int32_t* first, const int32_t* pos,
                                 const float* A, const float* s_x, const float* s_B, float* state, int32_t* status, cudaStream_t st) {
  auto go = [&](auto kernel) {
    return launch_configured(kernel, dim3((unsigned)(d.b * d.H)), dim3(SC_T), 0, -1, false, st, view_of(c), slots, first, pos, A, s_x, s_B,
                             reinterpret_cast<float4*>(state), status, d.H, d.G);
  };
  return d.N == 128 ? go(cache_read_kernel<128>) : go(cache_read_kernel<64>);
}

}  // namespace ssdi8
