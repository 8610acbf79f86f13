// Writing states into the 8-bit cache and reading them back.  Both stream: the fp32 state is 4 of the 5 bytes per element that
// have to move (write: one pass, the row in registers between its absmax and its codes; read: codes in, fp32 out, with the
// waiting tokens as up to 16 rank-one updates in registers).
#include "kernels.h"
#include "state_cache.cuh"

namespace ssdi8 {
namespace {

constexpr int SC_T = 256;

// One block per (sequence, head): N / 4 lanes per row, P N / (4 * 256) rows of four elements per thread, all in flight.
template <int N>
__global__ void __launch_bounds__(SC_T) cache_write_kernel(CacheView c, const int32_t* __restrict__ slots, const int32_t* __restrict__ pos,
                                                           const float4* __restrict__ state, int32_t* status, int H) {
  constexpr int N4 = N / 4, RPP = SC_T / N4, R = 64 / RPP;   // lanes per row, rows per pass, passes
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.x / H, h = blockIdx.x % H;
  const int lane = threadIdx.x % N4, p0 = threadIdx.x / N4;
  float4 v[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
    v[r] = state ? __ldcs(state + (((i64)b * H + h) * 64 + p0 + r * RPP) * N4 + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
  bool bad;
  const int slot = slot_of(slots, pos, c.nslots, b, &bad);
  if (bad && h == 0 && threadIdx.x == 0 && status) atomicExch(status, (int32_t)SSDI8_ERR_SHAPE);
  if (slot < 0) return;
  if (h == 0 && threadIdx.x == 0) c.start[slot] = pos ? pos[b] : 0;
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
__global__ void __launch_bounds__(SC_T) cache_read_kernel(CacheView c, const int32_t* __restrict__ slots, const int32_t* __restrict__ first,
                                                          const int32_t* __restrict__ pos, const float* __restrict__ A,
                                                          const float* __restrict__ s_x, const float* __restrict__ s_B,
                                                          float4* __restrict__ state, int32_t* status, int H, int G) {
  constexpr int N4 = N / 4, RPP = SC_T / N4, R = 64 / RPP;
  __shared__ float xw[kWin][64];
  __shared__ float4 Bf[kWin][N4];
  __shared__ float whole;
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.x / H, h = blockIdx.x % H, g = h / (H / G);
  const int lane = threadIdx.x % N4, p0 = threadIdx.x / N4;
  bool bad;
  const int slot = slot_of(slots, pos, c.nslots, b, &bad);
  int n = 0, f = 0;
  if (slot >= 0) {
    const int p = pos[b];
    f = first ? first[b] : max(c.start[slot], p - p % kWin);
    bad = f < 0 || f > p || p - f > kWin;
    n = bad ? 0 : p - f;
  }
  if (bad && h == 0 && threadIdx.x == 0 && status) atomicExch(status, (int32_t)SSDI8_ERR_SHAPE);
  if (slot < 0 || bad) return;
  const i64 sh = (i64)slot * H + h;
  uint32_t q[R];
  float sc[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    q[r] = __ldcs(reinterpret_cast<const uint32_t*>(c.codes) + (sh * 64 + p0 + r * RPP) * N4 + lane);
    sc[r] = c.scales[sh * 64 + p0 + r * RPP];
  }
  if (n > 0) {
    const int j = threadIdx.x & 15, order = (j - f % kWin + kWin) % kWin;
    const float dt = order < n ? c.dtwin[sh * kWin + j] : 0.f;
    const Waiting w = waiting_of(dt, order);
    const float wj = order < n ? (float)((double)dt * exp((double)A[h] * w.behind)) * s_B[g] : 0.f;
    if (threadIdx.x == 0) whole = (float)exp((double)A[h] * w.all);
    // x of the waiting tokens with all their factors, [order][p], and B, [order][n]
    for (int p = threadIdx.x >> 4; p < 64; p += SC_T / 16)
      xw[order][p] = order < n ? wj * s_x[h * 64 + p] * (float)c.xwin[(sh * kWin + j) * 64 + p] : 0.f;
    for (int k = threadIdx.x >> 4; k < N4; k += SC_T / 16) {
      const uint32_t w4 = reinterpret_cast<const uint32_t*>(c.Bwin)[(((i64)slot * G + g) * kWin + j) * N4 + k];
      Bf[order][k] = make_float4((float)sx8(w4, 0), (float)sx8(w4, 1), (float)sx8(w4, 2), (float)sx8(w4, 3));
    }
  } else if (threadIdx.x == 0) {
    whole = 1.f;
  }
  __syncthreads();
  float4 v[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float s = sc[r] * whole;
    v[r] = make_float4(s * (float)sx8(q[r], 0), s * (float)sx8(q[r], 1), s * (float)sx8(q[r], 2), s * (float)sx8(q[r], 3));
  }
  for (int i = 0; i < n; ++i) {
    const float4 B = Bf[i][lane];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float x = xw[i][p0 + r * RPP];
      v[r].x = fmaf(x, B.x, v[r].x);
      v[r].y = fmaf(x, B.y, v[r].y);
      v[r].z = fmaf(x, B.z, v[r].z);
      v[r].w = fmaf(x, B.w, v[r].w);
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) __stcs(state + (((i64)b * H + h) * 64 + p0 + r * RPP) * N4 + lane, v[r]);
}

}  // namespace

ssdi8_status_t launch_cache_write(const Dims& d, const ssdi8_cache_t& c, const int32_t* slots, const int32_t* pos, const float* state,
                                  int32_t* status, cudaStream_t st) {
  auto go = [&](auto kernel) {
    return launch_configured(kernel, dim3((unsigned)(d.b * d.H)), dim3(SC_T), 0, kStreamCarveout, false, st, view_of(c), slots, pos,
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
