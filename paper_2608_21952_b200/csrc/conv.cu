// Causal convolution of a prompt with bias, SiLU and the entry quantiser (Section 4.2, "Quantization of B,C"), and the time
// step beside it.  One pass over xBC: a thread owns four consecutive channels, keeps their taps, step sizes and the last
// width - 1 tokens in registers and walks a slab of tokens, eight loads in flight, so that every element is read once (and
// width - 1 of a slab's tokens once more, from L2) and leaves as one byte.
//
// What bounds it: instructions.  8 x 2048 tokens x 80 heads (bf16, 272 MB in and out: 42 us at the copy rate) takes 108 us, 58 M warp
// instructions (20 an element: the convolution, the SiLU, the code, and the test whether binary32 may decide it); without that test and
// the time steps it takes 77.  Five blocks of four warps to an SM: four or six take 126 and 118; loads of the next eight tokens ahead of the
// present ones 117 to 135; slabs of 48 or 32 tokens 115 and 122, of 128 128.
#include "block.cuh"
#include "kernels.h"

namespace ssdi8 {
namespace {

constexpr int CT = 128;     // threads of a block: 512 channels
constexpr int CROWS = 8;    // tokens in flight

template <typename T>
struct ConvParams {
  const T* xBC; i64 sb, stok;
  const float* weight; const float* bias;
  const int32_t *lens, *slots, *pos;
  T* ring; int nslots;
  const float *s_x, *s_B, *s_C;
  uint32_t *xq, *Bq, *Cq;
  T* out;
  const T* dt_raw; i64 dt_sb, dt_stok;
  const float* dt_bias; float* dt;
  int32_t* status;
  int L, D, GN, N, H, slab, nslab, cblocks, softplus;
};

// tokens of sequence b in this call, its slot (-1: none) and position
template <typename T>
__device__ __forceinline__ int sequence(const ConvParams<T>& p, int b, bool first_block, int* slot, int* pos) {
  int len = p.lens ? min(max(p.lens[b], 0), p.L) : p.L;
  *slot = -1;
  *pos = 0;
  if (p.ring) {
    bool bad;
    *slot = slot_of(p.slots, p.pos, p.nslots, b, &bad);
    *pos = p.pos && *slot >= 0 ? p.pos[b] : 0;
    if (*slot < 0) len = 0;
    if (bad && first_block && threadIdx.x == 0 && p.status) atomicExch(p.status, (int32_t)SSDI8_ERR_SHAPE);
  }
  return len;
}

// largest magnitude of so many raw elements, as floats: magnitudes are ordered as their bits are
template <typename T> struct RawMax;
template <> struct RawMax<float> {
  uint4 m = make_uint4(0u, 0u, 0u, 0u);
  __device__ __forceinline__ void add(const float4& v) {
    m = make_uint4(max(m.x, __float_as_uint(v.x) & 0x7fffffffu), max(m.y, __float_as_uint(v.y) & 0x7fffffffu),
                   max(m.z, __float_as_uint(v.z) & 0x7fffffffu), max(m.w, __float_as_uint(v.w) & 0x7fffffffu));
  }
  __device__ __forceinline__ float4 get() const {
    return make_float4(__uint_as_float(m.x), __uint_as_float(m.y), __uint_as_float(m.z), __uint_as_float(m.w));
  }
};
template <typename T> struct RawMax16 {
  uint2 m = make_uint2(0u, 0u);
  __device__ __forceinline__ void add(const uint2& v) { m = make_uint2(__vmaxu2(m.x, v.x & 0x7fff7fffu), __vmaxu2(m.y, v.y & 0x7fff7fffu)); }
  __device__ __forceinline__ float4 get() const { return Elem<T>::cvt(m); }
};
template <> struct RawMax<__half> : RawMax16<__half> {};
template <> struct RawMax<__nv_bfloat16> : RawMax16<__nv_bfloat16> {};

// The code of token t, channel ch, in binary64, from the inputs (the ring still holds what it held before the call).
template <typename T, int W>
__device__ __noinline__ void code_exact(const ConvParams<T>& p, int b, int t, int ch, int slot, int pos) {
  const int Ch = p.D + 2 * p.GN, at = ch - p.D;
  float x[W], w[W];
#pragma unroll
  for (int k = 0; k < W; ++k) {
    const int tk = t - (W - 1) + k;
    x[k] = 0.f;
    if (tk >= 0) x[k] = Elem<T>::get(p.xBC[b * p.sb + tk * p.stok + ch]);
    else if (slot >= 0 && pos + tk >= 0) x[k] = Elem<T>::get(p.ring[((i64)slot * W + ((uint32_t)pos + tk) % W) * Ch + ch]);
    w[k] = p.weight[(i64)ch * W + k];
  }
  const float bias = p.bias ? p.bias[ch] : 0.f;
  const float step = at < 0 ? p.s_x[ch] : at < p.GN ? p.s_B[at / p.N] : p.s_C[(at - p.GN) / p.N];
  double e = (double)bias;
#pragma unroll
  for (int k = 0; k < W; ++k) e = __fma_rn((double)w[k], (double)x[k], e);
  const double r = e / ((1.0 + exp(-e)) * (double)step);
  int8_t* const out = reinterpret_cast<int8_t*>(at < 0 ? p.xq : at < p.GN ? p.Bq : p.Cq);
  const int width = at < 0 ? p.D : p.GN, col = at < 0 ? ch : at < p.GN ? at : at - p.GN;
  out[((i64)b * p.L + t) * width + col] = (int8_t)__double2int_rn(fmax(fmin(r, 127.0), -127.0));   // (fmin(NaN, 127) = 127)
}

// Groups of four quotients (a token, four channels) one of which may lie near the middle of two integers: they wait for the end of the
// block, whose threads then have a quotient each.  (Each at once by the lane that met it, its warp waiting: 157 us where
// 8 x 2048 x 80 heads with a longer and narrower test took 119.)
constexpr int kQueue = 256;
struct Queue {
  uint32_t item[kQueue];   // token of the slab << 8 | thread
  int count;
};

template <typename T, int W, bool CODES, bool ALIGNED>
__device__ __forceinline__ void conv_block(const ConvParams<T>& p, int b, int slab, int cblock, Queue& queue) {
  typedef typename Elem<T>::raw4 raw4;
  const int Ch = p.D + 2 * p.GN;
  const int own_col = 4 * (cblock * CT + threadIdx.x);
  const bool active = own_col < Ch;
  const int col = active ? own_col : 0;   // (the others come along for the end of the block)
  // what does not depend on the sequence is on its way while the slot is looked up
  float w[4][W];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if (W == 4) {
      const float4 v = *reinterpret_cast<const float4*>(p.weight + (i64)(col + c) * W);
      w[c][0] = v.x; w[c][1] = v.y; w[c][W - 2] = v.z; w[c][W - 1] = v.w;
    } else {
#pragma unroll
      for (int k = 0; k < W; ++k) w[c][k] = p.weight[(i64)(col + c) * W + k];
    }
  }
  const float4 bias = p.bias ? make_float4(p.bias[col], p.bias[col + 1], p.bias[col + 2], p.bias[col + 3])
                             : make_float4(0.f, 0.f, 0.f, 0.f);
  float4 step = make_float4(1.f, 1.f, 1.f, 1.f);
  uint32_t* out = nullptr;
  int ow4 = 0;
  if (CODES) {
    int oq;
    if (col < p.D) {
      step = *reinterpret_cast<const float4*>(p.s_x + col);
      out = p.xq; ow4 = p.D / 4; oq = col / 4;
    } else {
      const bool isC = col >= p.D + p.GN;
      const int at = col - p.D - (isC ? p.GN : 0);
      const float a = (isC ? p.s_C : p.s_B)[at / p.N];
      step = make_float4(a, a, a, a);
      out = isC ? p.Cq : p.Bq; ow4 = p.GN / 4; oq = at / 4;
    }
    out += (i64)b * p.L * ow4 + oq;
  }
  int slot, pos;
  if (CODES && threadIdx.x == 0) queue.count = 0;
  const int len = sequence(p, b, cblock == 0 && slab == 0, &slot, &pos);
  if (CODES) __syncthreads();
  float2 w01[W], w23[W];   // taps of channels 0, 1 and 2, 3
  float wsum[4];
#pragma unroll
  for (int k = 0; k < W; ++k) {
    w01[k] = make_float2(w[0][k], w[1][k]);
    w23[k] = make_float2(w[2][k], w[3][k]);
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    wsum[c] = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) wsum[c] += fabsf(w[c][k]);
  }
  const float2 step01 = make_float2(step.x, step.y), step23 = make_float2(step.z, step.w);
  auto normal = [](float x) { return x >= 1e-30f && x <= 1e30f; };
  const bool usable = normal(step.x) && normal(step.y) && normal(step.z) && normal(step.w);
  const float fac[4] = {5.1f * kEps * rcp_approx(step.x), 5.1f * kEps * rcp_approx(step.y), 5.1f * kEps * rcp_approx(step.z),
                        5.1f * kEps * rcp_approx(step.w)};   // 5 eps / step
  const int t0 = slab * p.slab, t1 = min(t0 + p.slab, p.L);
  const int live = active ? min(t1, len) : t0;
  const T* src = p.xBC + b * p.sb + col;
  T* const ring = slot >= 0 ? p.ring + (i64)slot * W * Ch + col : nullptr;
  raw4 past[W - 1];   // the W - 1 tokens ahead
#pragma unroll
  for (int k = 0; k < W - 1; ++k) {
    const int t = t0 - (W - 1) + k;
    past[k] = {};
    if (t0 < live) {
      if (t >= 0) past[k] = load4<T, ALIGNED>(src + t * p.stok);
      else if (ring && pos + t >= 0) past[k] = *reinterpret_cast<const raw4*>(ring + (i64)(((uint32_t)pos + t) % W) * Ch);
    }
  }
  src += t0 * p.stok;
  if (CODES) out += (i64)t0 * ow4;
  // eight tokens from t on; WHOLE: all of them live
  auto eight = [&](auto whole, int t) {
    constexpr bool WHOLE = decltype(whole)::value;
    raw4 raw[CROWS];
#pragma unroll
    for (int u = 0; u < CROWS; ++u) {
      if (!WHOLE) raw[u] = {};
      if (WHOLE || t + u < live) raw[u] = load4<T, ALIGNED>(src + u * p.stok);
    }
    // the nearest to an integer's middle that a quotient may come: 5 eps M / step + (12 + 2 |v|) eps |q| off, M from the largest |x| at
    // hand, |v| <= M, |q| <= 127
    float least[4];
    if (CODES) {
      RawMax<T> top;
#pragma unroll
      for (int k = 0; k < W - 1; ++k) top.add(past[k]);
#pragma unroll
      for (int u = 0; u < CROWS; ++u) top.add(raw[u]);
      const float4 m = top.get();
      const float M[4] = {fmaf(wsum[0], m.x, fabsf(bias.x)), fmaf(wsum[1], m.y, fabsf(bias.y)), fmaf(wsum[2], m.z, fabsf(bias.z)),
                          fmaf(wsum[3], m.w, fabsf(bias.w))};
#pragma unroll
      for (int c = 0; c < 4; ++c) least[c] = fmaf(M[c], -(fac[c] + 2.0f * 127.0f * kEps), 0.5f - 12.0f * 127.0f * kEps);
    }
    float2 h01[W], h23[W];   // the window, oldest first
#pragma unroll
    for (int k = 0; k < W - 1; ++k) {
      const float4 v = Elem<T>::cvt(past[k]);
      h01[k + 1] = make_float2(v.x, v.y);
      h23[k + 1] = make_float2(v.z, v.w);
    }
    uint32_t near = 0;   // bit u: one of the token's quotients comes nearer
#pragma unroll
    for (int u = 0; u < CROWS; ++u) {
      const float4 own = Elem<T>::cvt(raw[u]);
#pragma unroll
      for (int k = 0; k < W - 1; ++k) { h01[k] = h01[k + 1]; h23[k] = h23[k + 1]; }
      h01[W - 1] = make_float2(own.x, own.y);
      h23[W - 1] = make_float2(own.z, own.w);
      float2 v01 = make_float2(bias.x, bias.y), v23 = make_float2(bias.z, bias.w);
#pragma unroll
      for (int k = 0; k < W; ++k) {
        v01 = __ffma2_rn(w01[k], h01[k], v01);
        v23 = __ffma2_rn(w23[k], h23[k], v23);
      }
      const float2 L = make_float2(-1.44269504f, -1.44269504f);
      const float2 a01 = __fmul2_rn(v01, L), a23 = __fmul2_rn(v23, L);
      const float2 e01 = make_float2(ex2_approx(a01.x), ex2_approx(a01.y)), e23 = make_float2(ex2_approx(a23.x), ex2_approx(a23.y));
      const float2 d01 = __ffma2_rn(e01, step01, step01), d23 = __ffma2_rn(e23, step23, step23);   // (1 + e) step
      const float2 p01 = __fmul2_rn(v01, make_float2(rcp_approx(d01.x), rcp_approx(d01.y))), p23 = __fmul2_rn(v23, make_float2(rcp_approx(d23.x), rcp_approx(d23.y)));
      if (CODES) {
        float2 q01, q23;
        asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(q01.x) : "f"(p01.x), "f"(127.0f));
        asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(q01.y) : "f"(p01.y), "f"(127.0f));
        asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(q23.x) : "f"(p23.x), "f"(127.0f));
        asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(q23.y) : "f"(p23.y), "f"(127.0f));
        const float2 mg = make_float2(kMagicOut, kMagicOut), mn = make_float2(-kMagicOut, -kMagicOut), neg = make_float2(-1.f, -1.f);
        const float2 m01 = __fadd2_rn(q01, mg), m23 = __fadd2_rn(q23, mg);
        const float2 f01 = __ffma2_rn(__fadd2_rn(m01, mn), neg, q01), f23 = __ffma2_rn(__fadd2_rn(m23, mn), neg, q23);   // from the integer (exact)
        // (a NaN among the bounds: not below)
        const bool far = fabsf(f01.x) <= least[0] && fabsf(f01.y) <= least[1] && fabsf(f23.x) <= least[2] && fabsf(f23.y) <= least[3];
        if (!far) near |= 1u << u;
        if (WHOLE || t + u < live) out[(i64)u * ow4] = pack4_bits(__float_as_uint(m01.x), __float_as_uint(m01.y), __float_as_uint(m23.x), __float_as_uint(m23.y));
      } else if (WHOLE || t + u < live) {
        *reinterpret_cast<raw4*>(p.out + ((i64)b * p.L + t + u) * Ch + col) = Elem<T>::pack(make_float4(p01.x, p01.y, p23.x, p23.y));
      }
    }
#pragma unroll
    for (int k = 0; k < W - 1; ++k) past[k] = raw[CROWS - (W - 1) + k];
    src += CROWS * p.stok;
    if (CODES) {
      out += (i64)CROWS * ow4;
      if (!usable) near = (1u << CROWS) - 1u;
#pragma unroll 1
      for (; near; near &= near - 1) {
        const int at = t + __ffs(near) - 1;
        if (at >= live) break;
        const int k = atomicAdd(&queue.count, 1);
        if (k < kQueue) queue.item[k] = (uint32_t)(at - t0) << 8 | threadIdx.x;
        else   // (no room: at once)
          for (int c = 0; c < 4; ++c) code_exact<T, W>(p, b, at, col + c, slot, pos);
      }
    }
  };
  int t = t0;
#pragma unroll 1
  for (; t + CROWS <= live; t += CROWS) eight(std::true_type{}, t);
  if (t < live) eight(std::false_type{}, t);
  // (`out` stands behind the last eight tokens that were begun)
  const int begun = t0 + (max(live - t0, 0) + CROWS - 1) / CROWS * CROWS;
  for (t = max(t0, live); t < t1 && active; ++t) {
    if (CODES) out[(i64)(t - begun) * ow4] = 0u;
    else *reinterpret_cast<raw4*>(p.out + ((i64)b * p.L + t) * Ch + col) = Elem<T>::pack(make_float4(0.f, 0.f, 0.f, 0.f));
  }
  if (CODES) {
    __syncthreads();   // (single codes go over the words)
    const int n = 4 * min(queue.count, kQueue);
    for (int k = threadIdx.x; k < n; k += CT) {
      const uint32_t item = queue.item[k >> 2];
      code_exact<T, W>(p, b, t0 + (int)(item >> 8), 4 * (cblock * CT + (int)(item & 255u)) + (k & 3), slot, pos);
    }
    if (ring && slab == 0) __syncthreads();   // (what the ring held before the call has been read)
  }
  // the last W tokens stay in the ring
  if (ring && slab == 0 && active) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      t = len - 1 - k;
      if (t >= 0) *reinterpret_cast<raw4*>(ring + (i64)(((uint32_t)pos + t) % W) * Ch) = load4<T, ALIGNED>(p.xBC + b * p.sb + t * p.stok + col);
    }
  }
}

// the time steps of a slab: a thread has up to four (token, head) pairs at a time
template <typename T>
__device__ __forceinline__ void dt_block(const ConvParams<T>& p, int b, int slab) {
  int slot, pos;
  const int len = sequence(p, b, false, &slot, &pos);
  const int t0 = slab * p.slab, n = (min(t0 + p.slab, p.L) - t0) * p.H;
  const T* src = p.dt_raw + b * p.dt_sb;
  float* dst = p.dt + ((i64)b * p.L + t0) * p.H;
  // (token and head go on by CT pairs without a division)
  int t = threadIdx.x / p.H, hd = threadIdx.x % p.H;
  const int dt = CT / p.H, dh = CT % p.H;
  for (int i0 = threadIdx.x; i0 < n; i0 += 4 * CT) {
    float v[4], o[4];
    bool live[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      live[u] = i0 + u * CT < n && t0 + t < len;
      v[u] = live[u] ? Elem<T>::get(src[(t0 + t) * p.dt_stok + hd]) : 0.f;
      if (p.softplus && p.dt_bias) v[u] = __fadd_rn(v[u], p.dt_bias[hd]);
      o[u] = v[u];
      t += dt;
      hd += dh;
      if (hd >= p.H) { hd -= p.H; ++t; }
    }
    if (p.softplus) softplus_dt<4>(v, 0.f, o);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u * CT < n) dst[i0 + u * CT] = live[u] ? o[u] : 0.f;
  }
}

template <typename T, int W, bool CODES, bool ALIGNED>
__global__ void __launch_bounds__(CT, sizeof(T) == 4 ? 4 : 5) conv_kernel(const __grid_constant__ ConvParams<T> p) {
  pdl_launch_dependents();
  pdl_wait();
  const int nx = p.cblocks + (p.dt ? 1 : 0), cblock = blockIdx.x % nx, at = blockIdx.x / nx;
  const int b = at / p.nslab, slab = at % p.nslab;
  __shared__ Queue queue;
  if (cblock < p.cblocks) conv_block<T, W, CODES, ALIGNED>(p, b, slab, cblock, queue);
  else dt_block(p, b, slab);
}

template <typename T>
ssdi8_status_t launch(const Dims& d, const ssdi8_conv_args_t& a, int width, bool softplus, cudaStream_t st) {
  ConvParams<T> p = {};
  p.xBC = static_cast<const T*>(a.xBC); p.sb = a.stride_b; p.stok = a.stride_t;
  p.weight = a.weight; p.bias = a.bias; p.lens = a.lens; p.slots = a.slots; p.pos = a.pos;
  p.ring = static_cast<T*>(a.ring); p.nslots = a.nslots;
  p.s_x = a.s_x; p.s_B = a.s_B; p.s_C = a.s_C;
  p.xq = reinterpret_cast<uint32_t*>(a.xq); p.Bq = reinterpret_cast<uint32_t*>(a.Bq); p.Cq = reinterpret_cast<uint32_t*>(a.Cq);
  p.out = static_cast<T*>(a.out);
  p.dt_raw = static_cast<const T*>(a.dt_raw); p.dt_sb = a.dt_stride_b; p.dt_stok = a.dt_stride_t;
  p.dt_bias = a.dt_bias; p.dt = a.dt; p.status = a.status;
  p.L = d.L; p.D = d.H * d.P; p.GN = d.G * d.N; p.N = d.N; p.H = d.H; p.softplus = softplus;
  const int Ch = p.D + 2 * p.GN;
  p.cblocks = (Ch / 4 + CT - 1) / CT;
  // Slabs of up to 64 tokens (each reads width - 1 tokens more), shorter where that leaves SMs without a block.
  int slab = 64;
  while (slab > CROWS && (i64)p.cblocks * d.b * ((d.L + slab - 1) / slab) < 4 * 148) slab /= 2;
  p.slab = slab;
  p.nslab = (d.L + slab - 1) / slab;
  const i64 blocks = (i64)(p.cblocks + (a.dt ? 1 : 0)) * d.b * p.nslab;
  if (blocks > 0x7fffffff) return SSDI8_ERR_SHAPE;
  const bool aligned = reinterpret_cast<uintptr_t>(a.xBC) % (4 * sizeof(T)) == 0 && a.stride_b % 4 == 0 && a.stride_t % 4 == 0;
  const dim3 grid((unsigned)blocks);
  auto go = [&](auto kernel) { return launch_configured(kernel, grid, dim3(CT), 0, kStreamCarveout, false, st, p); };
  auto pick = [&](auto w) -> ssdi8_status_t {
    constexpr int W = decltype(w)::value;
    if (a.xq) return aligned ? go(conv_kernel<T, W, true, true>) : go(conv_kernel<T, W, true, false>);
    return aligned ? go(conv_kernel<T, W, false, true>) : go(conv_kernel<T, W, false, false>);
  };
  return width == 4 ? pick(std::integral_constant<int, 4>{}) : width == 3 ? pick(std::integral_constant<int, 3>{})
                                                                          : pick(std::integral_constant<int, 2>{});
}

}  // namespace

ssdi8_status_t launch_conv(const Dims& d, const ssdi8_conv_args_t& a, int dtype, int width, bool softplus, cudaStream_t st) {
  return dtype == 0 ? launch<float>(d, a, width, softplus, st)
       : dtype == 1 ? launch<__half>(d, a, width, softplus, st)
                    : launch<__nv_bfloat16>(d, a, width, softplus, st);
}

}  // namespace ssdi8
