// Causal convolution of a prompt with bias, SiLU and the entry quantiser (Section 4.2, "Quantization of B,C"), and the time
// step beside it.  One pass over xBC: a thread owns two consecutive channels, keeps their taps, step sizes and the last
// width - 1 tokens in registers and walks a slab of tokens, eight loads in flight, so that every element is read once (and
// width - 1 of a slab's tokens once more, from L2) and leaves as one byte.
//
// What bounds it: instructions, with the latencies around them.  8 x 2048 tokens x 80 heads (bf16, 272 MB in and out: 42 us at the copy
// rate) takes 97 us, 60 % of the issue slots, the quarter-rate pipe busy for 46 % of the time (two exponentials and two reciprocals a
// pair).  Without the test whether binary32 may decide a code and without the time steps it takes 77.  Nine blocks of four warps to an
// SM: eight 100, seven 104, six 117, ten 104 us; slabs of 32 tokens 105, of 96 and 128 98 and 101, but 32 and 39 where 64 take 28
// (5 x 1787 tokens x 50 heads, ragged).  One channel a thread, in arithmetic of single elements, took 108.
#include "block.cuh"
#include "kernels.h"

namespace ssdi8 {
namespace {

constexpr int CT = 128;     // threads of a block: 256 channels
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
    if (bad && first_block && threadIdx.x == 0) bad_row(p.status);
  }
  return len;
}

// Two consecutive elements, and the largest magnitude of so many of them: magnitudes are ordered as their bits are.
template <typename T> struct Two;
template <> struct Two<float> {
  typedef float2 raw;
  static __device__ __forceinline__ float2 cvt(const raw& v) { return v; }
  static __device__ __forceinline__ raw pack(const float2& v) { return v; }
  static __device__ __forceinline__ raw most(const raw& m, const raw& v) {
    return make_float2(__uint_as_float(max(__float_as_uint(m.x), __float_as_uint(v.x) & 0x7fffffffu)),
                       __uint_as_float(max(__float_as_uint(m.y), __float_as_uint(v.y) & 0x7fffffffu)));
  }
};
template <> struct Two<__half> {
  typedef uint32_t raw;
  static __device__ __forceinline__ float2 cvt(const raw& v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
  static __device__ __forceinline__ raw pack(const float2& v) {
    const __half2 h = __floats2half2_rn(v.x, v.y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ raw most(const raw& m, const raw& v) { return __vmaxu2(m, v & 0x7fff7fffu); }
};
template <> struct Two<__nv_bfloat16> {
  typedef uint32_t raw;
  static __device__ __forceinline__ float2 cvt(const raw& v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
  static __device__ __forceinline__ raw pack(const float2& v) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ raw most(const raw& m, const raw& v) { return __vmaxu2(m, v & 0x7fff7fffu); }
};
template <typename T, bool ALIGNED>
__device__ __forceinline__ typename Two<T>::raw load2(const T* p) {
  typename Two<T>::raw r;
  if (ALIGNED) {
    r = __ldcs(reinterpret_cast<const typename Two<T>::raw*>(p));
  } else {
    T* e = reinterpret_cast<T*>(&r);
    e[0] = p[0];
    e[1] = p[1];
  }
  return r;
}

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

// Pairs of quotients (a token, two channels) one of which may lie near the middle of two integers: they wait for the end of the
// block, whose threads then have a quotient each.  (Each at once by the lane that met it, its warp waiting, took 119 us
// where the queue took 111, with one channel a thread.)
constexpr int kQueue = 256;
struct Queue {
  uint32_t item[kQueue];   // token of the slab << 8 | thread
  int count;
};

template <typename T, int W, bool CODES, bool ALIGNED>
__device__ __forceinline__ void conv_block(const ConvParams<T>& p, int b, int slab, int cblock, Queue& queue) {
  typedef typename Two<T>::raw raw2;
  const int Ch = p.D + 2 * p.GN;
  const int own_col = 2 * (cblock * CT + threadIdx.x);
  const bool active = own_col < Ch;
  const int col = active ? own_col : 0;   // (the others come along for the end of the block)
  // what does not depend on the sequence is on its way while the slot is looked up
  float w[2][W];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    if (W == 4) {
      const float4 v = *reinterpret_cast<const float4*>(p.weight + (i64)(col + c) * W);
      w[c][0] = v.x; w[c][1] = v.y; w[c][W - 2] = v.z; w[c][W - 1] = v.w;
    } else {
#pragma unroll
      for (int k = 0; k < W; ++k) w[c][k] = p.weight[(i64)(col + c) * W + k];
    }
  }
  const float2 bias = p.bias ? make_float2(p.bias[col], p.bias[col + 1]) : make_float2(0.f, 0.f);
  float2 step = make_float2(1.f, 1.f);
  uint16_t* out = nullptr;
  int ow2 = 0;
  if (CODES) {
    int oq;
    if (col < p.D) {
      step = *reinterpret_cast<const float2*>(p.s_x + col);
      out = reinterpret_cast<uint16_t*>(p.xq); ow2 = p.D / 2; oq = col / 2;
    } else {
      const bool isC = col >= p.D + p.GN;
      const int at = col - p.D - (isC ? p.GN : 0);
      const float a = (isC ? p.s_C : p.s_B)[at / p.N];
      step = make_float2(a, a);
      out = reinterpret_cast<uint16_t*>(isC ? p.Cq : p.Bq); ow2 = p.GN / 2; oq = at / 2;
    }
    out += (i64)b * p.L * ow2 + oq;
  }
  int slot, pos;
  if (CODES && threadIdx.x == 0) queue.count = 0;
  const int len = sequence(p, b, cblock == 0 && slab == 0, &slot, &pos);
  if (CODES) __syncthreads();
  float2 wk[W];
  float wsum[2] = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < W; ++k) {
    wk[k] = make_float2(w[0][k], w[1][k]);
    wsum[0] += fabsf(w[0][k]);
    wsum[1] += fabsf(w[1][k]);
  }
  auto normal = [](float x) { return x >= 1e-30f && x <= 1e30f; };
  const bool usable = normal(step.x) && normal(step.y);
  const float fac[2] = {5.1f * kEps * rcp_approx(step.x), 5.1f * kEps * rcp_approx(step.y)};   // 5 eps / step
  const int t0 = slab * p.slab, t1 = min(t0 + p.slab, p.L);
  const int live = active ? min(t1, len) : t0;
  const T* src = p.xBC + b * p.sb + col;
  T* const ring = slot >= 0 ? p.ring + (i64)slot * W * Ch + col : nullptr;
  raw2 past[W - 1];   // the W - 1 tokens ahead
#pragma unroll
  for (int k = 0; k < W - 1; ++k) {
    const int t = t0 - (W - 1) + k;
    past[k] = {};
    if (t0 < live) {
      if (t >= 0) past[k] = load2<T, ALIGNED>(src + t * p.stok);
      else if (ring && pos + t >= 0) past[k] = *reinterpret_cast<const raw2*>(ring + (i64)(((uint32_t)pos + t) % W) * Ch);
    }
  }
  src += t0 * p.stok;
  if (CODES) out += (i64)t0 * ow2;
  // eight tokens from t on; WHOLE: all of them live
  auto eight = [&](auto whole, int t) {
    constexpr bool WHOLE = decltype(whole)::value;
    raw2 raw[CROWS];
#pragma unroll
    for (int u = 0; u < CROWS; ++u) {
      if (!WHOLE) raw[u] = {};
      if (WHOLE || t + u < live) raw[u] = load2<T, ALIGNED>(src + u * p.stok);
    }
    // the nearest to an integer's middle that a quotient may come, M from the largest |x| at hand and |q| <= 127: 5 eps M / step of the
    // convolution; of the exponential's argument 1.5 |v| eps, which reaches the quotient times 1 - sigmoid, v^2 sigmoid (1 - sigmoid) being
    // below 0.44: 0.7 eps / step; of the other operations 8 eps |q| (the exponential 4, 1 + e with the step size 1, reciprocal 2, product 1)
    float least[2];
    if (CODES) {
      raw2 top = {};
#pragma unroll
      for (int k = 0; k < W - 1; ++k) top = Two<T>::most(top, past[k]);
#pragma unroll
      for (int u = 0; u < CROWS; ++u) top = Two<T>::most(top, raw[u]);
      const float2 m = Two<T>::cvt(top);
      const float M[2] = {fmaf(wsum[0], m.x, fabsf(bias.x)), fmaf(wsum[1], m.y, fabsf(bias.y))};
#pragma unroll
      for (int c = 0; c < 2; ++c) least[c] = fmaf(M[c] + 0.2f, -fac[c], 0.5f - 8.5f * 127.0f * kEps);
    }
    float2 h[W];   // the window, oldest first
#pragma unroll
    for (int k = 0; k < W - 1; ++k) h[k + 1] = Two<T>::cvt(past[k]);
    uint32_t near = 0;   // bit u: one of the token's quotients comes nearer
#pragma unroll
    for (int u = 0; u < CROWS; ++u) {
#pragma unroll
      for (int k = 0; k < W - 1; ++k) h[k] = h[k + 1];
      h[W - 1] = Two<T>::cvt(raw[u]);
      float2 v = bias;
#pragma unroll
      for (int k = 0; k < W; ++k) v = __ffma2_rn(wk[k], h[k], v);
      const float2 a = __fmul2_rn(v, make_float2(-1.44269504f, -1.44269504f));
      const float2 d = __ffma2_rn(make_float2(ex2_approx(a.x), ex2_approx(a.y)), step, step);   // (1 + e) step
      const float2 r = __fmul2_rn(v, make_float2(rcp_approx(d.x), rcp_approx(d.y)));
      if (CODES) {
        float2 q;
        asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(q.x) : "f"(r.x), "f"(127.0f));
        asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(q.y) : "f"(r.y), "f"(127.0f));
        const float2 m = __fadd2_rn(q, make_float2(kMagicOut, kMagicOut));
        const float2 f = __ffma2_rn(__fadd2_rn(m, make_float2(-kMagicOut, -kMagicOut)), make_float2(-1.f, -1.f), q);   // from the integer (exact)
        // (a NaN among the bounds: not below)
        if (!(fabsf(f.x) <= least[0] && fabsf(f.y) <= least[1])) near |= 1u << u;
        if (WHOLE || t + u < live) out[(i64)u * ow2] = (uint16_t)__byte_perm(__float_as_uint(m.x), __float_as_uint(m.y), 0x0040u);
      } else if (WHOLE || t + u < live) {
        *reinterpret_cast<raw2*>(p.out + ((i64)b * p.L + t + u) * Ch + col) = Two<T>::pack(r);
      }
    }
#pragma unroll
    for (int k = 0; k < W - 1; ++k) past[k] = raw[CROWS - (W - 1) + k];
    src += CROWS * p.stok;
    if (CODES) {
      out += (i64)CROWS * ow2;
      if (!usable) near = (1u << CROWS) - 1u;   // (all: the block's queue runs over)
#pragma unroll 1
      for (; near; near &= near - 1) {
        const int at = t + __ffs(near) - 1;
        if (at >= live) break;
        const int k = atomicAdd(&queue.count, 1);
        if (k < kQueue) queue.item[k] = (uint32_t)(at - t0) << 8 | threadIdx.x;
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
    if (CODES) out[(i64)(t - begun) * ow2] = 0;
    else *reinterpret_cast<raw2*>(p.out + ((i64)b * p.L + t) * Ch + col) = Two<T>::pack(make_float2(0.f, 0.f));
  }
  if (CODES) {
    __syncthreads();   // (single codes go over the pairs)
    if (queue.count <= kQueue) {
      const int n = 2 * queue.count;
      for (int k = threadIdx.x; k < n; k += CT) {
        const uint32_t item = queue.item[k >> 1];
        code_exact<T, W>(p, b, t0 + (int)(item >> 8), 2 * (cblock * CT + (int)(item & 255u)) + (k & 1), slot, pos);
      }
    } else {   // more than that, as with step sizes outside the normal range: all of the block
      const int end = min(t1, len), first = 2 * cblock * CT;
#pragma unroll 1
      for (t = t0; t < end; ++t)
        for (int k = threadIdx.x; k < 2 * CT; k += CT)
          if (first + k < Ch) code_exact<T, W>(p, b, t, first + k, slot, pos);
    }
    if (ring && slab == 0) __syncthreads();   // (what the ring held before the call has been read)
  }
  // the last W tokens stay in the ring
  if (ring && slab == 0 && active) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      t = len - 1 - k;
      if (t >= 0) *reinterpret_cast<raw2*>(ring + (i64)(((uint32_t)pos + t) % W) * Ch) = load2<T, ALIGNED>(p.xBC + b * p.sb + t * p.stok + col);
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
__global__ void __launch_bounds__(CT, 9) conv_kernel(const __grid_constant__ ConvParams<T> p) {
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
  p.cblocks = (Ch / 2 + CT - 1) / CT;
  // Slabs of up to 64 tokens (each reads width - 1 tokens more), shorter where that leaves SMs without a block.
  int slab = 64;
  while (slab > CROWS && (i64)p.cblocks * d.b * ((d.L + slab - 1) / slab) < 4 * 148) slab /= 2;
  p.slab = slab;
  p.nslab = (d.L + slab - 1) / slab;
  const i64 blocks = (i64)(p.cblocks + (a.dt ? 1 : 0)) * d.b * p.nslab;
  if (blocks > 0x7fffffff) return SSDI8_ERR_SHAPE;
  const bool aligned = reinterpret_cast<uintptr_t>(a.xBC) % (2 * sizeof(T)) == 0 && a.stride_b % 2 == 0 && a.stride_t % 2 == 0;
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
