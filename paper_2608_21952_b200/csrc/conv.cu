// Causal convolution of a prompt with bias, SiLU and the entry quantiser (Section 4.2, "Quantization of B,C"), and the time
// step beside it.  One pass over xBC: a thread owns four consecutive channels, keeps their taps, step sizes and the last
// width - 1 tokens in registers and walks a slab of tokens, eight loads in flight, so that every element is read once (and
// width - 1 of a slab's tokens once more, from L2) and leaves as one byte.
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

template <typename T, int W, bool CODES, bool ALIGNED>
__device__ __forceinline__ void conv_block(const ConvParams<T>& p, int b, int slab, int cblock) {
  typedef typename Elem<T>::raw4 raw4;
  const int Ch = p.D + 2 * p.GN;
  int slot, pos;
  const int len = sequence(p, b, cblock == 0 && slab == 0, &slot, &pos);
  const int col = 4 * (cblock * CT + threadIdx.x);
  if (col >= Ch) return;
  float2 w01[W], w23[W];   // taps of channels 0, 1 and 2, 3
  float wsum[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    float w[W];
    if (W == 4) {
      const float4 v = *reinterpret_cast<const float4*>(p.weight + (i64)(col + c) * W);
      w[0] = v.x; w[1] = v.y; w[W - 2] = v.z; w[W - 1] = v.w;
    } else {
#pragma unroll
      for (int k = 0; k < W; ++k) w[k] = p.weight[(i64)(col + c) * W + k];
    }
    wsum[c] = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      (c < 2 ? (c == 0 ? w01[k].x : w01[k].y) : (c == 2 ? w23[k].x : w23[k].y)) = w[k];
      wsum[c] += fabsf(w[k]);
    }
  }
  const float4 bias = p.bias ? make_float4(p.bias[col], p.bias[col + 1], p.bias[col + 2], p.bias[col + 3])
                             : make_float4(0.f, 0.f, 0.f, 0.f);
  float4 step = make_float4(1.f, 1.f, 1.f, 1.f), inv = step;
  uint32_t* out = nullptr;
  int ow4 = 0;
  bool usable = true;
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
    inv = make_float4(__frcp_rn(step.x), __frcp_rn(step.y), __frcp_rn(step.z), __frcp_rn(step.w));
    auto normal = [](float x) { return x >= 1e-30f && x <= 1e30f; };
    usable = normal(step.x) && normal(step.y) && normal(step.z) && normal(step.w);
  }
  const int t0 = slab * p.slab, t1 = min(t0 + p.slab, p.L);
  const int live = min(t1, len);
  const T* src = p.xBC + b * p.sb + col;
  T* ring = slot >= 0 ? p.ring + (i64)slot * W * Ch + col : nullptr;
  float4 h[W + CROWS - 1];   // the W - 1 tokens ahead and the eight at hand
#pragma unroll
  for (int k = 0; k < W - 1; ++k) {
    const int t = t0 - (W - 1) + k;
    h[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (t0 < live) {
      if (t >= 0) h[k] = Elem<T>::cvt(load4<T, ALIGNED>(src + t * p.stok));
      else if (ring && pos + t >= 0) h[k] = Elem<T>::cvt(*reinterpret_cast<const raw4*>(ring + (i64)(((uint32_t)pos + t) % W) * Ch));
    }
  }
  // the last W tokens stay in the ring (its rows ahead of this call have been read above, by this very thread: only the first slab does)
  if (ring && slab == 0) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const int t = len - 1 - k;
      if (t >= 0) *reinterpret_cast<raw4*>(ring + (i64)(((uint32_t)pos + t) % W) * Ch) = load4<T, ALIGNED>(src + t * p.stok);
    }
  }
  for (int t = t0; t < live; t += CROWS) {
    raw4 raw[CROWS];
#pragma unroll
    for (int u = 0; u < CROWS; ++u)
      if (t + u < live) raw[u] = load4<T, ALIGNED>(src + (t + u) * p.stok);
    float4 mx = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int u = 0; u < CROWS; ++u) h[W - 1 + u] = t + u < live ? Elem<T>::cvt(raw[u]) : make_float4(0.f, 0.f, 0.f, 0.f);
    float4 d0;   // 5 eps M / step, M from the largest |x| at hand
    if (CODES) {
#pragma unroll
      for (int u = 0; u < W + CROWS - 1; ++u)
        mx = make_float4(fmaxf(mx.x, fabsf(h[u].x)), fmaxf(mx.y, fabsf(h[u].y)), fmaxf(mx.z, fabsf(h[u].z)), fmaxf(mx.w, fabsf(h[u].w)));
      d0 = make_float4(5.f * kEps * fmaf(wsum[0], mx.x, fabsf(bias.x)) * inv.x, 5.f * kEps * fmaf(wsum[1], mx.y, fabsf(bias.y)) * inv.y,
                       5.f * kEps * fmaf(wsum[2], mx.z, fabsf(bias.z)) * inv.z, 5.f * kEps * fmaf(wsum[3], mx.w, fabsf(bias.w)) * inv.w);
    }
#pragma unroll
    for (int u = 0; u < CROWS; ++u) {
      if (t + u < live) {
        float2 v01 = make_float2(bias.x, bias.y), v23 = make_float2(bias.z, bias.w);
#pragma unroll
        for (int k = 0; k < W; ++k) {
          v01 = __ffma2_rn(w01[k], make_float2(h[u + k].x, h[u + k].y), v01);
          v23 = __ffma2_rn(w23[k], make_float2(h[u + k].z, h[u + k].w), v23);
        }
        const float v[4] = {v01.x, v01.y, v23.x, v23.y};
        float s[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) s[c] = v[c] * rcp_approx(1.0f + ex2_approx(v[c] * -1.44269504f));
        if (CODES) {
          const float iv[4] = {inv.x, inv.y, inv.z, inv.w}, dd[4] = {d0.x, d0.y, d0.z, d0.w};
          float m[4];
          bool near[4], any = !usable;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float q = s[c] * iv[c];
            float cl;
            asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(cl) : "f"(q), "f"(127.0f));
            m[c] = __fadd_rn(cl, kMagicOut);
            const float off = fabsf(cl - __fadd_rn(m[c], -kMagicOut));
            near[c] = !(fmaf(fmaf(2.0f * kEps, fabsf(v[c]), 12.0f * kEps), fabsf(cl), off + dd[c]) <= 0.5f) || !usable;
            any |= near[c];
          }
          if (any) {
            const float st[4] = {step.x, step.y, step.z, step.w}, bi[4] = {bias.x, bias.y, bias.z, bias.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              float x[4] = {0.f, 0.f, 0.f, 0.f}, w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int k = 0; k < W; ++k) {
                const float4& hv = h[u + k];
                x[k] = c == 0 ? hv.x : c == 1 ? hv.y : c == 2 ? hv.z : hv.w;
                w[k] = c == 0 ? w01[k].x : c == 1 ? w01[k].y : c == 2 ? w23[k].x : w23[k].y;
              }
              if (near[c])
                m[c] = __uint_as_float(rne_clamp_bits(
                    silu_quotient_exact<W>(x[0], x[1], x[2], x[3], w[0], w[1], w[2], w[3], bi[c], st[c])));
            }
          }
          out[(i64)(t + u) * ow4] = pack4_bits(__float_as_uint(m[0]), __float_as_uint(m[1]), __float_as_uint(m[2]), __float_as_uint(m[3]));
        } else {
          *reinterpret_cast<raw4*>(p.out + ((i64)b * p.L + t + u) * Ch + col) = Elem<T>::pack(make_float4(s[0], s[1], s[2], s[3]));
        }
      }
    }
#pragma unroll
    for (int k = 0; k < W - 1; ++k) h[k] = h[CROWS + k];
  }
  for (int t = max(t0, live); t < t1; ++t) {
    if (CODES) out[(i64)t * ow4] = 0u;
    else *reinterpret_cast<raw4*>(p.out + ((i64)b * p.L + t) * Ch + col) = Elem<T>::pack(make_float4(0.f, 0.f, 0.f, 0.f));
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
  for (int i0 = threadIdx.x; i0 < n; i0 += 4 * CT) {
    float v[4], o[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + u * CT, t = t0 + i / p.H, hd = i % p.H;
      v[u] = i < n && t < len ? Elem<T>::get(src[t * p.dt_stok + hd]) : 0.f;
      if (p.softplus && p.dt_bias) v[u] = __fadd_rn(v[u], p.dt_bias[hd]);
      o[u] = v[u];
    }
    if (p.softplus) softplus_dt<4>(v, 0.f, o);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + u * CT;
      if (i < n) dst[i] = t0 + i / p.H < len ? o[u] : 0.f;
    }
  }
}

template <typename T, int W, bool CODES, bool ALIGNED>
__global__ void __launch_bounds__(CT) conv_kernel(const __grid_constant__ ConvParams<T> p) {
  pdl_launch_dependents();
  pdl_wait();
  const int nx = p.cblocks + (p.dt ? 1 : 0), cblock = blockIdx.x % nx, at = blockIdx.x / nx;
  const int b = at / p.nslab, slab = at % p.nslab;
  if (cblock < p.cblocks) conv_block<T, W, CODES, ALIGNED>(p, b, slab, cblock);
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
