// RMS norm of a row, with the gate of a Mamba-2 block (u = x SiLU(z)), ending in int8 codes: o = u w / sqrt(mean_group u^2 + eps),
// code = rne(o / step), step = absmax(o) / 127 of the row or a given static one.  One pass: a block has a row, every thread keeps its
// u w in registers between the reductions (sum of squares and absmax, one exchange through shared memory) and the codes.
//
// Codes are those of the exact quotient.  With eps = 2^-24, u w is off by at most 12 eps (exponential 5, its argument is compensated;
// 1 + e, reciprocal and the products 1, 2, 1, 1, 1).  In a row of one group with its own step size the norm cancels out of the quotient
// 127 u w / max |u w|: 24 eps of both sides and 4 of the quotient.  Elsewhere 1 / sqrt(mean) adds 24 (21 of the squares and 20 of
// the sum, halved; 3).  A quotient that lies nearer than that to the middle of two integers is formed again in binary64, from the row's
// absmax in binary64 (of the few elements that can be it) and, where it does not cancel, the norm in binary64.  Rows whose sums leave
// binary32's range have all of their codes formed so.
#include "block.cuh"
#include "kernels.h"

namespace ssdi8 {
namespace {

constexpr int kMaxWarps = 16;
constexpr int kMaxChunks = kMaxNormWidth / 128;

struct None {};   // no gate

template <typename T, typename Z>
struct NormParams {
  const T* x; i64 sx;
  const Z* z; i64 sz;
  const float* weight;
  int8_t* xq;
  float* scale;
  const float* static_scale;
  int D, groups, valigned, zaligned;
  float eps;
};

template <typename T>
__device__ __forceinline__ float4 load_row4(const T* p, bool aligned) {
  return Elem<T>::cvt(aligned ? load4<T, true>(p) : load4<T, false>(p));
}

// z / (1 + exp(-z)), 9 eps: ex2's argument as a rounded product and its remainder
__device__ __forceinline__ float silu_compensated(float z) {
  const float L = -1.44269504f, L_LO = -1.92596299e-8f;   // -log2(e) as two numbers
  const float t = z * L;
  const float lo = fmaf(z, L_LO, fmaf(z, L, -t));
  float e = ex2_approx(t);
  // (from 2^127 on the value would be 0 for something that is not: NaN, which sends the row to binary64)
  e = t < 127.0f ? fmaf(e, lo * 0.693147181f, e) : __uint_as_float(0x7fffffffu);
  return z * rcp_approx(1.0f + e);
}

// u w of column i in binary64
template <typename T, typename Z>
__device__ __noinline__ double gated_exact(const NormParams<T, Z>& p, i64 row, int i, double* u) {
  double v = (double)Elem<T>::get(p.x[row * p.sx + i]);
  if constexpr (!std::is_same<Z, None>::value) {
    const double z = (double)Elem<Z>::get(p.z[row * p.sz + i]);
    v *= z / (1.0 + exp(-z));
  }
  *u = v;
  return p.weight ? v * (double)p.weight[i] : v;
}

// NCH chunks of 128 columns per warp: chunk c = warp + k * warps
template <typename T, typename Z, int NCH>
__global__ void __launch_bounds__(32 * kMaxWarps) norm_kernel(const __grid_constant__ NormParams<T, Z> p) {
  constexpr bool GATE = !std::is_same<Z, None>::value;
  __shared__ float part[2][kMaxWarps];
  __shared__ float csum[kMaxChunks], cmax[kMaxChunks];   // of chunks, where the row has several groups
  __shared__ double dsum[kMaxChunks], dmax[kMaxWarps];
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const i64 row = blockIdx.x;
  const int D = p.D, nchunks = (D + 127) / 128, cpg = p.groups > 1 ? nchunks / p.groups : nchunks;
  const bool many = p.groups > 1, dynamic = p.static_scale == nullptr;
  float4 t[NCH];
  float cs[NCH], mx[NCH];
  {
    float4 zv[GATE ? NCH : 1];
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int col = ((warp + k * nwarps) * 32 + lane) * 4;
      t[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (GATE) zv[GATE ? k : 0] = t[k];
      if (col < D) {
        t[k] = load_row4<T>(p.x + row * p.sx + col, p.valigned);
        if constexpr (GATE) zv[k] = load_row4<Z>(p.z + row * p.sz + col, p.zaligned);
      }
    }
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int col = ((warp + k * nwarps) * 32 + lane) * 4;
      if constexpr (GATE) {
        t[k].x *= silu_compensated(zv[k].x);
        t[k].y *= silu_compensated(zv[k].y);
        t[k].z *= silu_compensated(zv[k].z);
        t[k].w *= silu_compensated(zv[k].w);
      }
      cs[k] = fmaf(t[k].x, t[k].x, t[k].y * t[k].y) + fmaf(t[k].z, t[k].z, t[k].w * t[k].w);
      if (p.weight && col < D) {
        const float4 w = *reinterpret_cast<const float4*>(p.weight + col);
        t[k] = make_float4(t[k].x * w.x, t[k].y * w.y, t[k].z * w.z, t[k].w * w.w);
      }
      mx[k] = fmaxf(fmaxf(fabsf(t[k].x), fabsf(t[k].y)), fmaxf(fabsf(t[k].z), fabsf(t[k].w)));
    }
  }
  // sum of squares and absmax of the row, or of its groups (whole chunks each)
  float r = 0.f, rk[NCH], top = 0.f, total = 0.f;   // 1 / sqrt(mean + eps) of the row or of each chunk's group; absmax of o; sum of squares
  bool range = true;                   // the sums are where binary32 is safe
  auto safe = [](float v) { return v > 1e-30f && v < 1e37f; };
  if (!many) {
    float s = cs[0], m = mx[0];
#pragma unroll
    for (int k = 1; k < NCH; ++k) { s += cs[k]; m = fmaxf(m, mx[k]); }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    }
    if (lane == 0) { part[0][warp] = s; part[1][warp] = m; }
    __syncthreads();
    s = lane < nwarps ? part[0][lane] : 0.f;
    m = lane < nwarps ? part[1][lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    }
    range = safe(s) && safe(m);
    total = s;
    r = 1.0f / sqrtf(s / (float)D + p.eps);
    top = m * r;
#pragma unroll
    for (int k = 0; k < NCH; ++k) rk[k] = r;
  } else {
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      float s = cs[k], m = mx[k];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      }
      const int c = warp + k * nwarps;
      if (lane == 0 && c < nchunks) { csum[c] = s; cmax[c] = m; }
    }
    __syncthreads();
    const float n = (float)(cpg * 128);
    for (int g = 0; g < p.groups; ++g) {
      float s = 0.f, m = 0.f;
      for (int c = lane; c < cpg; c += 32) { s += csum[g * cpg + c]; m = fmaxf(m, cmax[g * cpg + c]); }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      }
      const float rg = 1.0f / sqrtf(s / n + p.eps);
      range &= safe(s) && safe(m);
      total += s;
      top = fmaxf(top, m * rg);
#pragma unroll
      for (int k = 0; k < NCH; ++k)
        if ((warp + k * nwarps) / cpg == g) rk[k] = rg;
    }
  }
  const float step = dynamic ? top / 127.0f : *p.static_scale;
  range &= safe(step);
  const float inv = 1.0f / step;
  const float rel = (dynamic ? (many ? 80.f : 28.f) : 42.f) * kEps;
  uint32_t code[NCH];
  uint32_t near = 0;   // bit 4 k + c: the quotient lies near the middle of two integers
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
    const float f = (dynamic && !many) ? 127.0f / (top / r) : rk[k] * inv;
    const float v[4] = {t[k].x, t[k].y, t[k].z, t[k].w};
    float m[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float q;
      asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(q) : "f"(v[c] * f), "f"(127.0f));
      m[c] = __fadd_rn(q, kMagicOut);
      const float off = fabsf(q - __fadd_rn(m[c], -kMagicOut));
      near |= (!(fmaf(rel, fabsf(q), off) <= 0.5f) ? 1u : 0u) << (4 * k + c);
    }
    code[k] = pack4_bits(__float_as_uint(m[0]), __float_as_uint(m[1]), __float_as_uint(m[2]), __float_as_uint(m[3]));
    if (((warp + k * nwarps) * 32 + lane) * 4 >= D) near &= ~(15u << (4 * k));
  }
  float scale_out = step;
  bool exact = __syncthreads_or(near != 0 || !range);
  if (exact && total == 0.f) {
    // a row of zeros (padding) needs none of it; x that underflowed does
    bool any = false;
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int col = ((warp + k * nwarps) * 32 + lane) * 4;
      if (col < D) {
        const float4 v = load_row4<T>(p.x + row * p.sx + col, p.valigned);
        any |= v.x != 0.f || v.y != 0.f || v.z != 0.f || v.w != 0.f;
        code[k] = 0u;
      }
    }
    exact = __syncthreads_or(any);
    if (!exact) scale_out = 1.0f;
  }
  if (exact) {
    // binary64, for what is near (or for all of a row outside the safe range)
    double rd[NCH];
#pragma unroll
    for (int k = 0; k < NCH; ++k) rd[k] = 1.0;
    if (many || !dynamic || !range) {
#pragma unroll 1
      for (int k = 0; k < NCH; ++k) {
        const int c = warp + k * nwarps, col = (c * 32 + lane) * 4;
        double s = 0.0;
        if (col < D)
#pragma unroll 1
          for (int e = 0; e < 4; ++e) {
            double u;
            gated_exact(p, row, col + e, &u);
            s += u * u;
          }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0 && c < nchunks) dsum[c] = s;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < NCH; ++k) {
        const int c = warp + k * nwarps;
        if (c < nchunks) {
          double s = 0.0;
          for (int i = c / cpg * cpg; i < c / cpg * cpg + cpg; ++i) s += dsum[i];
          rd[k] = 1.0 / sqrt(s / (double)(many ? cpg * 128 : D) + (double)p.eps);
        }
      }
    }
    double m64 = 0.0;
    if (dynamic) {
#pragma unroll
      for (int k = 0; k < NCH; ++k) {
        const int col = ((warp + k * nwarps) * 32 + lane) * 4;
        const float v[4] = {t[k].x, t[k].y, t[k].z, t[k].w};
#pragma unroll 1
        for (int e = 0; e < 4; ++e)
          if (col < D && (!range || fabsf(v[e]) * rk[k] >= top * (1.0f - 160.0f * kEps))) {
            double u;
            m64 = fmax(m64, fabs(gated_exact(p, row, col + e, &u) * rd[k]));   // (a NaN counts for nothing)
          }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m64 = fmax(m64, __shfl_xor_sync(0xffffffffu, m64, o));
      if (lane == 0) dmax[warp] = m64;
      __syncthreads();
      for (int i = 0; i < nwarps; ++i) m64 = fmax(m64, dmax[i]);
    }
    const double sd = dynamic ? (m64 > 0.0 ? m64 / 127.0 : 1.0) : (double)*p.static_scale;
    if (!range && dynamic) scale_out = (float)sd;
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int col = ((warp + k * nwarps) * 32 + lane) * 4;
#pragma unroll 1
      for (int e = 0; e < 4; ++e)
        if (col < D && (!range || (near >> (4 * k + e) & 1u))) {
          double u;
          const double v = gated_exact(p, row, col + e, &u) * rd[k];
          const double q = dynamic && m64 > 0.0 ? 127.0 * v / m64 : v / sd;   // (exact ties stay ties)
          const uint32_t c = (uint32_t)__double2int_rn(fmax(fmin(q, 127.0), -127.0)) & 0xffu;   // (fmin(NaN, 127) = 127)
          code[k] = (code[k] & ~(0xffu << (8 * e))) | c << (8 * e);
        }
    }
  }
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
    const int col = ((warp + k * nwarps) * 32 + lane) * 4;
    if (col < D) *reinterpret_cast<uint32_t*>(p.xq + row * D + col) = code[k];
  }
  if (p.scale && threadIdx.x == 0) p.scale[row] = scale_out;
}

template <typename T, typename Z>
ssdi8_status_t launch(const ssdi8_norm_args_t& a, cudaStream_t st) {
  NormParams<T, Z> p = {};
  p.x = static_cast<const T*>(a.x); p.sx = a.stride_x;
  p.z = static_cast<const Z*>(a.z); p.sz = a.stride_z;
  p.weight = a.weight; p.xq = a.xq; p.scale = a.scale; p.static_scale = a.static_scale;
  p.D = a.width; p.groups = a.groups; p.eps = a.eps;
  p.valigned = reinterpret_cast<uintptr_t>(a.x) % (4 * sizeof(T)) == 0 && a.stride_x % 4 == 0;
  p.zaligned = a.z && reinterpret_cast<uintptr_t>(a.z) % (4 * sizeof(Z)) == 0 && a.stride_z % 4 == 0;
  const int chunks = (a.width + 127) / 128;
  auto go = [&](auto n) -> ssdi8_status_t {
    constexpr int NCH = decltype(n)::value;
    return launch_configured(norm_kernel<T, Z, NCH>, dim3((unsigned)a.rows), dim3(32 * ((chunks + NCH - 1) / NCH)), 0, -1, false, st, p);
  };
  if (chunks <= 32) return go(std::integral_constant<int, 2>{});
  if (chunks <= 64) return go(std::integral_constant<int, 5>{});
  return go(std::integral_constant<int, 8>{});
}

template <typename T>
ssdi8_status_t with_gate(const ssdi8_norm_args_t& a, int zdtype, cudaStream_t st) {
  if (!a.z) return launch<T, None>(a, st);
  return zdtype == 0 ? launch<T, float>(a, st) : zdtype == 1 ? launch<T, __half>(a, st) : launch<T, __nv_bfloat16>(a, st);
}

}  // namespace

ssdi8_status_t launch_norm_quantize(const ssdi8_norm_args_t& a, int dtype, int zdtype, cudaStream_t st) {
  return dtype == 0 ? with_gate<float>(a, zdtype, st)
       : dtype == 1 ? with_gate<__half>(a, zdtype, st)
                    : with_gate<__nv_bfloat16>(a, zdtype, st);
}

}  // namespace ssdi8
