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
// Such quotients are few, but one sends its row to binary64, whose norm (groups, static steps) is formed from all of the row's elements, one after
// the other by each thread: of rows of 5120 in one group 2 % go there, with a static step 13 to 20 %, of rows of 8192 in 8 groups 11 to 17 %, with a
// static step 25 % (normal values and 1 % outliers of 20, with the gate and without).  That is what bounds these: 16384 x 5120 with a
// static step 219 us, 10000 x 8192 in 8 groups (fp32 and a bf16 gate, 89 us of bytes) 305, both 358; and of 64 x 5120 (bf16, gated), 8.1 us on
// the device where a row of the 64 goes there (11 of 16 draws) and 2.7 where none does.
//
// What bounds the others: 16384 rows of 5120 (fp32 and a bf16 gate, 587 MB: 91 us at the copy rate) take 122 to 129 us: 30 instructions an element, two of them
// on the quarter-rate pipe (the exponential and the reciprocal), with three to five blocks to an SM (80 registers; 64 take 129 us with five
// chunks to a warp, 48 spill: 140).
// Codes and exact path in one body took 292 us, one element after the other; pairs, with the exact path out of line, 144; chunks of a warp side
// by side 135.
#include "block.cuh"
#include "kernels.h"

namespace ssdi8 {
namespace {

constexpr int kMaxWarps = 16;
constexpr int kMaxChunks = kMaxNormWidth / 128;

struct None {};   // no gate
template <typename Z> struct GateRaw { typedef typename Elem<Z>::raw4 raw4; };
template <> struct GateRaw<None> { struct raw4 {}; };

template <typename T, typename Z>
struct NormParams {
  const T* x; i64 sx;
  const Z* z; i64 sz;
  const float* weight;
  int8_t* xq;
  float* scale;
  const float* static_scale;
  int D, groups, valigned, zaligned, fast;
  float eps;
};

template <typename T>
__device__ __forceinline__ typename Elem<T>::raw4 load_row4(const T* p, bool aligned) {
  return aligned ? load4<T, true>(p) : load4<T, false>(p);
}
template <>
__device__ __forceinline__ float4 load_row4<float>(const float* p, bool aligned) {
  return aligned ? load4<float, true>(p) : load4<float, false>(p);
}

// z / (1 + exp(-z)) of two, 9 eps: ex2's argument as a rounded product and its remainder.  Not for z below kLeastGate, where exp(-z)
// leaves binary32's range.
constexpr float kLeastGate = -86.0f;
__device__ __forceinline__ float2 silu2(float2 z) {
  auto both = [](float v) { return make_float2(v, v); };
  const float2 L = both(-1.44269504f), t = __fmul2_rn(z, L);   // -log2(e) z; its rest below, times ln 2
  const float2 rest = __ffma2_rn(z, both(-1.33497567e-8f), __fmul2_rn(__ffma2_rn(z, L, make_float2(-t.x, -t.y)), both(0.693147181f)));
  const float2 e = make_float2(ex2_approx(t.x), ex2_approx(t.y));
  const float2 d = __fadd2_rn(__ffma2_rn(e, rest, e), both(1.0f));
  return __fmul2_rn(z, make_float2(rcp_approx(d.x), rcp_approx(d.y)));
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

// Codes of a row in binary64: those of the chunks in `near`, or all of them (and the row's step size) if the row is out of binary32's range
// (one with a group of zeros is).
// The absmax in binary64 is that of the chunks in `cand`.  All threads call it, behind their stores.
// In a row of several groups the quotient is 127 v / v_m times the ratio of the two norms: 1 in the group of the absmax, where ties stay ties.
struct Top {
  double o, v, r;   // |u w| r, |u w|, r = 1 / sqrt(mean + eps)
};
template <typename T, typename Z, int NCH>
__device__ __noinline__ void exact_row(const NormParams<T, Z>& p, i64 row, uint32_t near, uint32_t cand, bool range, bool zero, double* sum64,
                                       Top* top64) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const int D = p.D, nchunks = (D + 127) / 128, cpg = p.groups > 1 ? nchunks / p.groups : nchunks;
  const bool many = p.groups > 1, dynamic = p.static_scale == nullptr;
  const int c0 = warp * NCH;   // this warp's chunks
  auto col_of = [&](int k) { return ((c0 + k) * 32 + lane) * 4; };
  if (zero) {
    // a row of zeros (padding) needs none of it; x that underflowed does, and so does 0 times a weight or over a step that makes it NaN
    bool any = !dynamic && !(fabsf(*p.static_scale) > 0.f);
#pragma unroll 1
    for (int k = 0; k < NCH; ++k)
      if (col_of(k) < D) {
        const float4 v = Elem<T>::cvt(load_row4<T>(p.x + row * p.sx + col_of(k), p.valigned));
        any |= v.x != 0.f || v.y != 0.f || v.z != 0.f || v.w != 0.f;
        if (p.weight) {
          const float4 w = *reinterpret_cast<const float4*>(p.weight + col_of(k));
          any |= !(0.f * w.x + 0.f * w.y + 0.f * w.z + 0.f * w.w == 0.f);
        }
      }
    if (!__syncthreads_or(any)) {
#pragma unroll 1
      for (int k = 0; k < NCH; ++k)
        if (col_of(k) < D) *reinterpret_cast<uint32_t*>(p.xq + row * D + col_of(k)) = 0u;
      if (dynamic && p.scale && threadIdx.x == 0) p.scale[row] = 1.0f;
      return;
    }
  }
  const bool norms = many || !dynamic || !range;
  if (norms) {
#pragma unroll 1
    for (int k = 0; k < NCH; ++k) {
      double s = 0.0;
      if (col_of(k) < D)
#pragma unroll 1
        for (int e = 0; e < 4; ++e) {
          double u;
          gated_exact(p, row, col_of(k) + e, &u);
          s += u * u;
        }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (lane == 0 && c0 + k < nchunks) sum64[c0 + k] = s;
    }
    __syncthreads();
  }
  auto rnorm = [&](int k) {   // 1 / sqrt(mean + eps) of chunk k's group, or 1 where it cancels
    const int c = c0 + k;
    if (!norms || c >= nchunks) return 1.0;
    double s = 0.0;
    for (int i = c / cpg * cpg; i < c / cpg * cpg + cpg; ++i) s += sum64[i];
    const double m = s / (double)(many ? cpg * 128 : D) + (double)p.eps;
    return m == 0.0 ? 0.0 : 1.0 / sqrt(m);   // (zeros without eps: o = 0)
  };
  Top m = {0.0, 0.0, 1.0};
  if (dynamic) {
#pragma unroll 1
    for (int k = 0; k < NCH; ++k)
      if (col_of(k) < D && (!range || (cand >> k & 1u))) {
        const double r = rnorm(k);
#pragma unroll 1
        for (int e = 0; e < 4; ++e) {
          double u;
          const double v = fabs(gated_exact(p, row, col_of(k) + e, &u));
          if (v * r > m.o) m = {v * r, v, r};   // (a NaN counts for nothing)
        }
      }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const Top t = {__shfl_xor_sync(0xffffffffu, m.o, o), __shfl_xor_sync(0xffffffffu, m.v, o), __shfl_xor_sync(0xffffffffu, m.r, o)};
      if (t.o > m.o) m = t;
    }
    if (lane == 0) top64[warp] = m;
    __syncthreads();
    m = top64[0];   // (the same of equal ones for all threads)
    for (int i = 1; i < nwarps; ++i)
      if (top64[i].o > m.o) m = top64[i];
    if (!range && p.scale && threadIdx.x == 0) p.scale[row] = m.o > 0.0 ? (float)(m.o / 127.0) : 1.0f;
  }
#pragma unroll 1
  for (int k = 0; k < NCH; ++k)
    if (col_of(k) < D && (!range || (near >> k & 1u))) {
      const double r = rnorm(k);
#pragma unroll 1
      for (int e = 0; e < 4; ++e) {
        double u;
        const double v = gated_exact(p, row, col_of(k) + e, &u);
        const double q = !dynamic ? v * r / (double)*p.static_scale : m.o > 0.0 ? 127.0 * v / m.v * (r / m.r) : v * r;
        p.xq[row * D + col_of(k) + e] = (int8_t)__double2int_rn(fmax(fmin(q, 127.0), -127.0));        // (fmin(NaN, 127) = 127)
      }
    }
}

// u w of a warp's chunks, their sums of u^2 and absmax.  ALL: every chunk lies in the row and is aligned, so loads stand at fixed
// distances from one address.
template <typename T, typename Z, int NCH, bool ALL>
__device__ __forceinline__ void row_values(const NormParams<T, Z>& p, i64 row, int col0, float2 (&t)[NCH][2], float (&cs)[NCH], float (&mx)[NCH]) {
  constexpr bool GATE = !std::is_same<Z, None>::value;
  const T* const x = p.x + row * p.sx + col0;
  const float* const w = p.weight + col0;
  typename Elem<T>::raw4 xr[NCH];
  typename GateRaw<Z>::raw4 zr[NCH];
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
    xr[k] = {};
    zr[k] = {};
    if (ALL || col0 + 128 * k < p.D) {
      xr[k] = load_row4<T>(x + 128 * k, ALL || p.valigned);
      if constexpr (GATE) zr[k] = load_row4<Z>(p.z + row * p.sz + col0 + 128 * k, ALL || p.zaligned);
    }
  }
  float least = 0.f;
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
    const float4 v = Elem<T>::cvt(xr[k]);
    t[k][0] = make_float2(v.x, v.y);
    t[k][1] = make_float2(v.z, v.w);
    if constexpr (GATE) {
      const float4 z = Elem<Z>::cvt(zr[k]);
      least = fminf(fminf(least, fminf(z.x, z.y)), fminf(z.z, z.w));   // (a NaN shows in the sums)
      t[k][0] = __fmul2_rn(t[k][0], silu2(make_float2(z.x, z.y)));
      t[k][1] = __fmul2_rn(t[k][1], silu2(make_float2(z.z, z.w)));
    }
    const float2 sq = __ffma2_rn(t[k][0], t[k][0], __fmul2_rn(t[k][1], t[k][1]));
    cs[k] = sq.x + sq.y;
    if (p.weight && (ALL || col0 + 128 * k < p.D)) {
      const float4 f = *reinterpret_cast<const float4*>(w + 128 * k);
      t[k][0] = __fmul2_rn(t[k][0], make_float2(f.x, f.y));
      t[k][1] = __fmul2_rn(t[k][1], make_float2(f.z, f.w));
    }
    mx[k] = fmaxf(fmaxf(fabsf(t[k][0].x), fabsf(t[k][0].y)), fmaxf(fabsf(t[k][1].x), fabsf(t[k][1].y)));
  }
  if (least < kLeastGate) cs[0] = __uint_as_float(0x7fffffffu);   // (sends the row to binary64)
}

__device__ __forceinline__ float warp_max(float v) {   // of numbers >= 0; a NaN counts for nothing
  float m;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
  return m;
}

// A warp has NCH chunks of 128 columns, one after the other; WARPS at most.
template <typename T, typename Z, int NCH, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, WARPS == 16 ? 1 : NCH == 2 ? 4 : 3) norm_kernel(const __grid_constant__ NormParams<T, Z> p) {
  __shared__ struct {
    float part[2][kMaxWarps];
    float csum[kMaxChunks], cmax[kMaxChunks];   // of chunks, where the row has several groups
    double sum64[kMaxChunks];
    Top top64[kMaxWarps];
  } S;
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const i64 row = blockIdx.x;
  const int D = p.D, nchunks = (D + 127) / 128, c0 = warp * NCH, col0 = (c0 * 32 + lane) * 4;
  const bool many = p.groups > 1, dynamic = p.static_scale == nullptr, all = p.fast && (c0 + NCH) * 128 <= D;
  float2 t[NCH][2];
  float cs[NCH], mx[NCH];
  if (all) row_values<T, Z, NCH, true>(p, row, col0, t, cs, mx);
  else row_values<T, Z, NCH, false>(p, row, col0, t, cs, mx);
  // sum of squares and absmax of the row, or of its groups (whole chunks each)
  float r = 0.f, rk[NCH], top = 0.f, total = 0.f;   // 1 / sqrt(mean + eps) of the row (or its groups' largest) or of each chunk's group; absmax of o; sum of squares
  bool range = true;                                // the sums are where binary32 is safe
  auto safe = [](float v) { return v > 1e-30f && v < 1e37f; };
  if (!many) {
    float s = cs[0], m = mx[0];
#pragma unroll
    for (int k = 1; k < NCH; ++k) { s += cs[k]; m = fmaxf(m, mx[k]); }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    m = warp_max(m);
    if (lane == 0) { S.part[0][warp] = s; S.part[1][warp] = m; }
    __syncthreads();
    s = (lane & 15) < nwarps ? S.part[0][lane & 15] : 0.f;
    m = lane < nwarps ? S.part[1][lane] : 0.f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    m = warp_max(m);
    range = safe(s) && safe(m);
    total = s;
    r = 1.0f / sqrtf(s / (float)D + p.eps);
    top = m * r;
#pragma unroll
    for (int k = 0; k < NCH; ++k) rk[k] = r;
  } else {
    const int cpg = nchunks / p.groups;
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      float s = cs[k];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      const float m = warp_max(mx[k]);
      if (lane == 0 && c0 + k < nchunks) { S.csum[c0 + k] = s; S.cmax[c0 + k] = m; }
      rk[k] = 0.f;
    }
    __syncthreads();
    const float n = (float)(cpg * 128);
    for (int g = 0; g < p.groups; ++g) {
      float s = 0.f, m = 0.f;
      for (int c = lane; c < cpg; c += 32) { s += S.csum[g * cpg + c]; m = fmaxf(m, S.cmax[g * cpg + c]); }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      m = warp_max(m);
      const float rg = 1.0f / sqrtf(s / n + p.eps);
      range &= safe(s) && safe(m);
      total += s;
      top = fmaxf(top, m * rg);
      r = fmaxf(r, rg);
#pragma unroll
      for (int k = 0; k < NCH; ++k)
        if (c0 + k >= g * cpg && c0 + k < (g + 1) * cpg) rk[k] = rg;
    }
  }
  const float step = dynamic ? top / 127.0f : *p.static_scale;
  const float inv = 1.0f / step;
  range &= safe(step) && r * inv < 1e37f;   // (a larger factor could make infinities of products that are subnormal)
  const float rel = (dynamic ? (many ? 80.f : 28.f) : 42.f) * kEps;
  const float f_row = 127.0f / (top / r);
  uint32_t near = 0, cand = 0;   // bit k: one of the four quotients lies near the middle of two integers; one element can be the row's absmax
  int8_t* const xq = p.xq + row * D + col0;
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
    const float f = dynamic && !many ? f_row : rk[k] * inv;
    const float2 v0 = __fmul2_rn(t[k][0], make_float2(f, f)), v1 = __fmul2_rn(t[k][1], make_float2(f, f));
    float2 q0, q1;
    asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(q0.x) : "f"(v0.x), "f"(127.0f));
    asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(q0.y) : "f"(v0.y), "f"(127.0f));
    asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(q1.x) : "f"(v1.x), "f"(127.0f));
    asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(q1.y) : "f"(v1.y), "f"(127.0f));
    const float2 mg = make_float2(kMagicOut, kMagicOut), mn = make_float2(-kMagicOut, -kMagicOut);
    const float2 m0 = __fadd2_rn(q0, mg), m1 = __fadd2_rn(q1, mg);
    const float2 i0 = __fadd2_rn(m0, mn), i1 = __fadd2_rn(m1, mn);
    // how far from the integer, and how far off at most
    const float a = fmaf(rel, fabsf(q0.x), fabsf(q0.x - i0.x)), b = fmaf(rel, fabsf(q0.y), fabsf(q0.y - i0.y));
    const float c = fmaf(rel, fabsf(q1.x), fabsf(q1.x - i1.x)), d = fmaf(rel, fabsf(q1.y), fabsf(q1.y - i1.y));
    const uint32_t code = pack4_bits(__float_as_uint(m0.x), __float_as_uint(m0.y), __float_as_uint(m1.x), __float_as_uint(m1.y));
    if (all || col0 + 128 * k < D) {
      if (!(fmaxf(fmaxf(a, b), fmaxf(c, d)) <= 0.5f)) near |= 1u << k;   // (rows with a NaN are out of range)
      if (mx[k] * rk[k] >= top * (1.0f - 160.0f * kEps)) cand |= 1u << k;
      *reinterpret_cast<uint32_t*>(xq + 128 * k) = code;
    }
  }
  if (dynamic && p.scale && threadIdx.x == 0) p.scale[row] = step;
  if (__syncthreads_or(near != 0 || !range)) exact_row<T, Z, NCH>(p, row, near, cand, range, total == 0.f, S.sum64, S.top64);
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
  p.fast = p.valigned && (!a.z || p.zaligned);
  const int chunks = (a.width + 127) / 128;
  auto go = [&](auto n, auto warps) -> ssdi8_status_t {
    constexpr int NCH = decltype(n)::value, WARPS = decltype(warps)::value;
    return launch_configured(norm_kernel<T, Z, NCH, WARPS>, dim3((unsigned)a.rows), dim3(32 * ((chunks + NCH - 1) / NCH)), 0, -1, false, st, p);
  };
  typedef std::integral_constant<int, 2> Two;
  typedef std::integral_constant<int, 5> Five;
  typedef std::integral_constant<int, 8> Eight;
  typedef std::integral_constant<int, 16> Sixteen;
  // Few rows want many warps, many rows few warps with much each: a warp's share of the reductions is the same for two chunks as for
  // eight (fp32 and a bf16 gate, us with 2, 5, 8 chunks to a warp: 600 rows of 2048 8.2, 9.3, 9.9, of 5120 -, 11.1, 11.4; 4096 rows
  // of 512 9.9, 11.3, 12.4, of 2048 22.8, 20.9, 18.8, of 2560 28.7, 21.6, 24.3, of 4096 44.5, 37.3, 29.5, of 8192 -, 70.5, 55.2).  Five
  // where eight leave more of the last warp idle.
  if (chunks > 64) return go(Eight(), Sixteen());
  const bool few = a.rows <= 1024;
  if (chunks <= 4 || (few && chunks <= 16)) return go(Two(), Eight());
  if (chunks <= 40 && (few || (chunks + 4) / 5 * 5 < (chunks + 7) / 8 * 8)) return go(Five(), Eight());
  return go(Eight(), Eight());
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
