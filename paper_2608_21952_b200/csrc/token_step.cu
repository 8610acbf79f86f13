// One token for every sequence over the 8-bit state cache: convolution, codes of x, B and C, time step, y, and the token put into
// the slot's window.  The state is read once, as codes, and not written: with the tokens since its last fold beside it,
//   y = s_C (E scale sum_n C q + s_x s_B sum_j w_j (C . B_j) x_j) + D s_x x + corr,   E = exp(A sum dt), w_j = dt_j exp(A sum behind j)
// (ChunkScan1 and ChunkScan2 of Algorithm 2 for a single row, with int8 dot products), a quarter of the fp32 state's bytes one way
// instead of two.  Once in 16 tokens the full window is folded into the codes, in binary64.
#include "kernels.h"
#include "state_cache.cuh"

namespace ssdi8 {
namespace {

constexpr int TS_T = 256;

template <typename T>
struct TokenParams {
  CacheView c;
  T* ring; int width;
  const T* xBC; i64 sb;
  const float* weight; const float* bias;
  const T* dt_raw; i64 dt_sb;
  const float *dt_bias, *A, *D, *corr, *s_x, *s_B, *s_C;
  const int32_t *slots, *pos;
  void* y; int32_t* status;
  int H, G, softplus, ydt, hblocks;   // hblocks: blocks per group of heads
};

// code of one channel of the token: taps from the ring and the token itself, which goes into the ring
template <typename T>
__device__ __forceinline__ int channel(const TokenParams<T>& p, const T* x, T* ring, int Ch, int ch, int pos, float step, bool keep) {
  const int W = p.width;
  float xs[4], w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {   // taps 4 - W .. 3 are the convolution's
    const int t = pos - 3 + k;
    xs[k] = w[k] = 0.f;
    if (k == 3) xs[k] = Elem<T>::get(x[ch]);
    else if (k >= 4 - W && t >= 0) xs[k] = Elem<T>::get(ring[(i64)((uint32_t)t % (uint32_t)W) * Ch + ch]);
  }
  if (W == 4) {
    const float4 v = *reinterpret_cast<const float4*>(p.weight + (i64)ch * 4);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  } else {
#pragma unroll
    for (int k = 1; k < 4; ++k)
      if (k >= 4 - W) w[k] = p.weight[(i64)ch * W + k - 4 + W];
  }
  const float bias = p.bias ? p.bias[ch] : 0.f;
  if (keep) ring[(i64)((uint32_t)pos % (uint32_t)W) * Ch + ch] = x[ch];
  float v = bias, m = fabsf(bias);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v = fmaf(w[k], xs[k], v);
    m = fmaf(fabsf(w[k]), fabsf(xs[k]), m);
  }
  const float inv = __frcp_rn(step);
  const float q = v * rcp_approx(1.0f + ex2_approx(v * -1.44269504f)) * inv;
  float cl;
  asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(cl) : "f"(q), "f"(127.0f));
  float r = __fadd_rn(cl, kMagicOut);
  const float off = fabsf(cl - __fadd_rn(r, -kMagicOut));
  // (see block.cuh; M is the token's own here)
  if (!(fmaf(fmaf(2.0f * kEps, fabsf(v), 12.0f * kEps), fabsf(cl), fmaf(5.0f * kEps * m, inv, off)) <= 0.5f) || !(step >= 1e-30f && step <= 1e30f))
    r = __uint_as_float(rne_clamp_bits(silu_quotient_exact<4>(xs[0], xs[1], xs[2], xs[3], w[0], w[1], w[2], w[3], bias, step)));
  return (int)(int8_t)(__float_as_uint(r) & 0xffu);
}

__device__ __forceinline__ int dot16(const uint4& a, const uint4& b) {
  int s = __dp4a((int)a.x, (int)b.x, 0);
  s = __dp4a((int)a.y, (int)b.y, s);
  s = __dp4a((int)a.z, (int)b.z, s);
  return __dp4a((int)a.w, (int)b.w, s);
}

template <int N, int HPC>
struct TokenSmem {
  __align__(16) int8_t C[N];
  __align__(16) int8_t B[N];
  __align__(16) int8_t x[HPC][kWin][64];   // x of the window, rows as in the cache
  int CB[kWin];                            // C . B_j
  float w[HPC][kWin], E[HPC];
  double wd[HPC][kWin], Ed[HPC];           // the same in binary64, for a fold
  __align__(16) double xw[kWin][64];       // operands of a fold
  __align__(16) double Bd[kWin][N];
};

// A block has up to HPC heads of one group: the convolution of B and C is theirs together.  A thread holds 16 codes of a row at a
// time: N / 16 lanes per row.
template <typename T, int N, int HPC>
__global__ void __launch_bounds__(TS_T) token_kernel(const __grid_constant__ TokenParams<T> p) {
  constexpr int LPR = N / 16, RPP = TS_T / LPR, R = 64 / RPP;   // lanes per row, rows per pass, passes per head
  __shared__ TokenSmem<N, HPC> s;
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int hb = blockIdx.x % p.hblocks, bg = blockIdx.x / p.hblocks, g = bg % p.G, b = bg / p.G;
  const int hpg = p.H / p.G, h0 = g * hpg + hb * HPC, nh = min(HPC, hpg - hb * HPC);
  bool bad;
  const int slot = slot_of(p.slots, p.pos, p.c.nslots, b, &bad);
  int pos = 0, f = 0;
  if (slot >= 0) {
    pos = p.pos[b];
    f = max(p.c.start[slot], pos - pos % kWin);
    bad = f > pos;
  }
  if (bad && hb == 0 && g == 0 && tid == 0 && p.status) atomicExch(p.status, (int32_t)SSDI8_ERR_SHAPE);
  if (slot < 0 || bad) return;
  const int now = pos % kWin;
  const i64 sh0 = (i64)slot * p.H + h0;
  // the codes of all heads, the window's B rows, and x rows
  uint4 q[HPC][R];
  float sc[HPC][R];
  const int p0 = tid / LPR, part = tid % LPR;
#pragma unroll
  for (int i = 0; i < HPC; ++i)
    if (i < nh) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        q[i][r] = __ldcs(reinterpret_cast<const uint4*>(p.c.codes) + ((sh0 + i) * 64 + p0 + r * RPP) * LPR + part);
        sc[i][r] = p.c.scales[(sh0 + i) * 64 + p0 + r * RPP];
      }
    }
  const int j = tid >> 4, piece = tid & 15;   // row j of the window, N / 16 bytes of it
  int8_t* const Bw = p.c.Bwin + ((i64)slot * p.G + g) * kWin * N;
  uint32_t Bv[N / 64];
  const bool waits = (j - f % kWin + kWin) % kWin < pos - f;   // (the token's own row does not)
#pragma unroll
  for (int k = 0; k < N / 64; ++k) Bv[k] = waits ? reinterpret_cast<const uint32_t*>(Bw + j * N)[piece * (N / 64) + k] : 0u;
  for (int k = tid; k < nh * kWin * 4; k += TS_T) {
    const int row = (k >> 2) % kWin;
    if (row != now)
      *reinterpret_cast<uint4*>(&s.x[0][0][0] + k * 16) = reinterpret_cast<const uint4*>(p.c.xwin + sh0 * kWin * 64)[k];
  }
  // codes of x of the heads, then of B and C
  const int HP = p.H * 64, GN = p.G * N, Ch = HP + 2 * GN;
  const T* const x = p.xBC + b * p.sb;
  T* const ring = p.ring + (i64)slot * p.width * Ch;
  for (int k = tid; k < 64 * nh + 2 * N; k += TS_T) {
    if (k < 64 * nh) {
      const int ch = h0 * 64 + k;
      const int c = channel(p, x, ring, Ch, ch, pos, p.s_x[ch], true);
      s.x[k >> 6][now][k & 63] = (int8_t)c;
      p.c.xwin[((sh0 + (k >> 6)) * kWin + now) * 64 + (k & 63)] = (int8_t)c;
    } else {
      const int n = k - 64 * nh;
      const bool isC = n >= N;
      const int c = channel(p, x, ring, Ch, HP + (isC ? GN : 0) + g * N + n % N, pos, (isC ? p.s_C : p.s_B)[g], hb == 0);
      (isC ? s.C : s.B)[n % N] = (int8_t)c;
      if (!isC && hb == 0) Bw[now * N + n] = (int8_t)c;
    }
  }
  // time steps and decays: a warp per head, half of it idle
  for (int i = warp; i < nh; i += TS_T / 32) {
    const int row = lane & 15, order = (row - f % kWin + kWin) % kWin, h = h0 + i;
    float dt = 0.f;
    if (row == now) {
      dt = Elem<T>::get(p.dt_raw[b * p.dt_sb + h]);
      if (p.softplus) dt = softplus_dt(dt, p.dt_bias ? p.dt_bias[h] : 0.f);
      if (lane < 16) p.c.dtwin[(sh0 + i) * kWin + now] = dt;
    } else if (order < pos - f) {
      dt = p.c.dtwin[(sh0 + i) * kWin + row];
    }
    const Waiting w = waiting_of(dt, order);
    const double A = (double)p.A[h];
    if (lane < 16) {
      s.w[i][row] = dt * expf((float)(A * w.behind));
      if (lane == 0) s.E[i] = expf((float)(A * w.all));
      if (now == kWin - 1) {
        s.wd[i][row] = (double)dt * exp(A * w.behind);
        if (lane == 0) s.Ed[i] = exp(A * w.all);
      }
    }
  }
  __syncthreads();
  // C . B_j
  {
    int d = 0;
#pragma unroll
    for (int k = 0; k < N / 64; ++k) {
      const int at = piece * (N / 64) + k;
      if (j == now) Bv[k] = reinterpret_cast<const uint32_t*>(s.B)[at];
      d = __dp4a((int)Bv[k], reinterpret_cast<const int*>(s.C)[at], d);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
    if (piece == 0) s.CB[j] = d;
  }
  const uint4 C16 = reinterpret_cast<const uint4*>(s.C)[part];
  const float sB = p.s_B[g], sC = p.s_C[g];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < HPC; ++i)
    if (i < nh) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int pp = p0 + r * RPP, ch = (h0 + i) * 64 + pp;
        // each lane of the row: its codes, and kWin / LPR of the window's tokens
        float win = 0.f;
#pragma unroll
        for (int k = 0; k < kWin / LPR; ++k) {
          const int jj = part * (kWin / LPR) + k;
          // (a row that holds no waiting token has w = 0, and int8 codes are finite)
          win = fmaf(s.w[i][jj] * (float)s.CB[jj], (float)s.x[i][jj][pp], win);
        }
        const float sx = p.s_x[ch];
        float v = s.E[i] * sc[i][r] * (float)dot16(q[i][r], C16) + sx * sB * win;
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (part == 0) {
          v *= sC;
          if (p.D) v += p.D[h0 + i] * sx * (float)s.x[i][now][pp];
          if (p.corr) v += p.corr[ch];
          const i64 at = (i64)b * HP + ch;
          if (p.ydt == 0) static_cast<float*>(p.y)[at] = v;
          else if (p.ydt == 1) static_cast<__half*>(p.y)[at] = __float2half_rn(v);
          else static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(v);
        }
      }
    }
  if (now != kWin - 1) return;
  // the window is full: S = E scale q + sum_j (w_j s_x s_B x_j) B_j, the row's new step size and codes, in binary64
#pragma unroll 1
  for (int i = 0; i < nh; ++i) {
    __syncthreads();   // (the operands of the head before have been read)
    for (int k = tid; k < kWin * 64; k += TS_T) {
      const int row = k >> 6, pp = k & 63;
      s.xw[row][pp] = s.wd[i][row] * (double)p.s_x[(h0 + i) * 64 + pp] * (double)sB * (double)s.x[i][row][pp];
    }
    if (i == 0)
#pragma unroll
      for (int k = 0; k < N / 64; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) s.Bd[j][(piece * (N / 64) + k) * 4 + e] = (double)sx8(Bv[k], e);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int pp = p0 + r * RPP;
      const i64 row = (sh0 + i) * 64 + pp;
      uint4 qv = q[0][r];
      float scale = sc[0][r];
#pragma unroll
      for (int k = 1; k < HPC; ++k)
        if (k == i) { qv = q[k][r]; scale = sc[k][r]; }
      const double e = s.Ed[i] * (double)scale;
      double S[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) S[k] = e * (double)sx8(k < 4 ? qv.x : k < 8 ? qv.y : k < 12 ? qv.z : qv.w, k & 3);
#pragma unroll 1
      for (int t = 0; t < kWin; ++t) {
        const double xv = s.xw[t][pp];
        const double2* Bt = reinterpret_cast<const double2*>(&s.Bd[t][part * 16]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const double2 B2 = Bt[k];
          S[2 * k] = __fma_rn(xv, B2.x, S[2 * k]);
          S[2 * k + 1] = __fma_rn(xv, B2.y, S[2 * k + 1]);
        }
      }
      double m = 0.0;
#pragma unroll
      for (int k = 0; k < 16; ++k) m = fmax(m, fabs(S[k]));
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
      float step = (float)__ddiv_rn(m, 127.0);
      if (step == 0.f) step = 1.f;
      uint32_t out[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        int c[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) c[u] = __double2int_rn(fmax(fmin(__ddiv_rn(S[4 * k + u], (double)step), 127.0), -127.0));
        out[k] = pack4(c[0], c[1], c[2], c[3]);
      }
      reinterpret_cast<uint4*>(p.c.codes)[row * LPR + part] = make_uint4(out[0], out[1], out[2], out[3]);
      if (part == 0) p.c.scales[row] = step;
    }
  }
}

template <typename T>
ssdi8_status_t launch(const Dims& d, const ssdi8_cache_t& c, const ssdi8_token_args_t& a, bool softplus, int ydt, cudaStream_t st) {
  TokenParams<T> p = {};
  p.c = view_of(c);
  p.ring = static_cast<T*>(c.ring); p.width = c.width;
  p.xBC = static_cast<const T*>(a.xBC); p.sb = a.stride_b; p.weight = a.weight; p.bias = a.bias;
  p.dt_raw = static_cast<const T*>(a.dt_raw); p.dt_sb = a.dt_stride_b; p.dt_bias = a.dt_bias;
  p.A = a.A; p.D = a.D; p.corr = a.corr; p.s_x = a.s_x; p.s_B = a.s_B; p.s_C = a.s_C;
  p.slots = a.slots; p.pos = a.pos; p.y = a.y; p.status = a.status;
  p.H = d.H; p.G = d.G; p.softplus = softplus; p.ydt = ydt;
  constexpr int HPC = 2;
  p.hblocks = (d.H / d.G + HPC - 1) / HPC;
  const i64 blocks = (i64)d.b * d.G * p.hblocks;
  if (blocks > 0x7fffffff) return SSDI8_ERR_SHAPE;
  auto go = [&](auto kernel) { return launch_configured(kernel, dim3((unsigned)blocks), dim3(TS_T), 0, -1, false, st, p); };
  return d.N == 128 ? go(token_kernel<T, 128, HPC>) : go(token_kernel<T, 64, HPC>);
}

}  // namespace

ssdi8_status_t launch_token_step(const Dims& d, const ssdi8_cache_t& c, const ssdi8_token_args_t& a, bool softplus, int ydt, cudaStream_t st) {
  return c.dtype == 0 ? launch<float>(d, c, a, softplus, ydt, st)
       : c.dtype == 1 ? launch<__half>(d, c, a, softplus, ydt, st)
                      : launch<__nv_bfloat16>(d, c, a, softplus, ydt, st);
}

}  // namespace ssdi8
