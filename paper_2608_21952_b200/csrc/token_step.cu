// One token for every sequence over the 8-bit state cache: convolution, codes of x, B and C, time step, y, and the token put into
// the slot's window.  The state is read once, as codes, and not written: with the tokens since its last fold beside it,
//   y = s_C (E scale sum_n C q + s_x s_B sum_j w_j (C . B_j) x_j) + D s_x x + corr,   E = exp(A sum dt), w_j = dt_j exp(A sum behind j)
// (ChunkScan1 and ChunkScan2 of Algorithm 2 for a single row, with int8 dot products), a quarter of the fp32 state's bytes one way
// instead of two.  Once in 16 tokens the full window is folded into the codes, in binary64.
#include "kernels.h"
#include "sm100.cuh"
#include "state_cache.cuh"

namespace ssdi8 {
namespace {

#ifndef TOKEN_HPC
#define TOKEN_HPC 4
#endif
constexpr int TS_T = 256;            // threads that convolve and have rows of y
constexpr int TS_ALL = TS_T + 32;    // and a warp for the time steps

__device__ __forceinline__ void named_bar(uint32_t id, uint32_t nthreads) { sm100::named_bar_sync(id, nthreads); }

// a wait has given up: the copies in flight get a bounded time to land before the block ends
__device__ __noinline__ void drain() {
  for (int i = 0; i < 50; ++i) __nanosleep(1000);
}

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

// codes of channels ch and ch + 1 (ch even) of the token, as two bytes: taps from the ring and the token itself, which goes into the ring
template <typename T>
__device__ __forceinline__ uint32_t channel_pair(const TokenParams<T>& p, const T* x, T* ring, int Ch, int ch, int pos, float2 step, bool keep) {
  struct alignas(2 * sizeof(T)) T2 { T a, b; };
  const int W = p.width;
  float2 xs[4], w[4];
  T2 own;
  own.a = x[ch];
  own.b = x[ch + 1];
#pragma unroll
  for (int k = 0; k < 3; ++k) {   // taps 4 - W .. 3 are the convolution's
    const int t = pos - 3 + k;
    xs[k] = w[k] = make_float2(0.f, 0.f);
    if (k >= 4 - W && t >= 0) {
      const T2 v = *reinterpret_cast<const T2*>(ring + (i64)((uint32_t)t % (uint32_t)W) * Ch + ch);
      xs[k] = make_float2(Elem<T>::get(v.a), Elem<T>::get(v.b));
    }
  }
  xs[3] = make_float2(Elem<T>::get(own.a), Elem<T>::get(own.b));
  if (W == 4) {
    const float4 u = *reinterpret_cast<const float4*>(p.weight + (i64)ch * 4), v = *reinterpret_cast<const float4*>(p.weight + (i64)ch * 4 + 4);
    w[0] = make_float2(u.x, v.x); w[1] = make_float2(u.y, v.y); w[2] = make_float2(u.z, v.z); w[3] = make_float2(u.w, v.w);
  } else {
#pragma unroll
    for (int k = 1; k < 4; ++k)
      if (k >= 4 - W) w[k] = make_float2(p.weight[(i64)ch * W + k - 4 + W], p.weight[(i64)(ch + 1) * W + k - 4 + W]);
  }
  const float2 bias = p.bias ? make_float2(p.bias[ch], p.bias[ch + 1]) : make_float2(0.f, 0.f);
  if (keep) *reinterpret_cast<T2*>(ring + (i64)((uint32_t)pos % (uint32_t)W) * Ch + ch) = own;
  float2 v = bias, m = make_float2(fabsf(bias.x), fabsf(bias.y));
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v = __ffma2_rn(w[k], xs[k], v);
    m = make_float2(fmaf(fabsf(w[k].x), fabsf(xs[k].x), m.x), fmaf(fabsf(w[k].y), fabsf(xs[k].y), m.y));
  }
  auto one = [&](float v, float m, float step, float* r) -> bool {   // true: near the middle of two integers (see block.cuh; M is the token's own here)
    const float inv = __frcp_rn(step);
    const float q = v * rcp_approx(1.0f + ex2_approx(v * -1.44269504f)) * inv;
    float cl;
    asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(cl) : "f"(q), "f"(127.0f));
    *r = __fadd_rn(cl, kMagicOut);
    const float off = fabsf(cl - __fadd_rn(*r, -kMagicOut));
    return !(fmaf(fmaf(2.0f * kEps, fabsf(v), 12.0f * kEps), fabsf(cl), fmaf(5.0f * kEps * m, inv, off)) <= 0.5f) || !(step >= 1e-30f && step <= 1e30f);
  };
  float r0, r1;
  if (one(v.x, m.x, step.x, &r0))
    r0 = __uint_as_float(rne_clamp_bits(silu_quotient_exact<4>(xs[0].x, xs[1].x, xs[2].x, xs[3].x, w[0].x, w[1].x, w[2].x, w[3].x, bias.x, step.x)));
  if (one(v.y, m.y, step.y, &r1))
    r1 = __uint_as_float(rne_clamp_bits(silu_quotient_exact<4>(xs[0].y, xs[1].y, xs[2].y, xs[3].y, w[0].y, w[1].y, w[2].y, w[3].y, bias.y, step.y)));
  return __byte_perm(__float_as_uint(r0), __float_as_uint(r1), 0x0040u) & 0xffffu;
}

__device__ __forceinline__ int dot16(const uint4& a, const uint4& b, int s) {
  s = __dp4a((int)a.x, (int)b.x, s);
  s = __dp4a((int)a.y, (int)b.y, s);
  s = __dp4a((int)a.z, (int)b.z, s);
  return __dp4a((int)a.w, (int)b.w, s);
}

template <int N, int HPC>
struct TokenSmem {
  __align__(128) int8_t codes[HPC][64][N];
  __align__(128) int8_t x[HPC][kWin][64];    // x of the window, rows as in the cache; the token's own row is stale
  __align__(16) int8_t xnow[HPC][64];        // x of the token
  __align__(16) int8_t C[N];
  __align__(16) int8_t B[N];
  __align__(16) int CB[kWin];                // C . B_j
  __align__(16) float w[HPC][kWin];          // w_j
  float E[HPC];
  uint64_t bar[HPC];
};

// A block has up to HPC heads of one group: the convolution of B and C is theirs together.  The codes and windows of its heads are
// requested as bulk copies into shared memory as soon as the slot is known; a thread then has a whole row of one head, its dot
// product as 4 N / 16 dp4a in turned order (no two lanes on one bank) and nothing to exchange.  Eight warps convolve, one more forms the time
// steps and decays beside them.
template <typename T, int N, int HPC>
__global__ void __launch_bounds__(TS_ALL, 4) token_kernel(const __grid_constant__ TokenParams<T> p) {
  extern __shared__ uint8_t smem_raw[];
  TokenSmem<N, HPC>& s = *reinterpret_cast<TokenSmem<N, HPC>*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~(uintptr_t)127);
  const int tid = threadIdx.x, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < HPC; ++i) sm100::mbar_init(&s.bar[i], 1);
    sm100::fence_mbar_init();
  }
  pdl_wait();
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
  const int now = pos % kWin, first = f % kWin, n = pos - f;   // rows of the token and of the first waiting one, and how many wait
  const i64 sh0 = (i64)slot * p.H + h0;
  if (tid == 0)
    for (int i = 0; i < nh; ++i) {
      sm100::mbar_expect_tx(&s.bar[i], 64 * N + kWin * 64);
      sm100::bulk_load(&s.codes[i][0][0], p.c.codes + (sh0 + i) * 64 * N, 64 * N, &s.bar[i]);
      sm100::bulk_load(&s.x[i][0][0], p.c.xwin + (sh0 + i) * kWin * 64, kWin * 64, &s.bar[i]);
    }
  const int HP = p.H * 64, GN = p.G * N, Ch = HP + 2 * GN;
  const int j = tid >> 4, piece = tid & 15;   // row j of the window, N / 16 bytes of it
  const int head = tid >> 6, row = tid & 63;  // of y
  uint32_t Bv[N / 64];
  float scale[(HPC + 3) / 4], sx[(HPC + 3) / 4];
  if (tid < TS_T) {
    int8_t* const Bw = p.c.Bwin + ((i64)slot * p.G + g) * kWin * N;
    const bool waits = (j - first + kWin) % kWin < n;   // (the token's own row does not)
#pragma unroll
    for (int k = 0; k < N / 64; ++k) Bv[k] = waits ? reinterpret_cast<const uint32_t*>(Bw + j * N)[piece * (N / 64) + k] : 0u;
#pragma unroll
    for (int q = 0; q < (HPC + 3) / 4; ++q) {
      const bool in = 4 * q + head < nh;
      scale[q] = in ? p.c.scales[(sh0 + 4 * q + head) * 64 + row] : 0.f;
      sx[q] = in ? p.s_x[(h0 + 4 * q + head) * 64 + row] : 0.f;
    }
    // codes of x of the heads, then of B and C
    const T* const x = p.xBC + b * p.sb;
    T* const ring = p.ring + (i64)slot * p.width * Ch;
    for (int k = 2 * tid; k < 64 * nh + 2 * N; k += 2 * TS_T) {
      if (k < 64 * nh) {
        const int ch = h0 * 64 + k;
        const uint32_t c = channel_pair(p, x, ring, Ch, ch, pos, *reinterpret_cast<const float2*>(p.s_x + ch), true);
        *reinterpret_cast<uint16_t*>(&s.xnow[0][0] + k) = (uint16_t)c;
        *reinterpret_cast<uint16_t*>(p.c.xwin + ((sh0 + (k >> 6)) * kWin + now) * 64 + (k & 63)) = (uint16_t)c;
      } else {
        const int at = (k - 64 * nh) % N;
        const bool isC = k - 64 * nh >= N;
        const float st = (isC ? p.s_C : p.s_B)[g];
        const uint32_t c = channel_pair(p, x, ring, Ch, HP + (isC ? GN : 0) + g * N + at, pos, make_float2(st, st), hb == 0);
        *reinterpret_cast<uint16_t*>((isC ? s.C : s.B) + at) = (uint16_t)c;
        if (!isC && hb == 0) *reinterpret_cast<uint16_t*>(Bw + now * N + at) = (uint16_t)c;
      }
    }
  } else {
    // time steps and decays, two heads at a time, lane j of a half-warp for row j of the window; the new time steps of all first
    float dtn = 0.f;
    if (lane < nh) {
      dtn = Elem<T>::get(p.dt_raw[b * p.dt_sb + h0 + lane]);
      if (p.softplus) dtn = softplus_dt(dtn, p.dt_bias ? p.dt_bias[h0 + lane] : 0.f);
      p.c.dtwin[(sh0 + lane) * kWin + now] = dtn;
    }
    const int rw = lane & 15, order = (rw - first + kWin) % kWin;
#pragma unroll
    for (int i0 = 0; i0 < HPC; i0 += 2) {
      const int i = i0 + (lane >> 4);
      float dt = __shfl_sync(0xffffffffu, dtn, i & 31);
      if (rw != now) dt = i < nh && order < n ? p.c.dtwin[(sh0 + i) * kWin + rw] : 0.f;
      const Waiting w = waiting_of(dt, order);
      if (i < nh) {
        const double A = (double)p.A[h0 + i];
        s.w[i][rw] = dt * expf((float)(A * w.behind));
        if (rw == 0) s.E[i] = expf((float)(A * w.all));
      }
    }
  }
  __syncthreads();
  if (tid >= TS_T) return;
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
  const float sB = p.s_B[g], sC = p.s_C[g];
  named_bar(1, TS_T);
#pragma unroll
  for (int q = 0; q < (HPC + 3) / 4; ++q) {
    const int i = 4 * q + head;
    if (i < nh) {
      // the waiting tokens and the token itself
      const float xn = (float)s.xnow[i][row];
      float win = s.w[i][now] * (float)s.CB[now] * xn;
      if (!sm100::mbar_wait_inline<0>(&s.bar[i], 0, p.status)) drain();
#pragma unroll 4
      for (int o = 0; o < n; ++o) {
        const int jj = (first + o) % kWin;
        win = fmaf(s.w[i][jj] * (float)s.CB[jj], (float)s.x[i][jj][row], win);
      }
      int d = 0;
      const uint4* const cr = reinterpret_cast<const uint4*>(&s.codes[i][row][0]);
#pragma unroll
      for (int k = 0; k < N / 16; ++k) {
        const int c = N == 128 ? (k + row) & 7 : (k + (row >> 1)) & 3;
        d = dot16(cr[c], reinterpret_cast<const uint4*>(s.C)[c], d);
      }
      const int ch = (h0 + i) * 64 + row;
      float v = sC * fmaf(s.E[i] * scale[q], (float)d, sx[q] * sB * win);
      if (p.D) v = fmaf(p.D[h0 + i] * sx[q], xn, v);
      if (p.corr) v += p.corr[ch];
      const i64 at = (i64)b * HP + ch;
      if (p.ydt == 0) static_cast<float*>(p.y)[at] = v;
      else if (p.ydt == 1) static_cast<__half*>(p.y)[at] = __float2half_rn(v);
      else static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(v);
    }
  }
}

// ------------------------------------------------------------------------------------------------ fold
constexpr int kSeqs = 128;       // sequences looked over at a time

template <int N>
struct FoldSmem {
  static constexpr int kWarps = N / 16, kRows = 64 / kWarps;   // eight rows per lane: 8 (N = 128) or 16 rows of a warp
  __align__(16) int8_t codes[64][N];
  __align__(16) int8_t x[kWin][64];
  __align__(16) float Bf[kWin][N];
  __align__(16) float xw[kWarps][kWin][kRows];   // x with its factors
  float scale[64], sx[64], step[64], size[64];   // size: how far off an element of the row can be
  int cand[64];                                  // an element that can be the row's absmax
  double w[kWin], E;
  int warps[kSeqs / 32], full[kSeqs];            // sequences with a full window
};

// The full window of a head into its codes.  binary32 decides where it can: an element is off by at most 22 eps of its terms'
// magnitudes (E, the row's factor and the product 3, x's factors 4, up to 16 fused additions), so one whose quotient lies nearer than that
// to the middle of two integers is formed again in binary64, and so is the row's absmax (of the few elements that can be it): step
// sizes and codes are those of binary64, E scale q + sum_j (w_j s_x s_B x_j) B_j.
// A lane has four n of eight rows, N / 4 lanes per row; from the operands on a warp works on its rows alone.  (Lists of such elements
// for all threads of the block and a barrier between the steps: 25 thousand cycles a head, 37 us a step of 64 x 80 heads, eight of
// the sequences with full windows; 256 threads with two heads in turn 47 us; wholly in binary64 with its divisions 80 us a head.)
template <int N>
__device__ __forceinline__ void fold(FoldSmem<N>& s, float sB, int8_t* codes, float* scales) {
  constexpr int LPR = N / 4, ROWS = FoldSmem<N>::kRows, LR = LPR / 8, PER = kWin / LR;   // lanes per row; lanes and terms of each where a row is a few lanes' work
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / LPR, n0 = (lane % LPR) * 4, base = warp * ROWS, row0 = base + 8 * sub;
  const int mine = (lane % LPR) / LR, my_row = row0 + mine, t0 = lane % LR * PER;   // the row that this lane shares with LR - 1 others
  const double f = (double)s.sx[my_row] * (double)sB;
  {
    float m = 0.f;
    const float f32 = s.sx[my_row] * sB;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const float x = (float)s.w[t0 + j] * f32 * (float)s.x[t0 + j][my_row];
      s.xw[warp][t0 + j][my_row - base] = x;
      m += fabsf(x);
    }
#pragma unroll
    for (int o = 1; o < LR; o <<= 1) m += __shfl_xor_sync(0xffffffffu, m, o);
    if (t0 == 0) s.size[my_row] = (fabsf((float)s.E * s.scale[my_row]) + m) * (24.0f * 127.0f * kEps);
  }
  __syncwarp();
  float2 v[8][2];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const float e = (float)s.E * s.scale[row0 + r];
    const uint32_t q = *reinterpret_cast<const uint32_t*>(&s.codes[row0 + r][n0]) ^ 0x80808080u;
    v[r][0] = make_float2(e * s8_to_f32(q, 0), e * s8_to_f32(q, 1));
    v[r][1] = make_float2(e * s8_to_f32(q, 2), e * s8_to_f32(q, 3));
  }
#pragma unroll 4
  for (int j = 0; j < kWin; ++j) {
    const float4 B = *reinterpret_cast<const float4*>(&s.Bf[j][n0]);
    const float4 xa = *reinterpret_cast<const float4*>(&s.xw[warp][j][8 * sub]), xb = *reinterpret_cast<const float4*>(&s.xw[warp][j][8 * sub + 4]);
    const float xr[8] = {xa.x, xa.y, xa.z, xa.w, xb.x, xb.y, xb.z, xb.w};
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      v[r][0] = __ffma2_rn(make_float2(xr[r], xr[r]), make_float2(B.x, B.y), v[r][0]);
      v[r][1] = __ffma2_rn(make_float2(xr[r], xr[r]), make_float2(B.z, B.w), v[r][1]);
    }
  }
  // absmax of eight rows at once: each exchange halves the rows that a lane still has
  float m[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) m[r] = fmaxf(fmaxf(fabsf(v[r][0].x), fabsf(v[r][0].y)), fmaxf(fabsf(v[r][1].x), fabsf(v[r][1].y)));
#pragma unroll
  for (int k = 4, o = LPR / 2; k >= 1; k >>= 1, o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int r = 0; r < k; ++r) {
      const float keep = up ? m[r + k] : m[r], give = up ? m[r] : m[r + k];
      m[r] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, o));
    }
  }
#pragma unroll
  for (int o = 1; o < LR; o <<= 1) m[0] = fmaxf(m[0], __shfl_xor_sync(0xffffffffu, m[0], o));
  const float least_of_mine = m[0] - 2.0f * s.size[my_row];
  // the elements that can be it: one of each row into its place, more of them (few) stay flagged
  uint32_t flags = 0;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const float least = __shfl_sync(0xffffffffu, least_of_mine, lane / LPR * LPR + r * LR);
    uint32_t fl = 0;
    const bool any = !(fmaxf(fmaxf(fabsf(v[r][0].x), fabsf(v[r][0].y)), fmaxf(fabsf(v[r][1].x), fabsf(v[r][1].y))) < least);
    const uint32_t who = __ballot_sync(0xffffffffu, any) >> (lane / LPR * LPR) & (LPR == 32 ? 0xffffffffu : 0xffffu);
    if (any) {
      const float q[4] = {v[r][0].x, v[r][0].y, v[r][1].x, v[r][1].y};
#pragma unroll
      for (int c = 0; c < 4; ++c) fl |= fabsf(q[c]) < least ? 0u : 1u << c;
      if (__ffs(who) - 1 == lane % LPR) {
        s.cand[row0 + r] = n0 + __ffs(fl) - 1;
        fl &= fl - 1;
      }
    }
    flags |= fl << (4 * r);
  }
  __syncwarp();
  auto term = [&](int row, int col, double fr, int j) { return s.w[j] * fr * (double)s.x[j][row] * (double)s.Bf[j][col]; };
  double top;
  {
    const int col = s.cand[my_row];
    double S = t0 == 0 ? s.E * (double)s.scale[my_row] * (double)s.codes[my_row][col] : 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) S += term(my_row, col, f, t0 + j);
#pragma unroll
    for (int o = 1; o < LR; o <<= 1) S += __shfl_xor_sync(0xffffffffu, S, o);
    top = fmax(fabs(S), 0.0);   // (a NaN counts for nothing)
  }
  // one flagged element after the other by the warp, a term per lane: S, its row and column, the lane and the bit that it was flagged by
  auto next = [&](uint32_t& fl, int* from, int* bit, int* row) {
    *from = __ffs(__ballot_sync(0xffffffffu, fl != 0)) - 1;
    *bit = __ffs(__shfl_sync(0xffffffffu, fl, *from)) - 1;
    if (lane == *from) fl &= fl - 1;
    *row = base + 8 * (*from / LPR) + (*bit >> 2);
    const int col = (*from % LPR) * 4 + (*bit & 3), j = lane & 15;
    double S = term(*row, col, (double)s.sx[*row] * (double)sB, j);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) S += __shfl_xor_sync(0xffffffffu, S, o);
    return S + s.E * (double)s.scale[*row] * (double)s.codes[*row][col];
  };
  while (__any_sync(0xffffffffu, flags != 0)) {
    int from, bit, row = 0;
    const double S = fabs(next(flags, &from, &bit, &row));
    if (row == my_row) top = fmax(top, S);
  }
  {
    float step = (float)__ddiv_rn(top, 127.0);
    if (step == 0.f) step = 1.f;
    if (t0 == 0) {
      s.step[my_row] = step;
      scales[my_row] = step;
    }
  }
  __syncwarp();
  uint32_t code[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const float q[4] = {v[r][0].x, v[r][0].y, v[r][1].x, v[r][1].y};
    const float step = s.step[row0 + r], inv = __frcp_rn(step), least = 0.5f - s.size[row0 + r] * inv;
    float t[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float cl;
      asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(cl) : "f"(q[c] * inv), "f"(127.0f));
      t[c] = __fadd_rn(cl, kMagicOut);
      flags |= fmaf(4.0f * kEps, fabsf(cl), fabsf(cl - __fadd_rn(t[c], -kMagicOut))) <= least ? 0u : 1u << (4 * r + c);
    }
    if (!(step >= 1e-30f && step <= 1e30f)) flags |= 15u << (4 * r);
    code[r] = pack4_bits(__float_as_uint(t[0]), __float_as_uint(t[1]), __float_as_uint(t[2]), __float_as_uint(t[3]));
  }
  while (__any_sync(0xffffffffu, flags != 0)) {
    int from, bit, row = 0;
    const double q = next(flags, &from, &bit, &row) / (double)s.step[row];
    const uint32_t c = (uint32_t)__double2int_rn(fmax(fmin(q, 127.0), -127.0)) & 0xffu;   // (fmin(NaN, 127) = 127)
    const int at = 8 * (bit & 3);
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (lane == from && r == bit >> 2) code[r] = (code[r] & ~(0xffu << at)) | c << at;
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) *reinterpret_cast<uint32_t*>(codes + (row0 + r) * N + n0) = code[r];
}

struct FoldParams {
  CacheView c;
  const float *A, *s_x, *s_B;
  const int32_t *slots, *pos;
  int B, H, G;
};

// Behind the token kernel: the blocks share out the heads of the sequences whose windows have become full.  (Folded in the token kernel
// itself, the blocks of such a sequence met on a few SMs while the others had none: 83 us a step of 64 x 80 heads.)
template <int N>
__global__ void __launch_bounds__(2 * N, 768 / (2 * N)) token_fold_kernel(const __grid_constant__ FoldParams p) {
  extern __shared__ uint8_t smem_raw[];
  FoldSmem<N>& s = *reinterpret_cast<FoldSmem<N>*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~(uintptr_t)127);
  constexpr int THREADS = 2 * N;
  const int tid = threadIdx.x, lane = tid & 31;
  pdl_launch_dependents();
  pdl_wait();
  for (int b0 = 0; b0 < p.B; b0 += kSeqs) {
    // the full ones of these sequences in their order, the same in every block
    const int bt = b0 + tid, pt = tid < kSeqs && bt < p.B ? p.pos[bt] : -1;
    const bool full = pt >= 0 && pt % kWin == kWin - 1;
    const uint32_t mask = __ballot_sync(0xffffffffu, full);
    if (tid < kSeqs && lane == 0) s.warps[tid >> 5] = __popc(mask);
    __syncthreads();
    int before = 0, found = 0;
#pragma unroll
    for (int k = 0; k < kSeqs / 32; ++k) {
      if (k < tid >> 5) before += s.warps[k];
      found += s.warps[k];
    }
    if (full) s.full[before + __popc(mask & ((1u << lane) - 1u))] = bt;
    __syncthreads();
    for (int at = blockIdx.x; at < found * p.H; at += gridDim.x) {
      const int b = s.full[at / p.H], h = at % p.H, g = h / (p.H / p.G);
      bool bad;
      const int slot = slot_of(p.slots, p.pos, p.c.nslots, b, &bad);   // (its barrier: the block is done with the head before)
      const int pos = p.pos[b], start = slot >= 0 ? p.c.start[slot] : 0;
      if (slot < 0 || start > pos) continue;
      const i64 sh = (i64)slot * p.H + h;
      uint4 q[2];   // (32 codes of each thread)
#pragma unroll
      for (int k = 0; k < 2; ++k) q[k] = reinterpret_cast<const uint4*>(p.c.codes + sh * 64 * N)[tid + k * THREADS];
      uint32_t Bw[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) Bw[k] = reinterpret_cast<const uint32_t*>(p.c.Bwin + ((i64)slot * p.G + g) * kWin * N)[tid + k * THREADS];
      if (tid >= THREADS - 64) {
        const int k = tid - (THREADS - 64);
        reinterpret_cast<uint4*>(&s.x[0][0])[k] = reinterpret_cast<const uint4*>(p.c.xwin + sh * kWin * 64)[k];
        s.scale[k] = p.c.scales[sh * 64 + k];
        s.sx[k] = p.s_x[h * 64 + k];
        s.cand[k] = 0;   // (of a row of NaN there is none)
      }
      if (tid < 32) {   // lane j of a half-warp has row j of the window
        const int j = lane & 15;
        const float dt = j >= max(start, pos - (kWin - 1)) % kWin ? p.c.dtwin[sh * kWin + j] : 0.f;
        const Waiting w = waiting_of(dt, j);
        const double e = exp((double)p.A[h] * (lane < 16 ? w.behind : w.all));
        if (lane < 16) s.w[j] = (double)dt * e;
        if (lane == 16) s.E = e;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        reinterpret_cast<uint4*>(&s.codes[0][0])[tid + k * THREADS] = q[k];
        *reinterpret_cast<float4*>(&s.Bf[0][0] + 4 * (tid + k * THREADS)) =
            make_float4((float)sx8(Bw[k], 0), (float)sx8(Bw[k], 1), (float)sx8(Bw[k], 2), (float)sx8(Bw[k], 3));
      }
      __syncthreads();
      fold<N>(s, p.s_B[g], p.c.codes + sh * 64 * N, p.c.scales + sh * 64);
    }
    __syncthreads();
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
  auto go = [&](auto kernel, size_t smem) -> ssdi8_status_t {
    const i64 blocks = (i64)d.b * d.G * p.hblocks;
    if (blocks > 0x7fffffff) return SSDI8_ERR_SHAPE;
    return launch_configured(kernel, dim3((unsigned)blocks), dim3(TS_ALL), smem, -1, false, st, p);
  };
  auto pick = [&](auto hpc) -> ssdi8_status_t {
    constexpr int HPC = decltype(hpc)::value;
    p.hblocks = (d.H / d.G + HPC - 1) / HPC;
    return d.N == 128 ? go(token_kernel<T, 128, HPC>, sizeof(TokenSmem<128, HPC>) + 128) : go(token_kernel<T, 64, HPC>, sizeof(TokenSmem<64, HPC>) + 128);
  };
  const ssdi8_status_t s = pick(std::integral_constant<int, TOKEN_HPC>{});
  if (s != SSDI8_OK) return s;
  const int sms = sm_count();
  if (sms <= 0) return SSDI8_ERR_CUDA;
  const FoldParams f = {p.c, a.A, a.s_x, a.s_B, a.slots, a.pos, d.b, d.H, d.G};
  auto go_fold = [&](auto kernel, int N, size_t smem) {
    const i64 heads = (i64)d.b * d.H, most = (i64)sms * (768 / (2 * N));
    return launch_configured(kernel, dim3((unsigned)(heads < most ? heads : most)), dim3(2 * N), smem, -1, false, st, f);
  };
  return d.N == 128 ? go_fold(token_fold_kernel<128>, 128, sizeof(FoldSmem<128>) + 128) : go_fold(token_fold_kernel<64>, 64, sizeof(FoldSmem<64>) + 128);
}

}  // namespace

ssdi8_status_t launch_token_step(const Dims& d, const ssdi8_cache_t& c, const ssdi8_token_args_t& a, bool softplus, int ydt, cudaStream_t st) {
  return c.dtype == 0 ? launch<float>(d, c, a, softplus, ydt, st)
       : c.dtype == 1 ? launch<__half>(d, c, a, softplus, ydt, st)
                      : launch<__nv_bfloat16>(d, c, a, softplus, ydt, st);
}

}  // namespace ssdi8
