// One token for every sequence over the 8-bit state cache: convolution, codes of x, B and C, time step, y, and the token put into
// the slot's window.  The state is read once, as codes, and not written: with the tokens since its last fold beside it,
//   y = s_C (E scale sum_n C q + s_x s_B sum_j w_j (C . B_j) x_j) + D s_x x + corr,   E = exp(A sum dt), w_j = dt_j exp(A sum behind j)
// (ChunkScan1 and ChunkScan2 of Algorithm 2 for a single row, with int8 dot products), a quarter of the fp32 state's bytes one way
// instead of two.  Once in 16 tokens the full window is folded into the codes, as in binary64, by a second kernel.
//
// What bounds it: 64 sequences x 80 heads (53 MB, 8.3 us at the copy rate) take 22 us without full windows (16 where the slots stay in L2 from call
// to call), 250 x 128 (335 MB, 52 us) 93: about 760 instructions a warp, half of them the convolution of B and C, which every block of heads does for
// itself, and the chain of a block (slot, ring, codes, weights of the window, y: 10 thousand cycles) with 27 warps to an SM.  The fp32
// state's step (ssd_step.cu) with its two kernels ahead takes 58.8 for the first.  With one sequence in 16 folding, 31 to 36 and 134 to 145 us
// (all of them: 129 and 757): a fold is about 1700 instructions a warp, and its kernel starts when the last block of the step has ended.
#include "kernels.h"
#include "sm100.cuh"
#include "state_cache.cuh"

namespace ssdi8 {
namespace {

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
  int H, G, hpg, softplus, ydt, b0;   // hpg: heads per group; b0: the launch's first sequence
};

// The code of a channel in binary64, out of line, by the operations of a prompt's (conv.cu).  Four taps: of fewer, the first ones are 0.
__device__ __noinline__ float code_exact(float x0, float x1, float x2, float x3, float w0, float w1, float w2, float w3, float bias, float step) {
  const float x[4] = {x0, x1, x2, x3}, w[4] = {w0, w1, w2, w3};
  double v = (double)bias;
#pragma unroll
  for (int k = 0; k < 4; ++k) v = __fma_rn((double)w[k], (double)x[k], v);
  const double q = v / ((1.0 + exp(-v)) * (double)step);
  // (rounded to an integer here: a second rounding to binary32 must not decide)
  return (float)rint(fmax(fmin(q, 127.0), -127.0));   // (fmin(NaN, 127) = 127)
}

// Two channels of the token, ch and ch + 1 (ch even): what does not depend on the slot, loaded while the slot is on its way
template <typename T>
struct alignas(2 * sizeof(T)) Pair { T a, b; };
template <typename T>
struct ChannelPair {
  float2 w[4], bias, step, xs[3];
  Pair<T> own;
  __device__ __forceinline__ void load(const TokenParams<T>& p, const T* x, int ch, const float* steps, bool each) {
    const int W = p.width;
    own.a = x[ch];
    own.b = x[ch + 1];
    if (W == 4) {
      const float4 u = *reinterpret_cast<const float4*>(p.weight + (i64)ch * 4), v = *reinterpret_cast<const float4*>(p.weight + (i64)ch * 4 + 4);
      w[0] = make_float2(u.x, v.x); w[1] = make_float2(u.y, v.y); w[2] = make_float2(u.z, v.z); w[3] = make_float2(u.w, v.w);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)   // taps 4 - W .. 3 are the convolution's
        w[k] = k >= 4 - W ? make_float2(p.weight[(i64)ch * W + k - 4 + W], p.weight[(i64)(ch + 1) * W + k - 4 + W]) : make_float2(0.f, 0.f);
    }
    bias = p.bias ? make_float2(p.bias[ch], p.bias[ch + 1]) : make_float2(0.f, 0.f);
    step = each ? *reinterpret_cast<const float2*>(steps) : make_float2(*steps, *steps);
  }
  // the tokens ahead, from the ring; those of negative positions are zeros
  __device__ __forceinline__ void past(const TokenParams<T>& p, const T* ring, int Ch, int pos) {
    const int W = p.width;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const int t = pos - 3 + k;
      xs[k] = make_float2(0.f, 0.f);
      if (k >= 4 - W && t >= 0) {
        const Pair<T> v = *reinterpret_cast<const Pair<T>*>(ring + (i64)(W == 4 ? t & 3 : t % W) * Ch);
        xs[k] = make_float2(Elem<T>::get(v.a), Elem<T>::get(v.b));
      }
    }
  }
  // their codes as two bytes
  __device__ __forceinline__ uint32_t codes() const {
    const float2 x3 = make_float2(Elem<T>::get(own.a), Elem<T>::get(own.b));
    float2 v = bias, m = make_float2(fabsf(bias.x), fabsf(bias.y));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 x = k < 3 ? xs[k] : x3;
      v = __ffma2_rn(w[k], x, v);
      m = make_float2(fmaf(fabsf(w[k].x), fabsf(x.x), m.x), fmaf(fabsf(w[k].y), fabsf(x.y), m.y));
    }
    // true: near the middle of two integers, by 5 eps M / step + (14 + 2 |v|) eps |q| (see block.cuh)
    auto one = [&](float v, float m, float step, float* r) -> bool {
      const float inv = rcp_approx(step);
      const float q = v * rcp_approx(1.0f + ex2_approx(v * -1.44269504f)) * inv;
      float cl;
      asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(cl) : "f"(q), "f"(127.0f));
      *r = __fadd_rn(cl, kMagicOut);
      const float off = fabsf(cl - __fadd_rn(*r, -kMagicOut));
      return !(fmaf(fmaf(2.0f * kEps, fabsf(v), 14.0f * kEps), fabsf(cl), fmaf(5.0f * kEps * m, inv, off)) <= 0.5f) || !(step >= 1e-30f && step <= 1e30f);
    };
    float r0, r1;
    if (one(v.x, m.x, step.x, &r0))
      r0 = __uint_as_float(rne_clamp_bits(code_exact(xs[0].x, xs[1].x, xs[2].x, x3.x, w[0].x, w[1].x, w[2].x, w[3].x, bias.x, step.x)));
    if (one(v.y, m.y, step.y, &r1))
      r1 = __uint_as_float(rne_clamp_bits(code_exact(xs[0].y, xs[1].y, xs[2].y, x3.y, w[0].y, w[1].y, w[2].y, w[3].y, bias.y, step.y)));
    return __byte_perm(__float_as_uint(r0), __float_as_uint(r1), 0x0040u) & 0xffffu;
  }
};

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
  __align__(16) float g[HPC][kWin];          // w_j C . B_j
  __align__(16) float w[HPC][kWin];          // w_j
  float E[HPC];
  uint64_t bar[HPC];
};

// A block has up to HPC heads of one group: the convolution of B and C is theirs together.  The codes and windows of its heads are
// requested as bulk copies into shared memory as soon as the slot is known.  Eight warps convolve, one more forms the time
// steps and decays beside them.
template <typename T, int N, int HPC>
__global__ void __launch_bounds__(TS_ALL, HPC == 8 ? 3 : 4) token_kernel(const __grid_constant__ TokenParams<T> p) {
  constexpr int QH = (HPC + 3) / 4;   // heads that a thread has a row of
  constexpr int LPR = N / 16;
  extern __shared__ uint8_t smem_raw[];
  TokenSmem<N, HPC>& s = *reinterpret_cast<TokenSmem<N, HPC>*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~(uintptr_t)127);
  const int tid = threadIdx.x, lane = tid & 31;
  if (tid < HPC) sm100::mbar_init(&s.bar[tid], 1);
  if (tid < 32) sm100::fence_mbar_init();
  pdl_wait();
  const int hb = blockIdx.x, g = blockIdx.y, b = blockIdx.z + p.b0;
  const int h0 = g * p.hpg + hb * HPC, nh = min(HPC, p.hpg - hb * HPC);
  const int HP = p.H * 64, GN = p.G * N, Ch = HP + 2 * GN;
  const T* const x = p.xBC + b * p.sb;
  // channels of this thread: x of the heads, then B and C
  const int nch = 64 * nh + 2 * N;
  auto channel_of = [&](int k) { return k < 64 * nh ? h0 * 64 + k : k < 64 * nh + N ? HP + g * N + k - 64 * nh : HP + GN + g * N + k - 64 * nh - N; };
  auto steps_of = [&](int k) { return k < 64 * nh ? p.s_x + h0 * 64 + k : (k < 64 * nh + N ? p.s_B : p.s_C) + g; };
  ChannelPair<T> cp;
  float dtn = 0.f;   // the warp of the time steps: those of the token
  if (tid < TS_T) {
    if (2 * tid < nch) cp.load(p, x, channel_of(2 * tid), steps_of(2 * tid), 2 * tid < 64 * nh);
  } else if (lane < nh) {
    dtn = Elem<T>::get(p.dt_raw[b * p.dt_sb + h0 + lane]);
    if (p.softplus) dtn = softplus_dt(dtn, p.dt_bias ? p.dt_bias[h0 + lane] : 0.f);
  }
  bool bad;
  const int slot = slot_of(p.slots, p.pos, p.c.nslots, b, &bad);
  const int pos = slot >= 0 ? p.pos[b] : 0;
  if (bad && hb == 0 && g == 0 && tid == 0) bad_row(p.status);
  if (slot < 0) return;
  const int start = p.c.start[slot], now = pos % kWin, f = max(start, pos - now);
  const i64 sh0 = (i64)slot * p.H + h0;
  const int j = (tid >> 4) % kWin, piece = tid & 15;   // row j of the window, N / 16 bytes of it
  // y: a warp has 32 rows of a head, LPR lanes with 16 codes each per row, and a lane in the end the row whose sum it keeps
  const int head = tid >> 6, half = tid & 32, row = half + lane % LPR * (32 / LPR) + lane / LPR;
  int8_t* const Bw = p.c.Bwin + ((i64)slot * p.G + g) * kWin * N;
  T* const ring = p.ring + (i64)slot * p.width * Ch;
  uint32_t Bv[N / 64];
  if (tid < TS_T) {
    if (2 * tid < nch) cp.past(p, ring + channel_of(2 * tid), Ch, pos);
#pragma unroll
    for (int k = 0; k < N / 64; ++k) Bv[k] = reinterpret_cast<const uint32_t*>(Bw + j * N)[piece * (N / 64) + k];
  }
  if (start > pos) {   // the slot was written behind this position
    if (hb == 0 && g == 0 && tid == 0) bad_row(p.status);
    return;
  }
  if (tid >= TS_T && lane < nh) {
    sm100::mbar_expect_tx(&s.bar[lane], 64 * N + kWin * 64);
    sm100::bulk_load(&s.codes[lane][0][0], p.c.codes + (sh0 + lane) * 64 * N, 64 * N, &s.bar[lane]);
    sm100::bulk_load(&s.x[lane][0][0], p.c.xwin + (sh0 + lane) * kWin * 64, kWin * 64, &s.bar[lane]);
  }
  const int first = f % kWin, n = pos - f;   // row of the first waiting token, and how many wait
  float scale[QH], sx[QH], corr[QH], D[QH];
  if (tid < TS_T) {
#pragma unroll
    for (int q = 0; q < QH; ++q) {
      const bool in = 4 * q + head < nh;
      const int ch = (h0 + 4 * q + head) * 64 + row;
      scale[q] = in ? p.c.scales[(sh0 + 4 * q + head) * 64 + row] : 0.f;
      sx[q] = in ? p.s_x[ch] : 0.f;
      corr[q] = in && p.corr ? p.corr[ch] : 0.f;
      D[q] = in && p.D ? p.D[h0 + 4 * q + head] : 0.f;
    }
    if (((j - first) & (kWin - 1)) >= n) {   // (nor does the token's own row wait)
#pragma unroll
      for (int k = 0; k < N / 64; ++k) Bv[k] = 0u;
    }
#pragma unroll
    for (int k0 = 0; k0 < 64 * HPC + 2 * N; k0 += 2 * TS_T) {
      const int k = k0 + 2 * tid;
      if (k >= nch) break;
      const int ch = channel_of(k);
      const bool isx = k < 64 * nh;
      if (k0 > 0) {
        cp.load(p, x, ch, steps_of(k), isx);
        cp.past(p, ring + ch, Ch, pos);
      }
      if (isx || hb == 0) *reinterpret_cast<Pair<T>*>(ring + (i64)(p.width == 4 ? pos & 3 : pos % p.width) * Ch + ch) = cp.own;
      const uint32_t c = cp.codes();
      if (isx) {
        *reinterpret_cast<uint16_t*>(&s.xnow[0][0] + k) = (uint16_t)c;
        *reinterpret_cast<uint16_t*>(p.c.xwin + ((sh0 + (k >> 6)) * kWin + now) * 64 + (k & 63)) = (uint16_t)c;
      } else {
        const int at = (k - 64 * nh) & (N - 1);
        const bool isC = k - 64 * nh >= N;
        *reinterpret_cast<uint16_t*>((isC ? s.C : s.B) + at) = (uint16_t)c;
        if (!isC && hb == 0) *reinterpret_cast<uint16_t*>(Bw + now * N + at) = (uint16_t)c;
      }
    }
  } else {
    // decays, two heads at a time, lane j of a half-warp for row j of the window
    if (lane < nh) p.c.dtwin[(sh0 + lane) * kWin + now] = dtn;
    const int rw = lane & 15, order = (rw - first) & (kWin - 1);
    float old[(HPC + 1) / 2], A[(HPC + 1) / 2];
#pragma unroll
    for (int i0 = 0; i0 < HPC; i0 += 2) {
      const int i = i0 + (lane >> 4);
      old[i0 / 2] = i < nh && order < n ? p.c.dtwin[(sh0 + i) * kWin + rw] : 0.f;
      A[i0 / 2] = i < nh ? p.A[h0 + i] : 0.f;
    }
#pragma unroll
    for (int i0 = 0; i0 < HPC; i0 += 2) {
      const int i = i0 + (lane >> 4);
      const float fresh = __shfl_sync(0xffffffffu, dtn, i & 31), dt = rw == now ? fresh : old[i0 / 2];
      const Waiting w = waiting_of(dt, order);
      if (i < nh) {
        s.w[i][rw] = dt * expf((float)((double)A[i0 / 2] * w.behind));
        if (rw == 0) s.E[i] = expf((float)((double)A[i0 / 2] * w.all));
      }
    }
  }
  __syncthreads();
  if (tid >= TS_T) return;
  // C . B_j, with the weights of the heads (0 for a row without a waiting token)
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
    if (piece < nh) s.g[piece][j] = s.w[piece][j] * (float)d;
  }
  const float sB = p.s_B[g], sC = p.s_C[g];
  named_bar(1, TS_T);
  // a thread's rows side by side: what they read of C is read once
  if (head >= nh) return;
  float win[QH];
  int d[QH];
#pragma unroll
  for (int q = 0; q < QH; ++q) {
    const int i = 4 * q + head;
    win[q] = 0.f;
    d[q] = 0;
    if (i < nh) {
      win[q] = s.g[i][now] * (float)s.xnow[i][row];   // the token itself; its row of s.x is stale
      if (!sm100::mbar_wait_inline<0>(&s.bar[i], 0, p.status)) drain();
    }
  }
#pragma unroll
  for (int k = 0; k < kWin; k += 4)
#pragma unroll
    for (int q = 0; q < QH; ++q) {
      const int i = min(4 * q + head, HPC - 1);
      const float4 w = *reinterpret_cast<const float4*>(&s.g[i][k]);
      const float gj[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) win[q] = fmaf(k + e == now ? 0.f : gj[e], (float)s.x[i][k + e][row], win[q]);
    }
  const uint4 C16 = reinterpret_cast<const uint4*>(s.C)[lane % LPR];
#pragma unroll
  for (int q = 0; q < QH; ++q) {
    int part[LPR];   // of rows lane / LPR + t 32 / LPR
    const uint4* const codes = reinterpret_cast<const uint4*>(&s.codes[min(4 * q + head, HPC - 1)][half][0]) + lane;
#pragma unroll
    for (int t = 0; t < LPR; ++t) part[t] = dot16(codes[32 * t], C16, 0);
    // each exchange halves the rows that a lane still has
#pragma unroll
    for (int k = LPR / 2; k >= 1; k >>= 1) {
      const bool up = lane & k;
#pragma unroll
      for (int t = 0; t < k; ++t) part[t] = (up ? part[t + k] : part[t]) + __shfl_xor_sync(0xffffffffu, up ? part[t] : part[t + k], k);
    }
    d[q] = part[0];
  }
#pragma unroll
  for (int q = 0; q < QH; ++q) {
    const int i = 4 * q + head;
    if (i < nh) {
      const float v = sC * fmaf(s.E[i] * scale[q], (float)d[q], sx[q] * sB * win[q]) + fmaf(D[q] * sx[q], (float)s.xnow[i][row], corr[q]);
      const i64 at = (i64)b * HP + (h0 + i) * 64 + row;
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
  p.H = d.H; p.G = d.G; p.hpg = d.H / d.G; p.softplus = softplus; p.ydt = ydt;
  auto go = [&](auto kernel, int hpc, size_t smem) -> ssdi8_status_t {
    const int hblocks = (p.hpg + hpc - 1) / hpc;
    if (d.G > 65535) return SSDI8_ERR_SHAPE;
    // (the grid's third axis holds 65535 sequences)
    for (p.b0 = 0; p.b0 < d.b; p.b0 += 65535) {
      const ssdi8_status_t s = launch_configured(kernel, dim3(hblocks, d.G, d.b - p.b0 < 65535 ? d.b - p.b0 : 65535), dim3(TS_ALL), smem, -1, false, st, p);
      if (s != SSDI8_OK) return s;
    }
    return SSDI8_OK;
  };
  auto pick = [&](auto hpc) -> ssdi8_status_t {
    constexpr int HPC = decltype(hpc)::value;
    return d.N == 128 ? go(token_kernel<T, 128, HPC>, HPC, sizeof(TokenSmem<128, HPC>) + 128)
                      : go(token_kernel<T, 64, HPC>, HPC, sizeof(TokenSmem<64, HPC>) + 128);
  };
  const int sms = sm_count();
  if (sms <= 0) return SSDI8_ERR_CUDA;
  // Eight heads to a block (three of them per SM) from a full wave on, four (four per SM) below that.  Steps without full windows, eight /
  // four / two heads, us: 250 x 128 heads 92.9 / 97.5 / 141, 64 x 80 (slots that stay in L2) 16.8 / 19.1 / 27.
  const bool eight = p.hpg > 4 && (i64)d.b * d.G * ((p.hpg + 7) / 8) >= 3 * sms;
  const ssdi8_status_t s = eight ? pick(std::integral_constant<int, 8>{}) : pick(std::integral_constant<int, 4>{});
  if (s != SSDI8_OK) return s;
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
