// Next tokens drawn from the head outputs: temperature, top-k, top-p and min-p
// from one given uniform number per request (paper Section 4.2: token-based FMs
// served with long-lived decode iterations; the outputs are a task's LM head's).
//
// Weights.  w_j = 2^t_j, t_j = (l_j - M) log2(e) / T <= 0, in fp64 (at full rate
// here: 11 fused multiply-adds of a polynomial after the split of t into its nearest
// integer and a rest of at most 1/2), rounded to 2^-44 (rows of more than 2^19 outputs:
// to what a 64-bit sum of them holds): the sums are then integers, exact in any
// order, so the order of atomics, the split over threads and the block's shape cannot
// change a result.  fp32 would shift the borders of the running sum by 1e-7 of it, and a
// vocabulary has so many of them that the token drawn would now and then be another.
//
// The three filters each keep a prefix of the outputs in descending order (ties
// by index), so only the last kept output has to be found, never a full order:
// outputs are counted (and their weights summed) in bins of equal width in l
// over the range where weights are not 0; the bin in which a filter ends is the
// only one that is put in order, and where all bins up to it hold few outputs
// (top-k), nothing else is looked at again.  One block per request: the row is
// read once where it fits registers or LDS (up to 32768 outputs).
//
// Bound by the weights' fp64 work, 19 instructions each on the one CU that a row
// has, and by the latency of the block's steps; bytes would allow 7 us for 256 rows
// of 32000.  Measured, 256 rows of 32000: greedy 7.1 us, no filter 15.2, top-k 40
// 12.2, top-k 199 24.1, top-k 1000 27.8, top-p 0.9 26, with min-p 31.  One such row: 5.8
// to 26.  48 rows of 100003 (48 of 256 CUs): no filter 30.3, top-p 0.9 54.3.  256 rows of
// 700: 6 (a call) to 11.2.
// Several blocks per row would need a second launch and scratch memory from the caller.
#include <type_traits>

#include "decode_internal.h"

namespace {

typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));

struct SampleParams {
  const float* temperature; const int32_t* top_k; const float* top_p; const float* min_p;
};

// 2^t, t <= 0, scaled by 2^sh and rounded to an integer.  t = n + f, |f| <= 1/2, and
// 2^f by the polynomial of degree 10 through 1 at 0 that interpolates it at the
// Chebyshev nodes (relative error 6e-16).  Adding 1.5 2^52 rounds t to n and leaves
// n (plus what is added beside it: the exponent field of 2^(n + sh)) in the low
// bits; adding 2^52 rounds the weight and leaves it there.  t below -100 (-inf) and
// NaN count as -100: 0.  No branch, so that a thread's four chains run beside each
// other.  The coefficients are made anew for every four outputs, in scalar registers:
// as literals each product would move one into a vector register, and held over the
// whole kernel they do not fit beside the rest.
struct Exp2 {
  double c[10], magic;
  __device__ __forceinline__ explicit Exp2(int sh) {
    magic = 6755399441055744.0 + (double)(1023 + sh);
    constexpr double k[10] = {7.0709785640393195e-09, 1.0205905435457491e-07, 1.3215451629202315e-06,
                              1.5252672924749049e-05, 1.5403530424784571e-04, 1.3333558200794733e-03,
                              9.6181291076186601e-03, 5.5504108664651670e-02, 2.4022650695910075e-01,
                              6.9314718055994617e-01};
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      c[i] = k[i];
      asm volatile("" : "+s"(c[i]));
    }
  }
  // the weight beside the bits of 2^52, which a sum takes out at its end
  static constexpr uint64_t BIAS = 0x4330000000000000ull;
  __device__ __forceinline__ uint64_t biased(double t) const {
    t = fmax(t, -100.0);
    const double x = t + magic, f = t - (x - magic);
    double p = c[0];
#pragma unroll
    for (int i = 1; i < 10; ++i) p = fma(p, f, c[i]);
    p = fma(p, f, 1.0);
    const uint32_t e = (uint32_t)__double_as_longlong(x) << 20;        // of 2^(n + sh): a normal number
    const double d = fma(p, __longlong_as_double((long long)((uint64_t)e << 32)), 4503599627370496.0);
    return (uint64_t)__double_as_longlong(d);
  }
  __device__ __forceinline__ uint64_t operator()(double t) const { return biased(t) & 0xFFFFFFFFFFFFFull; }
};

// ln x, x >= 1: x = 2^e m, m in [2/3, 4/3), ln m = 2 atanh((m - 1) / (m + 1)) by its
// series (|s| <= 1/5: the first term left out is below 1e-13).
__device__ __forceinline__ double log_of(double x) {
  int e = __builtin_amdgcn_frexp_exp(x);
  double m = __builtin_amdgcn_frexp_mant(x);             // [1/2, 1)
  if (m < 2.0 / 3.0) { m *= 2.0; --e; }
  const double s = (m - 1.0) / (m + 1.0), z = s * s;
  double p = 2.0 / 15;
  p = fma(p, z, 2.0 / 13);
  p = fma(p, z, 2.0 / 11);
  p = fma(p, z, 2.0 / 9);
  p = fma(p, z, 2.0 / 7);
  p = fma(p, z, 2.0 / 5);
  p = fma(p, z, 2.0 / 3);
  p = fma(p, z, 2.0);
  return fma((double)e, 0.6931471805599453, p * s);
}

// Integers in the order of the floats (no NaN); -0 and +0 are one.
__device__ __forceinline__ uint32_t float_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

// Sums, maxima and scans over a wave with DPP moves (no LDS round trips); every
// lane is active.  A 64-bit value moves as two halves.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp0(uint32_t v) {   // 0 where no lane is the source
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, true);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp0(uint64_t v) {
  return ((uint64_t)dpp0<CTRL, ROWS>((uint32_t)(v >> 32)) << 32) | dpp0<CTRL, ROWS>((uint32_t)v);
}
// inclusive sums over the lanes: within rows of 16 lanes, then lane 15 of rows
// 0 and 2 into the row behind, then lane 31 into the upper half
template <typename T>
__device__ __forceinline__ T wave_scan(T v) {
  v += dpp0<0x111, 0xF>(v);
  v += dpp0<0x112, 0xF>(v);
  v += dpp0<0x114, 0xF>(v);
  v += dpp0<0x118, 0xF>(v);
  v += dpp0<0x142, 0xA>(v);
  v += dpp0<0x143, 0xC>(v);
  return v;
}
__device__ __forceinline__ uint32_t last_lane(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, 63); }
__device__ __forceinline__ uint64_t last_lane(uint64_t v) {
  return ((uint64_t)last_lane((uint32_t)(v >> 32)) << 32) | last_lane((uint32_t)v);
}
// every LDS access of the wave has finished (reads whose values a path does not use among them)
__device__ __forceinline__ void lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
template <typename T> __device__ __forceinline__ T wave_sum(T v) { return last_lane(wave_scan(v)); }

// maximum over aligned groups of 2^(S + 1) lanes from that over groups of 2^S, in every lane
template <int S>
__device__ __forceinline__ uint32_t lane_pair(uint32_t v) {
  static_assert(S >= 0 && S < 6, "64 lanes");
  if constexpr (S == 0) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);
  if constexpr (S == 1) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);
  if constexpr (S == 2) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true);   // 7 - lane of 8
  if constexpr (S == 3) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true);   // 15 - lane of 16
  // the two results of a lane swap are the lane's own value and its partner's, in one order or the other
  if constexpr (S == 4) { const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false); return r[0] ^ r[1] ^ v; }
  const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return r[0] ^ r[1] ^ v;
}
template <int S> __device__ __forceinline__ float lane_pair(float v) { return __uint_as_float(lane_pair<S>(__float_as_uint(v))); }
template <int S = 0>
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, lane_pair<S>(v));
  if constexpr (S < 5) return wave_max<S + 1>(v);
  else return v;
}
template <int S = 0>
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, lane_pair<S>(v));
  if constexpr (S < 5) return wave_max<S + 1>(v);
  else return v;
}

// Where a row's outputs are between the passes over them.
enum { IN_REGS = 0, IN_LDS = 1, IN_MEMORY = 2 };
template <int NT, int WHERE> struct Shape;
// up to 1024 outputs: 4 per thread in registers
template <> struct Shape<256, IN_REGS> { static constexpr int RUNS = 1, PB = 256, SETS = 4; };
// up to 32768: 128 KB of LDS, which leaves room for 4 sets of bins of weights
template <> struct Shape<1024, IN_LDS> { static constexpr int RUNS = 8, PB = 512, SETS = 4; };
// more: read again (from L2) by every pass; a set of bins per wave
template <> struct Shape<1024, IN_MEMORY> { static constexpr int RUNS = 0, PB = 1024, SETS = 16; };

template <int NT, int WHERE>
__global__ __launch_bounds__(NT) void sample_kernel(Plan pl, const float* __restrict__ out, SampleParams sp,
                                                    const float* __restrict__ us, int32_t* __restrict__ ids,
                                                    float* __restrict__ logprob) {
  using Sh = Shape<NT, WHERE>;
  constexpr int NW = NT / 64, NB = NT;
  constexpr int CAP = NT == 256 ? 256 : 512;   // outputs that are put in order at once, each against each
  constexpr int NG = 256;              // at most this many groups of threads, whose largest outputs bound a top-k from below
  constexpr int PB = Sh::PB, SETS = Sh::SETS, PER = NW / SETS;   // bins of weights; sets of them; waves per set
  __shared__ __attribute__((aligned(16))) float s_row[WHERE == IN_LDS ? NT * 4 * Sh::RUNS : 4];
  __shared__ float red_f[2][NW];
  __shared__ uint64_t red_u[NW], set_u[SETS], run_u[64];
  __shared__ uint32_t red_c[2][NW];
  // bins: weights per set and bin (top-p), or of all outputs (a bin's weight, then up to and with it; its outputs)
  constexpr size_t BINS = SETS * PB * 8 > NB * 12 ? SETS * PB * 8 : NB * 12;
  __shared__ __attribute__((aligned(16))) char s_bins[BINS];
  __shared__ __attribute__((aligned(16))) uint64_t l_key[CAP + 8];   // (float_key, ~index): descending order; then running sums
  __shared__ uint64_t l_sorted[CAP], l_mass[CAP];
  __shared__ uint32_t l_rank[CAP];
  __shared__ uint32_t s_n, s_listed[2], s_sel[3];   // kept outputs; listed ones, by turns; bin, outputs before it, outputs in it
  __shared__ uint64_t s_before;
  __shared__ float s_bound;
  auto h_mass = [&](int b) -> uint64_t& { return reinterpret_cast<uint64_t*>(s_bins)[b]; };
  auto h_cnt = [&](int b) -> uint32_t& { return reinterpret_cast<uint32_t*>(s_bins + NB * 8)[b]; };
  auto set_mass = [&](int set, int b) -> uint64_t& { return reinterpret_cast<uint64_t*>(s_bins)[set * PB + b]; };
  uint64_t* const l_cum = l_key;
  float* const g_max = reinterpret_cast<float*>(l_sorted);   // the groups' largest outputs and their ranks, before any list
  static_assert(CAP * 8 >= NG * 4 && CAP >= NG / 2, "");

  const int row = blockIdx.x;
  const int o0 = pl.out_off[row], n = pl.out_off[row + 1] - o0;
  const float* src = out + o0;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nr = (n + NT * 4 - 1) / (NT * 4);          // runs of 256 outputs per wave; a wave's runs are one piece
  const int first = wave * nr * 256 + lane * 4;
  // the row's parameters, requested with its first outputs
  const float temp = sp.temperature ? sp.temperature[row] : 1.f;
  const int tk = sp.top_k ? sp.top_k[row] : 0;
  const float tp = sp.top_p ? sp.top_p[row] : 1.f, mp = sp.min_p ? sp.min_p[row] : 0.f;
  const float u_row = us[row];

  const float nan = __uint_as_float(0x7FC00000u);
  // An infinite largest output M0: those that equal it share the weight, the others have none.
  // Once `remap` is set the row is taken as 0 there and as -inf elsewhere.
  float M0 = -INFINITY;
  bool remap = false;
  auto mapped = [&](float v) { return v == M0 ? 0.f : v == v ? -INFINITY : v; };
  auto fetch_at = [&](int i) -> f4u {
    f4u v = {nan, nan, nan, nan};
    if (i + 4 <= n) v = *reinterpret_cast<const f4u*>(src + i);
    else
#pragma unroll
      for (int c = 0; c < 4; ++c) if (i + c < n) v[c] = src[i + c];
    if (WHERE == IN_MEMORY && remap)
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = mapped((float)v[c]);
    return v;
  };
  f4u reg = {nan, nan, nan, nan};
  if constexpr (WHERE == IN_REGS) reg = fetch_at(first);
  // the four outputs from index i, which some thread of the block owns (registers: this one)
  auto at = [&](int i) -> f4u {
    if constexpr (WHERE == IN_REGS) return reg;
    else if constexpr (WHERE == IN_LDS) { const f32x4 q = *reinterpret_cast<const f32x4*>(&s_row[i]); return f4u{q[0], q[1], q[2], q[3]}; }
    else return fetch_at(i);
  };
  // f(four values, index of the first) for every run of the wave, in order
  auto each4 = [&](auto&& f) {
    if constexpr (WHERE == IN_MEMORY) {
      for (int r0 = 0; r0 < nr; r0 += 4) {               // four runs' loads in flight
        f4u q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = r0 + j < nr ? fetch_at(first + (r0 + j) * 256) : f4u{nan, nan, nan, nan};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (r0 + j < nr) f(q[j], first + (r0 + j) * 256);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    } else {
      for (int r = 0; r < nr; ++r) f(at(first + r * 256), first + r * 256);
    }
  };
  auto each = [&](auto&& f) {                            // f(value, index) for every output of the thread
    each4([&](const f4u& q, int i0) {
#pragma unroll
      for (int c = 0; c < 4; ++c) f((float)q[c], i0 + c);
    });
  };

  // 0: off.  No weight reaches a min-p above 1: the first output alone stays
  const int k = mp > 1.f && n > 1 ? 1 : tk > 0 && tk < n ? tk : 0;
  const bool p_on = tp < 1.f;
  const double p = (double)tp;
  // (registers: up to 56, where bins take 7.7 us for 256 rows of 1000 and a list of twice as many as k 14 and more)
  const bool small_k = k > 0 && k <= (WHERE == IN_REGS ? 56 : NG);   // block-uniform, as every branch on the row's values below
  const double T = fmin(fmax((double)temp, 1e-30), 1e30);
  const double c2 = 1.4426950408889634 / T;
  if (tid < 2) s_listed[tid] = 0;
  int turn = 0;
  if (p_on && k == 0)                                    // while the row's loads are in flight
    for (int b = tid; b < SETS * PB; b += NT) set_mass(0, b) = 0;

  // The largest and the smallest output, and for a small top-k the largest of each
  // of 256 groups of threads
  float mx = -INFINITY, mn = INFINITY;
  if constexpr (WHERE == IN_LDS) {
    f4u q[Sh::RUNS];
#pragma unroll
    for (int r = 0; r < Sh::RUNS; ++r) q[r] = r < nr ? fetch_at(first + r * 256) : f4u{nan, nan, nan, nan};
#pragma unroll
    for (int r = 0; r < Sh::RUNS; ++r)
      if (r < nr) {
        *reinterpret_cast<f32x4*>(&s_row[first + r * 256]) = f32x4{q[r][0], q[r][1], q[r][2], q[r][3]};
#pragma unroll
        for (int c = 0; c < 4; ++c) { mx = fmaxf(mx, q[r][c]); mn = fminf(mn, q[r][c]); }
      }
  } else {
    each([&](float v, int) { mx = fmaxf(mx, v); mn = fminf(mn, v); });
  }
  const bool any = mn <= mx;                             // some output is no NaN
  // 64 groups up to k = 56 (then some 150 outputs lie above the 56th of them), else 256
  const int lgg = k <= 56 ? 6 : 8, per_group = NT >> lgg;   // threads per group: 16 or 4 of 1024, 4 of 256
  if (small_k) {
    float gm = mx;
    gm = fmaxf(gm, lane_pair<0>(gm));
    gm = fmaxf(gm, lane_pair<1>(gm));
    if (per_group >= 16) {
      gm = fmaxf(gm, lane_pair<2>(gm));
      gm = fmaxf(gm, lane_pair<3>(gm));
    }
    if ((tid & (per_group - 1)) == 0) g_max[tid / per_group] = gm;
    if (tid < NG) l_rank[tid % CAP] = 0;
  }
  {
    const float lo = -wave_max(-mn);
    mx = wave_max(mx);
    const bool anyw = __any(any);
    if (lane == 0) { red_f[0][wave] = mx; red_f[1][wave] = lo; red_c[1][wave] = anyw; }
  }
  __syncthreads();
  const int wl = lane % NW;                              // (short code: each block runs it once, from a cold cache)
  M0 = wave_max(red_f[0][wl]);
  mn = -wave_max(-red_f[1][wl]);
  const bool found = __any(red_c[1][wl]);
  if (!found) {
    if (tid == 0) { ids[row] = -1; if (logprob) logprob[row] = nan; }
    return;
  }
  if (!(temp > 0.f)) {                                   // greedy
    uint32_t best = 0;                                   // ~index: the largest is the lowest index
    each([&](float v, int i) { if (v == M0) best = max(best, ~(uint32_t)i); });
    best = wave_max(best);
    __syncthreads();                                     // red_c is read above
    if (lane == 0) red_c[0][wave] = best;
    __syncthreads();
    if (tid == 0) {
      for (int i = 1; i < NW; ++i) best = max(best, red_c[0][i]);
      ids[row] = (int)~best;
      if (logprob) logprob[row] = 0.f;
    }
    return;
  }
  float M = M0;
  if (!(fabsf(M0) < INFINITY)) {
    remap = true;
    M = 0.f;
    mn = -INFINITY;
    if constexpr (WHERE == IN_REGS) {
#pragma unroll
      for (int c = 0; c < 4; ++c) reg[c] = mapped((float)reg[c]);
    } else if constexpr (WHERE == IN_LDS) {
      for (int r = 0; r < nr; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) s_row[first + r * 256 + c] = mapped(s_row[first + r * 256 + c]);
      __syncthreads();
    }
  }
  const int sh = min(44, 31 + __builtin_clz((n - 1) | 1));   // 63 - ceil(log2 n): n weights of 2^sh sum to 2^63 at most
  const uint64_t one = (uint64_t)1 << sh;
  const float cut = fminf((float)(31.2 * T), 3e38f);     // 45 ln 2: below M - cut every weight is 0
  auto power = [&](float v) { return ((double)v - (double)M) * c2; };
  auto mass = [&](float v) -> uint64_t { return Exp2(sh)(power(v)); };
  auto value_of = [&](uint32_t key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu)); };
  const double uu = u_row > 0.f ? (double)u_row : 0.0;   // NaN: 0
  auto target_of = [&](uint64_t S) {
    const uint64_t t = (uint64_t)fmin(uu * (double)S, 1.8e19);   // above any S (2^63), below 2^64
    return t < S - 1 ? t : S - 1;
  };
  auto finish = [&](float v, int i, uint64_t total) {    // one thread: the drawn output
    ids[row] = i;
    if (logprob) logprob[row] = (float)(((double)v - (double)M) / T - log_of((double)total) + (double)sh * 0.6931471805599453);
  };

  // The outputs that f(value, index) picks, if they are at most CAP: in descending order in
  // l_sorted, their weights in l_mass and running sums in l_cum.  Returns their number.
  // One pass: a wave that finds some takes places behind those taken before; the order of the
  // places does not matter, and a wave that finds no place left stops.
  // by_index: each one's place in the order of the indices, at its place in l_sorted, in l_rank.
  auto list = [&](auto by_index, auto&& f) -> uint32_t {
    if (tid < CAP) l_rank[tid] = 0;
    __syncthreads();                                     // the list of before, and its number, have been read
    turn ^= 1;
    if (tid == 0) s_listed[turn ^ 1] = 0;
    bool room = true;
    each4([&](const f4u& q, int i0) {
      bool hit[4];
      uint64_t m[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) { hit[c] = f((float)q[c], i0 + c); m[c] = __ballot(hit[c]); }
      if (room && (m[0] | m[1] | m[2] | m[3])) {
        uint32_t base = 0;
        if (lane == 0) base = atomicAdd(&s_listed[turn], (uint32_t)(__popcll(m[0]) + __popcll(m[1]) + __popcll(m[2]) + __popcll(m[3])));
        base = (uint32_t)__builtin_amdgcn_readfirstlane((int)base);
        room = base < (uint32_t)CAP;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t pos = base + __builtin_amdgcn_mbcnt_hi((uint32_t)(m[c] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m[c], 0));
          if (hit[c] && pos < (uint32_t)CAP) l_key[pos] = ((uint64_t)float_key((float)q[c]) << 32) | (uint32_t)~(i0 + c);
          base += (uint32_t)__popcll(m[c]);
        }
      }
    });
    __syncthreads();
    const uint32_t cnt = s_listed[turn];                 // more than CAP: some that were not counted
    if (cnt > CAP) return cnt;
    if (tid < 8) l_key[cnt + tid] = 0;                   // below every key
    __syncthreads();
    // every listed output against every other: 2^lg of them at a time, the others split among the rest of the block
    const int lg = cnt <= 64 ? 6 : 32 - __builtin_clz(cnt - 1), parts = NT >> lg;
    const uint32_t e = tid & ((1 << lg) - 1), len = (cnt / parts + 8) & ~7u;
    const uint32_t j0 = (tid >> lg) * len, j1 = min(j0 + len, (cnt + 7) & ~7u);
    if (parts > 0 && j0 < j1) {
      const uint64_t me = l_key[min(e, cnt)];
      uint32_t r = 0;                                    // larger keys; in the upper half, smaller indices
      for (uint32_t j = j0; j < j1; j += 8) {
        u64x2 q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const u64x2*>(&l_key[j + 2 * i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) r += (uint32_t)(q[i][0] > me) + (uint32_t)(q[i][1] > me);
        if constexpr (by_index)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            r += ((uint32_t)q[i][0] > (uint32_t)me ? 1u << 16 : 0u) + ((uint32_t)q[i][1] > (uint32_t)me ? 1u << 16 : 0u);
      }
      if (e < cnt) atomicAdd(&l_rank[e], r);
    }
    __syncthreads();
    const uint32_t ranks = tid < CAP ? l_rank[tid] : 0;
    if ((uint32_t)tid < cnt) l_sorted[ranks & 0xFFFF] = l_key[tid];
    __syncthreads();
    if constexpr (by_index)
      if ((uint32_t)tid < cnt) l_rank[ranks & 0xFFFF] = ranks >> 16;
    uint64_t w = 0;
    if ((uint32_t)tid < cnt) w = mass(value_of((uint32_t)(l_sorted[tid] >> 32)));
    const uint64_t cw = wave_scan(w);
    if (lane == 63) red_u[wave] = cw;
    __syncthreads();
    uint64_t before = 0;
#pragma unroll
    for (int i = 0; i < CAP / 64; ++i) before += i < wave ? red_u[i] : 0;
    if (tid < CAP) { l_mass[tid] = w; l_cum[tid] = cw + before; }
    __syncthreads();
    return cnt;
  };

  const uint64_t least = mp > 0.f ? (uint64_t)ceil(fmin((double)mp, 1.0) * (double)one) : 0;   // min-p's smallest weight

  // ---- a small top-k: the k-th largest of the groups' largest outputs bounds it from below;
  // what is not below that fits the list as a rule, and nothing else is needed ----
  if (small_k) {
    // each group against 2^lgg / per_group of the others per thread
    const int groups = 1 << lgg, len = groups / per_group;
    const int me = tid & (groups - 1), j0 = (tid >> lgg) * len;
    const float g = g_max[me];
    uint32_t r = 0;
#pragma unroll 4
    for (int j = j0; j < j0 + len; j += 4) {
      const f32x4 q = *reinterpret_cast<const f32x4*>(&g_max[j]);
#pragma unroll
      for (int c = 0; c < 4; ++c) r += (uint32_t)((q[c] > g) | ((q[c] == g) & (j + c < me)));
    }
    atomicAdd(&l_rank[me], r);                           // at most 256 of 1024 or 64 of 256 threads' groups: within l_rank
    __syncthreads();
    r = l_rank[me];
    if (tid < groups && r == (uint32_t)k - 1) s_bound = remap ? -INFINITY : g;
    __syncthreads();
    const float bound = s_bound;
    const uint32_t cnt = list(std::true_type{}, [&](float v, int) { return v >= bound; });
    if (cnt <= CAP) {
      const uint32_t nk = min((uint32_t)k, cnt);
      const double target = p_on ? p * (double)l_cum[nk - 1] : INFINITY;
      auto keep = [&](uint32_t q) {
        return q == 0 || (q < nk && (double)l_cum[q - 1] < target && l_mass[q] >= least);
      };
      const bool mine = (uint32_t)tid < nk && keep(tid);
      if (mine && !((uint32_t)tid + 1 < nk && keep(tid + 1))) s_n = tid + 1;
      __syncthreads();
      const uint32_t kept = s_n;
      const uint64_t S = l_cum[kept - 1];
      const uint64_t tgt = target_of(S);
      // the listed ones in the order of their indices: weight (0 unless kept) and place
      uint64_t* const x_mass = reinterpret_cast<uint64_t*>(s_bins);
      uint32_t* const x_at = reinterpret_cast<uint32_t*>(s_bins + CAP * 8);
      static_assert(BINS >= CAP * 12, "");
      if ((uint32_t)tid < cnt) { x_mass[l_rank[tid]] = (uint32_t)tid < kept ? l_mass[tid] : 0; x_at[l_rank[tid]] = tid; }
      __syncthreads();
      const uint64_t x = (uint32_t)tid < cnt ? x_mass[tid] : 0;
      uint64_t c = wave_scan(x);
      if (lane == 63) red_u[wave] = c;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < CAP / 64; ++i) c += i < wave ? red_u[i] : 0;
      if (c > tgt && c - x <= tgt) {
        const uint64_t it = l_sorted[x_at[tid]];
        finish(value_of((uint32_t)(it >> 32)), (int)~(uint32_t)it, S);
      }
      return;
    }
  }

  float v_last = -INFINITY;                              // the last kept output: its value and index
  int i_last = INT32_MAX;
  auto above = [&](float v, int i) { return (v > v_last) | ((v == v_last) & (i <= i_last)); };   // NaN: no

  // bins of equal width in l from M down to `low` (or where weights end): -1 past it, and for a NaN
  auto bin_of = [&](float v, float range, float scale, int bins) -> int {
    const float d = M - v;
    const int b = (int)fminf(d * scale, (float)(bins - 1));
    return d <= range ? b : -1;
  };
  auto range_to = [&](float low) { const float d = M - low; return d < cut ? d : cut; };
  auto scale_of = [&](float range, int bins) { return range > 0.f ? fminf((float)bins / range, 3e38f) : 0.f; };

  // block-wide inclusive scan of NB bins in place: h_cnt and h_mass
  auto scan_bins = [&]() {
    const uint32_t cw = wave_scan(h_cnt(tid));
    const uint64_t mw = wave_scan(h_mass(tid));
    if (lane == 63) { red_c[0][wave] = cw; red_u[wave] = mw; }
    __syncthreads();
    uint32_t cb = 0;
    uint64_t mb = 0;
    for (int i = 0; i < wave; ++i) { cb += red_c[0][i]; mb += red_u[i]; }
    h_cnt(tid) = cw + cb;
    h_mass(tid) = mw + mb;
    __syncthreads();
  };
  // the bin in which the j-th output (j > 0) or the weight `target` lies; c0, m0: what lies before the bins
  auto select = [&](uint32_t j, double target, uint32_t c0, uint64_t m0) {
    const uint32_t ce = tid ? h_cnt(tid - 1) : 0, ci = h_cnt(tid);
    const uint64_t me = m0 + (tid ? h_mass(tid - 1) : 0), mi = m0 + h_mass(tid);
    const bool hit = j > 0 ? c0 + ce < j && c0 + ci >= j
                           : ci > ce && (double)mi >= target && ((double)me < target || c0 + ce == 0);
    if (hit) { s_sel[0] = tid; s_sel[1] = c0 + ce; s_sel[2] = ci - ce; s_before = me; }
    __syncthreads();
  };
  // The last output of a prefix of the kept ones: the j-th (j > 0), or the one with which the
  // weight reaches `target`; nothing changes where there are fewer with any weight (j).  The general
  // way: bins of l, then bins of the floats' own order within one bin, until what is left fits the list.
  auto resolve = [&](uint32_t j, double target, float low) {
    const bool masses = j == 0;
    const float range = range_to(low), scale = scale_of(range, NB);
    auto clear = [&]() {
      lds_done();
      __syncthreads();
      h_cnt(tid) = 0;
      h_mass(tid) = 0;
      __syncthreads();
    };
    auto add = [&](int b, float v) {
      atomicAdd(&h_cnt(b), 1u);
      if (masses) atomicAdd((unsigned long long*)&h_mass(b), (unsigned long long)mass(v));
    };
    clear();
    each([&](float v, int i) {
      const int b = bin_of(v, range, scale, NB);
      if (b >= 0 && above(v, i)) add(b, v);
    });
    __syncthreads();
    scan_bins();
    if (j > h_cnt(NB - 1)) return;
    select(j, target, 0, 0);
    const int bin = (int)s_sel[0];
    uint32_t before = s_sel[1], cnt = s_sel[2];
    uint64_t m0 = s_before;
    uint32_t lo = 0, hi = 0;                             // the bin's outputs as a range of keys
    bool keys = false;
    auto inside = [&](float v, int i) -> bool {
      const uint32_t q = float_key(v);
      return above(v, i) & (keys ? (q >= lo) & (q <= hi) : bin_of(v, range, scale, NB) == bin);
    };
    while (cnt > CAP) {
      uint32_t a = 0, z = 0;                             // ~smallest, largest key
      each([&](float v, int i) {
        if (inside(v, i)) { const uint32_t q = float_key(v); a = max(a, ~q); z = max(z, q); }
      });
      a = wave_max(a);
      z = wave_max(z);
      __syncthreads();
      if (lane == 0) { red_c[0][wave] = a; red_c[1][wave] = z; }
      __syncthreads();
      for (int i = 0; i < NW; ++i) { a = max(a, red_c[0][i]); z = max(z, red_c[1][i]); }
      lo = ~a; hi = z; keys = true;
      if (lo == hi) break;                               // all equal: by index alone
      const int shift = max(0, 32 - __builtin_clz(hi - lo) - (31 - __builtin_clz(NB)));
      clear();
      each([&](float v, int i) { if (inside(v, i)) add((int)((hi - float_key(v)) >> shift), v); });
      __syncthreads();
      scan_bins();
      select(j, target, before, m0);
      const uint32_t b = s_sel[0];
      before = s_sel[1]; cnt = s_sel[2]; m0 = s_before;
      hi -= b << shift;
      const uint32_t below = (1u << shift) - 1;
      lo = hi - lo > below ? hi - below : lo;
    }
    if (cnt > CAP) {                                     // the x-th of equal outputs, by index
      const float v = value_of(lo);
      const uint64_t w = mass(v);
      uint32_t want;
      if (j > 0) want = j - before;
      else {
        const double need = (target - (double)m0) / (double)(w ? w : 1);
        want = need <= 1.0 ? 1u : need >= (double)cnt ? cnt : (uint32_t)ceil(need);
      }
      uint32_t mine = 0;
      each([&](float q, int i) { mine += (q == v) & above(q, i); });
      mine = wave_sum(mine);
      __syncthreads();
      if (lane == 0) red_c[0][wave] = mine;
      __syncthreads();
      uint32_t skip = 0;
      int wv = 0;
      while (wv < NW - 1 && skip + red_c[0][wv] < want) skip += red_c[0][wv++];
      if (wave == wv) {
        each4([&](const f4u& q, int i0) {
          uint32_t c4 = 0;
#pragma unroll
          for (int c = 0; c < 4; ++c) c4 += ((float)q[c] == v) & above((float)q[c], i0 + c);
          const uint32_t inc = wave_scan(c4), tot = last_lane(inc);
          uint32_t x = skip + inc - c4;
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if ((float)q[c] == v && above((float)q[c], i0 + c) && ++x == want) s_sel[0] = (uint32_t)(i0 + c);
          skip += tot;
        });
      }
      __syncthreads();
      v_last = v;
      i_last = (int)s_sel[0];
      __syncthreads();
      return;
    }
    list(std::false_type{}, inside);
    if ((uint32_t)tid < cnt) {
      const uint64_t me = m0 + l_cum[tid] - l_mass[tid], mi = m0 + l_cum[tid];
      const bool hit = j > 0 ? before + tid + 1 == j
                             : ((double)mi >= target || (uint32_t)tid + 1 == cnt) && ((double)me < target || before + tid == 0);
      if (hit) s_sel[0] = tid;
    }
    __syncthreads();
    const uint64_t e = l_sorted[s_sel[0]];
    __syncthreads();
    v_last = value_of((uint32_t)(e >> 32));
    i_last = (int)~(uint32_t)e;
  };

  // ---- a large top-k, then top-p.  Top-p: the kept weights in bins, in several sets by wave: the
  // sums up to the last kept output are then each set's share of the kept weight ----
  bool have = false;                                     // set_u holds the sets' kept weights
#pragma unroll 1
  for (int stage = 0; stage < 2; ++stage) {
    if (stage == 0 ? k == 0 : !p_on) continue;
    uint32_t j = (uint32_t)k;
    double target = 0.0;
    const float low = fmaxf(mn, v_last);
    if (stage == 1) {
      const float range = range_to(low), scale = scale_of(range, PB);
      const int set = wave / PER;
      if (k > 0) {                                       // cleared at the start, but the top-k has used them
        lds_done();
        __syncthreads();
        for (int b = tid; b < SETS * PB; b += NT) set_mass(0, b) = 0;
        __syncthreads();
      }
      // an output without a weight (a NaN, too) adds nothing anywhere
      auto into_bins = [&](auto all) {
        each4([&](const f4u& q, int i0) {
          const Exp2 weight(sh);
          uint64_t w[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) w[c] = weight(power((float)q[c]));
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int b = (int)fminf((M - (float)q[c]) * scale, (float)(PB - 1));
            if ((w[c] != 0) & (all || above((float)q[c], i0 + c)))
              atomicAdd((unsigned long long*)&set_mass(set, b), (unsigned long long)w[c]);
          }
        });
      };
      if (k == 0) into_bins(std::true_type{});
      else into_bins(std::false_type{});
      __syncthreads();
      uint64_t sum = 0;
      if (tid < PB)
#pragma unroll
        for (int i = 0; i < SETS; ++i) sum += set_mass(i, tid);
      const uint64_t cw = wave_scan(sum);
      if (lane == 63) red_u[wave] = cw;
      __syncthreads();
      uint64_t incl = cw, total = 0;
#pragma unroll
      for (int i = 0; i < NW; ++i) { incl += i < wave ? red_u[i] : 0; total += red_u[i]; }
      target = p * (double)total;
      if (tid < PB) {
        const uint64_t excl = incl - sum;
        if (sum > 0 && (double)incl >= target && ((double)excl < target || excl == 0)) { s_sel[1] = tid; s_before = excl; }
      }
      __syncthreads();
      const int bin = (int)s_sel[1];
      const uint64_t m0 = s_before;
      // in the bin, by its borders: what truncation takes to it
      const float b0 = (float)bin, b1 = bin == PB - 1 ? INFINITY : (float)(bin + 1);
      const uint32_t cnt = list(std::false_type{}, [&](float v, int i) {
        const float d = M - v, x = d * scale;
        return (x >= b0) & (x < b1) & (d <= range) & above(v, i);
      });
      if (cnt <= CAP) {
        if ((uint32_t)tid < cnt) {
          const uint64_t me = m0 + l_cum[tid] - l_mass[tid], mi = m0 + l_cum[tid];
          if (((double)mi >= target || (uint32_t)tid + 1 == cnt) && ((double)me < target || (m0 == 0 && tid == 0))) s_sel[0] = tid;
        }
        uint64_t mine = 0;                               // one wave per set sums its bins before the last
        if (wave < SETS)
          for (int b = lane; b < bin; b += 64) mine += set_mass(wave, b);
        mine = wave_sum(mine);
        if (lane == 0 && wave < SETS) set_u[wave] = mine;
        __syncthreads();
        const uint32_t last = s_sel[0];
        if ((uint32_t)tid <= last) {
          const int i = (int)~(uint32_t)l_sorted[tid];
          atomicAdd((unsigned long long*)&set_u[i / (nr * 256 * PER)], (unsigned long long)l_mass[tid]);
        }
        const uint64_t e = l_sorted[last];
        v_last = value_of((uint32_t)(e >> 32));
        i_last = (int)~(uint32_t)e;
        have = l_mass[last] >= least;                    // else min-p keeps fewer still
        __syncthreads();
        continue;
      }
      j = 0;
    }
    resolve(j, target, low);
  }

  // ---- the draw: the waves' (or sets') kept weights, then the run of outputs that holds u times their sum ----
  float v_least = v_last;
  // below this, with room for every rounding, min-p keeps nothing (the weights themselves decide above it)
  if (mp > 0.f)
    v_least = fmaxf(v_least, (float)((double)M + T * ((double)__builtin_amdgcn_logf(fminf(mp, 1.f)) * 0.6932165 - 1e-5) -
                                     1e-5 * fabs((double)M)));
  // the kept weights of four outputs (0 for the others); returns their sum
  auto kept4 = [&](const f4u& q, int i0, uint64_t (&w)[4]) -> uint64_t {
    float x[4];
    bool any4 = false;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float v = (float)q[c];
      const bool in = (v >= v_least) & ((v != v_last) | (i0 + c <= i_last));            // NaN: no
      x[c] = in ? v : -INFINITY;
      any4 |= in;
      w[c] = 0;
    }
    if (any4) {
      const Exp2 weight(sh);
#pragma unroll
      for (int c = 0; c < 4; ++c) w[c] = weight(power(x[c]));
      if (mp > 0.f)
#pragma unroll
        for (int c = 0; c < 4; ++c) w[c] = w[c] >= least ? w[c] : 0;
    }
    return w[0] + w[1] + w[2] + w[3];
  };
  uint64_t S = 0, acc = 0;
  if (!have) {
    __syncthreads();                                     // red_u has been read
    uint64_t sum = 0;
    if (k == 0 && !p_on && !(mp > 0.f)) {                // no filter: every weight
      each4([&](const f4u& q, int) {
        const Exp2 weight(sh);
#pragma unroll
        for (int c = 0; c < 4; ++c) sum += weight.biased(power((float)q[c]));
      });
      sum -= (uint64_t)(4 * nr) * Exp2::BIAS;
    } else {
      each4([&](const f4u& q, int i0) { uint64_t w[4]; sum += kept4(q, i0, w); });
    }
    sum = wave_sum(sum);
    if (lane == 0) red_u[wave] = sum;
    __syncthreads();
  }
  // the piece (a wave's runs, or a set's) that holds the target
  const int pieces = have ? SETS : NW, per = have ? PER * nr : nr;
  // the first of the wave's 64 values (the later ones 0) with which acc passes tgt, the last of m if none: its
  // lane; acc is then what lies before it
  auto find = [&](uint64_t v, uint64_t tgt, int m) -> int {
    const uint64_t c = wave_scan(v) + acc;
    const uint64_t over = __ballot(c > tgt);
    const int i = over ? min((int)__builtin_ctzll(over), m - 1) : m - 1;
    const uint64_t before = c - v;
    acc = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(before >> 32), i) << 32) |
          (uint32_t)__builtin_amdgcn_readlane((int)before, i);
    return i;
  };
  const uint64_t part = lane < pieces ? (have ? set_u[lane] : red_u[lane]) : 0;
  S = wave_sum(part);
  const uint64_t tgt = target_of(S);
  const int piece = find(part, tgt, pieces);
  int run = 0;                                           // the piece's run
  if constexpr (WHERE == IN_REGS) {
    if (wave != piece) return;                           // a piece is one run
  } else {
    // its runs, 64 at a time, among all waves
    for (;;) {
      for (int i = wave; i < 64 && run + i < per; i += NW) {
        const int i0 = (piece * per + run + i) * 256 + lane * 4;
        uint64_t w[4];
        const uint64_t t = wave_sum(kept4(at(i0), i0, w));
        if (lane == 0) run_u[i] = t;
      }
      __syncthreads();
      const int m = min(64, per - run);
      const uint64_t v = lane < m ? run_u[lane] : 0, all = wave_sum(v);
      if (run + m >= per || acc + all > tgt) {
        run += find(v, tgt, m);
        break;
      }
      acc += all;
      run += m;
      __syncthreads();
    }
    if (wave != 0) return;
  }
  const int i0 = (piece * per + run) * 256 + lane * 4;
  uint64_t w[4];
  const f4u q = at(i0);
  const uint64_t l4 = kept4(q, i0, w);
  uint64_t x = acc + wave_scan(l4) - l4;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if (x <= tgt && x + w[c] > tgt) finish((float)q[c], i0 + c, S);
    x += w[c];
  }
}

}  // namespace

hipError_t launch_sample(const Plan& pl, const float* out, const vfm_sampling& sp, const float* u, int32_t* ids,
                         float* logprob, int max_out, hipStream_t s) {
  const SampleParams q = {sp.temperature, sp.top_k, sp.top_p, sp.min_p};
  const int pi = prof_begin(VFM_PROF_OTHER, s);
#define SAMPLE(NT_, W_) \
  hipLaunchKernelGGL((sample_kernel<NT_, W_>), dim3(pl.n_req), dim3(NT_), 0, s, pl, out, q, u, ids, logprob)
  if (sample_threads(max_out) == 256) SAMPLE(256, IN_REGS);
  else if (max_out <= 32768) SAMPLE(1024, IN_LDS);
  else SAMPLE(1024, IN_MEMORY);
#undef SAMPLE
  prof_end(pi, s);
  return hipGetLastError();
}
