// Next tokens drawn from the head outputs: temperature, top-k, top-p and min-p
// from one given uniform number per request (paper Section 4.2: token-based FMs
// served with long-lived decode iterations; the outputs are a task's LM head's).
//
// Weights.  w_j = 2^t_j, t_j = (l_j - M) log2(e) / T <= 0, in fp64 (at full rate
// here: 12 fused multiply-adds of a Taylor series after the split of t into
// its nearest integer and a rest of at most 1/2), rounded to 2^-44: the sums are
// then integers, exact in any order, so the order of atomics, the split over
// threads and the block's shape cannot change a result.  fp32 would shift the
// borders of the running sum by 1e-7 of it, and a vocabulary has so many of
// them that the token drawn would now and then be another.
//
// The three filters each keep a prefix of the outputs in descending order (ties
// by index), so only the last kept output has to be found, never a full order:
// outputs are counted (and their weights summed) in bins of equal width in l
// over the range where weights are not 0; the bin in which a filter ends is the
// only one that is put in order, and where all bins up to it hold few outputs
// (top-k), nothing else is looked at again.  One block per request: the row is
// read once where it fits the registers (up to 4096 outputs).
#include "decode_internal.h"

namespace {

typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));

struct SampleParams {
  const float* temperature; const int32_t* top_k; const float* top_p; const float* min_p;
};

// 2^t for t in [-46, 0], scaled by 2^sh and rounded to an integer.  Taylor series
// of e^(f ln 2) on |f| <= 1/2: the first term left out, (f ln 2)^12 / 12!, is
// below 7e-15.  Adding 2^52 leaves the integer in the low bits.
__device__ __forceinline__ uint64_t fixed_exp2(double t, int sh) {
  const double n = __builtin_rint(t), f = t - n;
  double p = 4.4455382718708101e-10;                  // ln2^11 / 11!
  p = fma(p, f, 7.0549116208011209e-09);               // ln2^10 / 10!
  p = fma(p, f, 1.0178086009239696e-07);
  p = fma(p, f, 1.3215486790144305e-06);
  p = fma(p, f, 1.5252733804059838e-05);
  p = fma(p, f, 1.5403530393381606e-04);
  p = fma(p, f, 1.3333558146428441e-03);
  p = fma(p, f, 9.6181291076284769e-03);
  p = fma(p, f, 5.5504108664821576e-02);
  p = fma(p, f, 2.4022650695910069e-01);
  p = fma(p, f, 6.9314718055994529e-01);
  p = fma(p, f, 1.0);
  const double d = __builtin_ldexp(p, (int)n + sh) + 4503599627370496.0;
  return (uint64_t)__double_as_longlong(d) & 0xFFFFFFFFFFFFFull;
}

// Integers in the order of the floats (no NaN); -0 and +0 are one.
__device__ __forceinline__ uint32_t float_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

__device__ __forceinline__ uint64_t shfl64(uint64_t v, int lane) { return __shfl((unsigned long long)v, lane, 64); }
// inclusive sums over the lanes of a wave
__device__ __forceinline__ uint64_t wave_scan(uint64_t v, int lane) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const uint64_t o = __shfl_up((unsigned long long)v, s, 64);
    if (lane >= s) v += o;
  }
  return v;
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v, int lane) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const uint32_t o = __shfl_up(v, s, 64);
    if (lane >= s) v += o;
  }
  return v;
}

// NT threads; R > 0: the row's outputs in R x 4 registers per thread (n <= NT R 4),
// R = 0: read again from memory (L2) by every pass.
template <int NT, int R>
__global__ __launch_bounds__(NT) void sample_kernel(Plan pl, const float* __restrict__ out, SampleParams sp,
                                                    const float* __restrict__ us, int32_t* __restrict__ ids,
                                                    float* __restrict__ logprob) {
  constexpr int NW = NT / 64, CAP = NT, NB = NT;
  __shared__ float red_f[2][NW];
  __shared__ uint64_t red_u[NW];
  __shared__ uint32_t red_c[NW];
  __shared__ int red_i[NW];
  __shared__ uint32_t h_cnt[NB];       // a bin's outputs, then the outputs up to and with it
  __shared__ uint64_t h_mass[NB];
  __shared__ uint64_t l_key[CAP];      // (float_key, ~index): descending order
  __shared__ uint64_t l_sorted[CAP], l_mass[CAP], l_cum[CAP];
  __shared__ uint32_t s_n, s_sel[3];   // list length; bin, outputs before it, outputs in it
  __shared__ uint64_t s_before, s_last, s_total;

  const int row = blockIdx.x;
  const int o0 = pl.out_off[row], n = pl.out_off[row + 1] - o0;
  const float* src = out + o0;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nr = (n + NT * 4 - 1) / (NT * 4);
  const int first = wave * nr * 256 + lane * 4;        // the wave's outputs are one run

  const float nan = __uint_as_float(0x7FC00000u);
  f4u reg[R > 0 ? R : 1];
  auto fetch = [&](int r) -> f4u {
    const int i = first + r * 256;
    f4u v = {nan, nan, nan, nan};
    if (i + 4 <= n) v = *reinterpret_cast<const f4u*>(src + i);
    else
#pragma unroll
      for (int c = 0; c < 4; ++c) if (i + c < n) v[c] = src[i + c];
    return v;
  };
  if constexpr (R > 0) {
#pragma unroll
    for (int r = 0; r < R; ++r) reg[r] = r < nr ? fetch(r) : f4u{nan, nan, nan, nan};
  }
  // f(value, index) for every output of the thread
  auto each = [&](auto&& f) {
    if constexpr (R > 0) {
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (r < nr) {
#pragma unroll
          for (int c = 0; c < 4; ++c) f((float)reg[r][c], first + r * 256 + c);
        }
    } else {
      for (int r = 0; r < nr; ++r) {
        const f4u v = fetch(r);
#pragma unroll
        for (int c = 0; c < 4; ++c) f((float)v[c], first + r * 256 + c);
      }
    }
  };

  // the largest output, and whether there is one
  float mx = -INFINITY;
  bool any = false;
  each([&](float v, int) { mx = fmaxf(mx, v); any = any || v == v; });
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) mx = fmaxf(mx, __shfl_xor(mx, s, 64));
  const bool any_w = __any(any);
  if (lane == 0) { red_f[0][wave] = mx; red_i[wave] = any_w; }
  __syncthreads();
  bool found = false;
  float M = -INFINITY;
#pragma unroll
  for (int i = 0; i < NW; ++i) { M = fmaxf(M, red_f[0][i]); found = found || red_i[i]; }
  if (!found) {                                          // block-uniform, as every branch on the row's values below
    if (tid == 0) { ids[row] = -1; if (logprob) logprob[row] = nan; }
    return;
  }
  const float temp = sp.temperature ? sp.temperature[row] : 1.f;
  const int tk = sp.top_k ? sp.top_k[row] : 0;
  const float tp = sp.top_p ? sp.top_p[row] : 1.f, mp = sp.min_p ? sp.min_p[row] : 0.f;
  if (!(temp > 0.f)) {                                   // greedy
    int best = INT32_MAX;
    each([&](float v, int i) { if (v == M) best = min(best, i); });
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) best = min(best, __shfl_xor(best, s, 64));
    __syncthreads();                                     // red_i is read above
    if (lane == 0) red_i[wave] = best;
    __syncthreads();
    if (tid == 0) {
      for (int i = 1; i < NW; ++i) best = min(best, red_i[i]);
      ids[row] = best;
      if (logprob) logprob[row] = 0.f;
    }
    return;
  }
  const double T = fmin(fmax((double)temp, 1e-30), 1e30);
  const double c2 = 1.4426950408889634 / T;
  const int sh = n < (1 << 19) ? 44 : 32;
  const uint64_t one = (uint64_t)1 << sh;
  const float cut = fminf((float)(31.2 * T), 3e38f);     // 45 ln 2: below M - cut every weight is 0
  auto mass = [&](float v) -> uint64_t {
    if (v == M) return one;
    const double t = ((double)v - (double)M) * c2;
    return t >= -45.0 ? fixed_exp2(t, sh) : 0;           // NaN: 0
  };
  const double uu = us[row] > 0.f ? (double)us[row] : 0.0;   // NaN: 0
  auto finish = [&](float v, int i, uint64_t total) {    // one thread: the drawn output
    ids[row] = i;
    if (logprob) {
      const double lw = v == M ? 0.0 : ((double)v - (double)M) / T;
      logprob[row] = (float)(lw - log((double)total) + (double)sh * 0.6931471805599453);
    }
  };
  // 0: off.  No weight reaches a min-p above 1: the first output alone stays
  const int k = mp > 1.f && n > 1 ? 1 : tk > 0 && tk < n ? tk : 0;
  const bool p_on = tp < 1.f;
  const double p = (double)tp;

  // block-wide inclusive scan of the bins in place: h_cnt and, with `masses`, h_mass
  auto scan_bins = [&](bool masses) {
    const uint32_t cw = wave_scan(h_cnt[tid], lane);
    uint64_t mw = 0;
    if (masses) mw = wave_scan(h_mass[tid], lane);
    if (lane == 63) { red_c[wave] = cw; red_u[wave] = mw; }
    __syncthreads();
    uint32_t cb = 0;
    uint64_t mb = 0;
    for (int i = 0; i < wave; ++i) { cb += red_c[i]; mb += red_u[i]; }
    h_cnt[tid] = cw + cb;
    if (masses) h_mass[tid] = mw + mb;
    __syncthreads();
  };

  float v_last = -INFINITY;                              // the last kept output: its value and index
  int i_last = INT32_MAX;
  if (k > 0 || p_on) {
    // range of the bins: the outputs whose weights are not 0
    float mn = M;
    each([&](float v, int) { if (M - v <= cut) mn = fminf(mn, v); });
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) mn = fminf(mn, __shfl_xor(mn, s, 64));
    if (lane == 0) red_f[1][wave] = mn;
    h_cnt[tid] = 0;
    h_mass[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) mn = fminf(mn, red_f[1][i]);
    const float cb = M - mn > 0.f ? (float)NB / (M - mn) : 0.f;
    auto bin0 = [&](float v) -> int {                    // -1: weight 0 or NaN
      if (v == M) return 0;
      const float d = M - v;
      return d <= cut ? (int)fminf(d * cb, (float)(NB - 1)) : -1;
    };
    // count outputs per bin, with their weights where a share of them is wanted.
    // A small top-k first counts only: it needs the weights of few outputs
    const bool small_k = k > 0 && k <= CAP / 2;
    bool masses = p_on && !small_k;
    auto fill = [&]() {
      each([&](float v, int) {
        const int b = bin0(v);
        if (b >= 0) {
          atomicAdd(&h_cnt[b], 1u);
          if (masses) atomicAdd((unsigned long long*)&h_mass[b], (unsigned long long)mass(v));
        }
      });
      __syncthreads();
      scan_bins(masses);
    };
    fill();
    // the bin in which the j-th output (j > 0) or the weight `target` lies; `c0`, `m0`: what lies before the bins
    auto select = [&](uint32_t j, double target, uint32_t c0, uint64_t m0) {
      const uint32_t ce = tid ? h_cnt[tid - 1] : 0, ci = h_cnt[tid];
      bool hit;
      if (j > 0) hit = c0 + ce < j && c0 + ci >= j;
      else {
        const uint64_t me = m0 + (tid ? h_mass[tid - 1] : 0), mi = m0 + h_mass[tid];
        hit = ci > ce && (double)mi >= target && ((double)me < target || c0 + ce == 0);
      }
      if (hit) {
        s_sel[0] = tid; s_sel[1] = c0 + ce; s_sel[2] = ci - ce;
        s_before = m0 + (tid && masses ? h_mass[tid - 1] : 0);
      }
      __syncthreads();
    };
    // the outputs that f(value) picks (at most CAP), in descending order in l_sorted, their weights
    // in l_mass and running sums (without what lies before) in l_cum
    auto list = [&](uint32_t cnt, auto&& f) {
      if (tid == 0) s_n = 0;
      __syncthreads();
      each([&](float v, int i) {
        if (f(v)) {
          const uint32_t at = atomicAdd(&s_n, 1u);
          if (at < CAP) l_key[at] = ((uint64_t)float_key(v) << 32) | (uint32_t)~i;
        }
      });
      __syncthreads();
      const uint64_t mine = tid < cnt ? l_key[tid] : 0;
      uint32_t rank = 0;
      for (uint32_t j = 0; j < cnt; ++j) rank += l_key[j] > mine;
      if (tid < cnt) l_sorted[rank] = mine;
      __syncthreads();
      uint64_t w = 0;
      if (tid < cnt) {
        const uint32_t key = (uint32_t)(l_sorted[tid] >> 32);
        w = mass(__uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu)));
      }
      const uint64_t cw = wave_scan(w, lane);
      if (lane == 63) red_u[wave] = cw;
      __syncthreads();
      uint64_t before = 0;
      for (int i = 0; i < wave; ++i) before += red_u[i];
      if (tid < CAP) { l_mass[tid] = w; l_cum[tid] = cw + before; }
      __syncthreads();
    };
    auto value_of = [&](uint64_t e) {
      const uint32_t key = (uint32_t)(e >> 32);
      return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu));
    };

    uint32_t kk = k > 0 && (uint32_t)k < h_cnt[NB - 1] ? (uint32_t)k : 0;   // outputs of weight 0 do not count
    if (kk == 0 && k > 0 && p_on && !masses) {
      __syncthreads();
      h_cnt[tid] = 0;
      masses = true;
      __syncthreads();
      fill();
    }
    // where all outputs up to the filter's last bin fit the list, the list is all that is needed
    bool listed = false;
    uint64_t total = 0;                                  // weight that top_p takes its share of
    if (kk > 0 || p_on) {
      if (kk == 0) total = h_mass[NB - 1];
      select(kk, p * (double)total, 0, 0);
      const uint32_t bin = s_sel[0], upto = s_sel[1] + s_sel[2];
      listed = upto <= CAP;
      if (listed) {
        list(upto, [&](float v) { const int b = bin0(v); return b >= 0 && (uint32_t)b <= bin; });
        const uint32_t nk = kk > 0 ? kk : upto;
        if (kk > 0) total = l_cum[kk - 1];
        const double target = p_on ? p * (double)total : INFINITY, least = mp > 0.f ? (double)mp * (double)one : 0.0;
        auto keep = [&](uint32_t r) {
          return r == 0 || (r < nk && (double)l_cum[r - 1] < target && (double)l_mass[r] >= least);
        };
        const bool mine = (uint32_t)tid < nk && keep(tid);
        if (mine && !((uint32_t)tid + 1 < nk && keep(tid + 1))) { s_n = tid + 1; s_total = l_cum[tid]; }
        __syncthreads();
        const uint32_t kept = s_n;
        const uint64_t S = s_total;
        const uint64_t tgt = min((uint64_t)fmin(uu * (double)S, 9.2e18), S - 1);
        if (mine) {
          const uint64_t me = l_sorted[tid];
          uint64_t c = 0;                                // kept weight up to this output, by index
          for (uint32_t j = 0; j < kept; ++j) c += (uint32_t)l_sorted[j] >= (uint32_t)me ? l_mass[j] : 0;
          if (c > tgt && c - l_mass[tid] <= tgt) finish(value_of(me), (int)~(uint32_t)me, S);
        }
        return;
      }
    }
    // else: the last output of each filter, then a pass over everything kept
    if (kk > 0 && p_on && !masses) {
      __syncthreads();
      h_cnt[tid] = 0;
      masses = true;
      __syncthreads();
      fill();
    }
    auto resolve = [&](uint32_t j, double target) {      // -> v_last, i_last, s_last (weight up to and with it)
      select(j, target, 0, 0);
      const int bin = (int)s_sel[0];
      uint32_t before = s_sel[1], cnt = s_sel[2];
      uint64_t m0 = s_before;
      // the bin's outputs as a range of keys, cut down while they are too many for the list
      uint32_t lo = 0, hi = 0;
      bool keys = false;
      while (cnt > CAP) {
        uint32_t a = 0xFFFFFFFFu, z = 0;
        each([&](float v, int) {
          if (!(v == v)) return;
          const uint32_t q = float_key(v);
          if (keys ? q >= lo && q <= hi : bin0(v) == bin) { a = min(a, q); z = max(z, q); }
        });
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) { a = min(a, (uint32_t)__shfl_xor(a, s, 64)); z = max(z, (uint32_t)__shfl_xor(z, s, 64)); }
        __syncthreads();
        if (lane == 0) { red_c[wave] = a; red_i[wave] = (int)z; }
        __syncthreads();
        for (int i = 0; i < NW; ++i) { a = min(a, red_c[i]); z = max(z, (uint32_t)red_i[i]); }
        lo = a; hi = z; keys = true;
        if (lo == hi) break;                             // all equal: by index alone
        const int shift = max(0, 32 - __builtin_clz(hi - lo) - (NB == 1024 ? 10 : 8));
        __syncthreads();
        h_cnt[tid] = 0;
        h_mass[tid] = 0;
        __syncthreads();
        each([&](float v, int) {
          if (!(v == v)) return;
          const uint32_t q = float_key(v);
          if (q >= lo && q <= hi) {
            const uint32_t b = (hi - q) >> shift;
            atomicAdd(&h_cnt[b], 1u);
            if (masses) atomicAdd((unsigned long long*)&h_mass[b], (unsigned long long)mass(v));
          }
        });
        __syncthreads();
        scan_bins(masses);
        select(j, target, before, m0);
        const uint32_t b = s_sel[0];
        before = s_sel[1]; cnt = s_sel[2]; m0 = s_before;
        const uint64_t top = (uint64_t)hi - ((uint64_t)b << shift);
        hi = (uint32_t)top;
        const uint64_t below = ((uint64_t)1 << shift) - 1;
        lo = top - lo > below ? (uint32_t)(top - below) : lo;
      }
      if (keys && lo == hi && cnt > CAP) {               // the x-th of equal outputs, by index
        const float v = __uint_as_float(lo ^ ((lo >> 31) ? 0x80000000u : 0xFFFFFFFFu));
        const uint64_t w = mass(v);
        uint32_t want;
        if (j > 0) want = j - before;
        else {
          const double need = (target - (double)m0) / (double)(w ? w : 1);
          want = need <= 1.0 ? 1u : need >= (double)cnt ? cnt : (uint32_t)ceil(need);
        }
        uint32_t mine = 0;
        each([&](float q, int) { mine += q == v; });
        uint32_t ws = mine;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) ws += __shfl_xor(ws, s, 64);
        __syncthreads();
        if (lane == 0) red_c[wave] = ws;
        __syncthreads();
        uint32_t skip = 0;
        int at = 0;
        while (at < NW - 1 && skip + red_c[at] < want) skip += red_c[at++];
        if (wave == at) {                                // runs of 256 outputs, 4 per lane, in index order
          bool done = false;
          auto step = [&](const f4u& q, int i0) {
            uint32_t c4 = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) c4 += q[c] == v;
            const uint32_t inc = wave_scan(c4, lane), tot = __shfl(inc, 63, 64);
            if (!done && skip + tot >= want) {
              uint32_t s = skip + inc - c4;
#pragma unroll
              for (int c = 0; c < 4; ++c)
                if (q[c] == v && ++s == want) s_sel[0] = (uint32_t)(i0 + c);
              done = true;
            }
            skip += tot;
          };
          if constexpr (R > 0) {
#pragma unroll
            for (int r = 0; r < R; ++r) if (r < nr) step(reg[r], first + r * 256);
          } else {
            for (int r = 0; r < nr; ++r) step(fetch(r), first + r * 256);
          }
        }
        __syncthreads();
        v_last = v;
        i_last = (int)s_sel[0];
        if (tid == 0) s_last = m0 + (uint64_t)want * w;
        __syncthreads();
        return;
      }
      list(cnt, [&](float v) {
        if (!(v == v)) return false;
        const uint32_t q = float_key(v);
        return keys ? q >= lo && q <= hi : bin0(v) == bin;
      });
      if ((uint32_t)tid < cnt) {
        const uint64_t me = m0 + l_cum[tid] - l_mass[tid], mi = m0 + l_cum[tid];
        const bool hit = j > 0 ? before + tid + 1 == j
                               : ((double)mi >= target || (uint32_t)tid + 1 == cnt) && ((double)me < target || before + tid == 0);
        if (hit) { s_sel[0] = tid; s_last = mi; }
      }
      __syncthreads();
      const uint64_t e = l_sorted[s_sel[0]];
      v_last = value_of(e);
      i_last = (int)~(uint32_t)e;
      __syncthreads();
    };
    if (kk > 0) {
      resolve(kk, 0.0);
      total = s_last;
    }
    if (p_on) {
      if (kk > 0) {                                      // the bins may have been cut down: fill them again
        __syncthreads();
        h_cnt[tid] = 0;
        h_mass[tid] = 0;
        __syncthreads();
        fill();
      }
      const float vk = v_last;
      const int ik = i_last;
      resolve(0, p * (double)total);
      if (kk > 0 && (v_last < vk || (v_last == vk && i_last > ik))) { v_last = vk; i_last = ik; }
    }
  }

  // a pass over the kept outputs: their sum, then the one at u times it
  const double least = mp > 0.f ? fmin((double)mp, 1.0) * (double)one : 0.0;
  float v_least = v_last;
  if (mp > 0.f) v_least = fmaxf(v_least, (float)((double)M + T * log(fmin((double)mp, 1.0)) * 1.0001 - 1e-5 * fabs((double)M)));
  auto kept_mass = [&](float v, int i) -> uint64_t {
    if (!(v >= v_least) || (v == v_last && i > i_last)) return 0;
    const uint64_t w = mass(v);
    return (double)w >= least ? w : 0;
  };
  __syncthreads();                                       // red_u has been read
  uint64_t sum = 0;
  each([&](float v, int i) { sum += kept_mass(v, i); });
  uint64_t ws = sum;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) ws += __shfl_xor((unsigned long long)ws, s, 64);
  if (lane == 0) red_u[wave] = ws;
  __syncthreads();
  uint64_t S = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) S += red_u[i];
  const uint64_t tgt = min((uint64_t)fmin(uu * (double)S, 9.2e18), S - 1);
  uint64_t acc = 0;
  int at = 0;
  while (at < NW - 1 && acc + red_u[at] <= tgt) acc += red_u[at++];
  if (wave != at) return;
  // the wave whose run holds it: 256 outputs at a time
  bool done = false;
  auto step = [&](const f4u& q, int i0) {
    if (done) return;
    uint64_t w[4], l4 = 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) { w[c] = kept_mass((float)q[c], i0 + c); l4 += w[c]; }
    const uint64_t inc = wave_scan(l4, lane), tot = shfl64(inc, 63);
    if (acc + tot > tgt) {
      uint64_t s = acc + inc - l4;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if (s <= tgt && s + w[c] > tgt) finish((float)q[c], i0 + c, S);
        s += w[c];
      }
      done = true;
    }
    acc += tot;
  };
  if constexpr (R > 0) {
#pragma unroll
    for (int r = 0; r < R; ++r) if (r < nr) step(reg[r], first + r * 256);
  } else {
    for (int r = 0; r < nr && !done; ++r) step(fetch(r), first + r * 256);
  }
}

}  // namespace

hipError_t launch_sample(const Plan& pl, const float* out, const vfm_sampling& sp, const float* u, int32_t* ids,
                         float* logprob, int max_out, hipStream_t s) {
  const SampleParams q = {sp.temperature, sp.top_k, sp.top_p, sp.min_p};
  const int pi = prof_begin(VFM_PROF_OTHER, s);
#define SAMPLE(NT_, R_) \
  hipLaunchKernelGGL((sample_kernel<NT_, R_>), dim3(pl.n_req), dim3(NT_), 0, s, pl, out, q, u, ids, logprob)
  if (max_out <= 1024) SAMPLE(256, 1);
  else if (max_out <= 4096) SAMPLE(256, 4);
  else SAMPLE(1024, 0);
#undef SAMPLE
  prof_end(pi, s);
  return hipGetLastError();
}
