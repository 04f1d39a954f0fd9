// Head outputs under penalties for repeated tokens, biases and masks, before a token is picked or drawn.
//
// A block takes a slice of one request's outputs.  It counts the request's earlier tokens that fall into the slice with
// LDS atomics (whole numbers, so their order cannot matter), enters the slice's biases, and passes over the slice once:
// in place it loads and stores only what changes.  Bound by its bytes, and for a request alone by latency: the chain plan
// -> list -> LDS -> outputs.  Every block of a request reads all of its earlier tokens: blocks are numbered so
// that a request's blocks run on one XCD, whose L2 serves all but the first.
#include "decode_internal.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t IN_PROMPT = 1u << 31;                  // of a count: the token was seen in the prompt

// `f(i, v)` for the n ints from p on, 16 bytes a load where they are aligned
template <int THREADS, typename F>
__device__ __forceinline__ void each(const int32_t* __restrict__ p, int n, F f) {
  const int tid = threadIdx.x;
  const int head = min(n, (int)((4 - (((uintptr_t)p >> 2) & 3)) & 3));
  const int quads = (n - head) >> 2, tail = head + 4 * quads;
  if (tid < head) f(tid, p[tid]);
  if (tid < n - tail) f(tail + tid, p[tail + tid]);
  const i32x4* q = reinterpret_cast<const i32x4*>(p + head);
  int i = tid;
  for (; i + 3 * THREADS < quads; i += 4 * THREADS) {
    i32x4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = q[i + k * THREADS];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) f(head + 4 * (i + k * THREADS) + e, v[k][e]);
  }
  for (; i < quads; i += THREADS) {
    const i32x4 v = q[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) f(head + 4 * i + e, v[e]);
  }
}

// The part of a list of n that [begin, begin + len) is
__device__ __forceinline__ int part(int64_t& begin, int64_t len, int64_t n) {
  if (begin < 0 || begin >= n || len <= 0) { begin = 0; return 0; }
  return (int)(len < n - begin ? len : n - begin);
}

template <int SLICE, int THREADS, bool BIAS>
__global__ __launch_bounds__(THREADS) void adjust_kernel(Plan pl, const float* in, float* out, vfm_adjust a, int padded) {
  __shared__ __attribute__((aligned(16))) uint32_t count[SLICE];   // generated so many times, IN_PROMPT
  __shared__ __attribute__((aligned(16))) uint32_t last[BIAS ? SLICE : 4];   // 1 + place of its last bias
  constexpr int G = SLICE / (4 * THREADS);                // groups of 4 outputs of a thread
  constexpr int WORDS = SLICE / 32 + 2;
  __shared__ uint32_t allow[WORDS];
  const int r = blockIdx.x % padded, slice = blockIdx.x / padded;
  if (r >= pl.n_req) return;                              // block-uniform, as every exit below
  const int tid = threadIdx.x;
  const int base = pl.out_off[r], n = pl.out_off[r + 1] - base;
  // slices begin at multiples of 4 outputs of the whole batch, so that 4 neighbours are one aligned access
  const int64_t lo = (int64_t)slice * SLICE - (base & 3); // first output of the slice, of the request's
  if (lo >= n) return;
  const float rep_ = a.repetition ? a.repetition[r] : 1.f, pres_ = a.presence ? a.presence[r] : 0.f;
  const float freq_ = a.frequency ? a.frequency[r] : 0.f;
  const double rep = rep_ > 0.f ? (double)rep_ : 1.0, inv = 1.0 / rep;
  const double pres = pres_ == pres_ ? (double)pres_ : 0.0, freq = freq_ == freq_ ? (double)freq_ : 0.0;
  int64_t hb = a.hist ? a.hist_begin[r] : 0, bb = BIAS ? a.bias_begin[r] : 0;
  int hist = a.hist ? part(hb, a.hist_len[r], a.n_hist) : 0;
  if (rep == 1.0 && pres == 0.0 && freq == 0.0) hist = 0;
  const int biases = BIAS ? part(bb, a.bias_len[r], a.n_bias) : 0;
  const int row = a.mask ? a.mask_row[r] : -1;
  const bool masked = row >= 0 && row < a.n_masks;
  const bool same = in == out;
  if (same && !hist && !biases && !masked) return;

  const float* src = in + base + lo;
  f32x4 v[G];
  auto fetch = [&](int g) {
    const int i = 4 * (tid + g * THREADS);
    const int64_t id = lo + i;
    if (id >= 0 && id + 4 <= n) v[g] = *reinterpret_cast<const f32x4*>(src + i);
    else
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (id + e >= 0 && id + e < n) v[g][e] = src[i + e];
  };
#pragma unroll
  for (int g = 0; g < G; ++g) {
    v[g] = f32x4{};
    if (!same) fetch(g);                                  // all of them, on their way while the tokens are counted
  }

  for (int i = 4 * tid; i < SLICE; i += 4 * THREADS) {
    *reinterpret_cast<u32x4*>(count + i) = u32x4{};
    if constexpr (BIAS) *reinterpret_cast<u32x4*>(last + i) = u32x4{};
  }
  // the request's outputs of the slice: span of them from output `from`, which is place `skip` of it
  const uint32_t from = lo > 0 ? (uint32_t)lo : 0u, skip = (uint32_t)(from - lo);
  const uint32_t span = (uint32_t)min((int64_t)n - from, (int64_t)SLICE - skip);
  __syncthreads();
  if (hist) {
    const int prompt = a.n_prompt ? a.n_prompt[r] : 0;
    each<THREADS>(a.hist + hb, hist, [&](int i, int32_t id) {
      const uint32_t k = (uint32_t)id - from;
      if (k < span) {
        if (i < prompt) atomicOr(&count[k + skip], IN_PROMPT);
        else atomicAdd(&count[k + skip], 1u);
      }
    });
  }
  if constexpr (BIAS)
    for (int i = tid; i < biases; i += THREADS) {
      const uint32_t k = (uint32_t)a.bias_id[bb + i] - from;
      if (k < span) atomicMax(&last[k + skip], (uint32_t)i + 1);
    }
  // the slice's words of the request's mask, bits past the request's outputs cleared
  const int first = lo > 0 ? (int)lo : 0, w0 = first >> 5;
  bool none = false;                                      // the mask allows no output of the request
  if (masked) {
    const uint32_t* mask = a.mask + (int64_t)row * a.mask_words;
    const int words = min(a.mask_words, (n + 31) >> 5);
    const uint32_t rest = (n & 31) ? (1u << (n & 31)) - 1 : ~0u;     // of word n / 32
    auto left = [&](int w) { return w < words ? mask[w] & (w == n >> 5 ? rest : ~0u) : 0u; };
    bool any = false;
    for (int w = tid; w < WORDS; w += THREADS) any = (allow[w] = left(w0 + w)) != 0 || any;
    if (!__syncthreads_or(any)) {
      for (int w = tid; w < words; w += THREADS) any = any || left(w) != 0;
      none = !__syncthreads_or(any);
    }
  }
  __syncthreads();

  float* dst = out + base + lo;
  u32x4 c[G], b[G];
  uint32_t ok[G];
  bool load[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int i = 4 * (tid + g * THREADS);
    c[g] = *reinterpret_cast<const u32x4*>(count + i);
    b[g] = u32x4{};
    if constexpr (BIAS) b[g] = *reinterpret_cast<const u32x4*>(last + i);
    ok[g] = 15;
    if (masked) {
      // bits of outputs lo + i .. + 3, those before the request's first as if after it
      const int64_t bit = lo + i - 32 * w0;
      const int w = bit < 0 ? 0 : (int)(bit >> 5), at = (int)(bit - 32 * w);
      const uint64_t two = allow[w] | (uint64_t)allow[w + 1] << 32;
      ok[g] = (uint32_t)(at < 0 ? two << -at : two >> at) & 15;
    }
  }
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int i = 4 * (tid + g * THREADS);
    const bool some = (c[g][0] | c[g][1] | c[g][2] | c[g][3] | b[g][0] | b[g][1] | b[g][2] | b[g][3]) != 0;
    load[g] = lo + i < n && (!same || some || ok[g] != 15);       // otherwise these 4 stay as they are
    if (same && load[g]) fetch(g);
  }
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int i = 4 * (tid + g * THREADS);
    if (!load[g]) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      double l = (double)v[g][e];
      if (c[g][e]) {
        l *= v[g][e] > 0.f ? inv : rep;
        const uint32_t times = c[g][e] & ~IN_PROMPT;
        if (times) l -= fma((double)times, freq, pres);
      }
      if constexpr (BIAS)
        if (b[g][e]) l += (double)a.bias[bb + b[g][e] - 1];
      if (c[g][e] | b[g][e]) v[g][e] = (float)l;
      if (masked) v[g][e] = none ? NAN : (ok[g] >> e & 1) ? v[g][e] : -INFINITY;
    }
    const int64_t id = lo + i;
    if (id >= 0 && id + 4 <= n) *reinterpret_cast<f32x4*>(dst + i) = v[g];
    else
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (id + e >= 0 && id + e < n) dst[i + e] = v[g][e];
  }
}

}  // namespace

hipError_t launch_adjust(const Plan& pl, const float* in, float* out, const vfm_adjust& a, int max_out, hipStream_t s) {
  const int padded = adjust_rows(pl.n_req), small = adjust_small(pl.n_req, max_out);
  const dim3 grid((unsigned)adjust_blocks(pl.n_req, max_out)), block(small ? ADJUST_SMALL_THREADS : ADJUST_THREADS);
#define ADJUST(S_, T_, B_) hipLaunchKernelGGL((adjust_kernel<S_, T_, B_>), grid, block, 0, s, pl, in, out, a, padded)
  if (small) { if (a.bias) ADJUST(ADJUST_SMALL, ADJUST_SMALL_THREADS, true); else ADJUST(ADJUST_SMALL, ADJUST_SMALL_THREADS, false); }
  else { if (a.bias) ADJUST(ADJUST_SLICE, ADJUST_THREADS, true); else ADJUST(ADJUST_SLICE, ADJUST_THREADS, false); }
#undef ADJUST
  return hipGetLastError();
}
