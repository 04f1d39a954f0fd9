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

  for (int i = 4 * tid; i < SLICE; i += 4 * THREADS) {
    *reinterpret_cast<u32x4*>(count + i) = u32x4{};
    if constexpr (BIAS) *reinterpret_cast<u32x4*>(last + i) = u32x4{};
  }
  __syncthreads();
  if (hist) {
    const int prompt = a.n_prompt ? a.n_prompt[r] : 0;
    each<THREADS>(a.hist + hb, hist, [&](int i, int32_t id) {
      const int64_t k = id - lo;
      if (id >= 0 && id < n && k >= 0 && k < SLICE) {
        if (i < prompt) atomicOr(&count[k], IN_PROMPT);
        else atomicAdd(&count[k], 1u);
      }
    });
  }
  if constexpr (BIAS)
    for (int i = tid; i < biases; i += THREADS) {
      const int32_t id = a.bias_id[bb + i];
      const int64_t k = id - lo;
      if (id >= 0 && id < n && k >= 0 && k < SLICE) atomicMax(&last[k], (uint32_t)i + 1);
    }
  const uint32_t* mask = masked ? a.mask + (int64_t)row * a.mask_words : nullptr;
  bool none = false;                                      // the mask allows no output of the request
  if (masked) {
    const int words = min(a.mask_words, (n + 31) >> 5);
    const uint32_t rest = (n & 31) ? (1u << (n & 31)) - 1 : ~0u;     // of word n / 32
    auto left = [&](int w) { return mask[w] & (w == n >> 5 ? rest : ~0u); };
    const int w0 = (int)(lo > 0 ? lo >> 5 : 0), w1 = (int)min((int64_t)words, (lo + SLICE + 31) >> 5);
    bool any = false;
    for (int w = w0 + tid; w < w1; w += THREADS) any = any || left(w) != 0;
    if (!__syncthreads_or(any)) {
      for (int w = tid; w < words; w += THREADS) any = any || left(w) != 0;
      none = !__syncthreads_or(any);
    }
  }
  __syncthreads();

  const float* src = in + base + lo;
  float* dst = out + base + lo;
  for (int i = 4 * tid; i < SLICE; i += 4 * THREADS) {
    const int64_t id = lo + i;                            // of the first of 4
    if (id >= n) break;
    const u32x4 c = *reinterpret_cast<const u32x4*>(count + i);
    u32x4 b = {};
    if constexpr (BIAS) b = *reinterpret_cast<const u32x4*>(last + i);
    uint32_t ok = 15;
    if (masked) {
      ok = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t w = (id + e) >> 5;
        if (id + e >= 0 && w < a.mask_words && id + e < n) ok |= ((mask[w] >> ((id + e) & 31)) & 1) << e;
      }
    }
    const bool whole = id >= 0 && id + 4 <= n;
    const uint32_t some = c[0] | c[1] | c[2] | c[3] | b[0] | b[1] | b[2] | b[3];
    if (same && !some && ok == 15) continue;
    f32x4 v = {};
    if (!(masked && ok == 0)) {
      if (whole) v = *reinterpret_cast<const f32x4*>(src + i);
      else
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (id + e >= 0 && id + e < n) v[e] = src[i + e];
    }
    if (some) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        double l = (double)v[e];
        if (c[e]) {
          l *= v[e] > 0.f ? inv : rep;
          const uint32_t times = c[e] & ~IN_PROMPT;
          if (times) l -= fma((double)times, freq, pres);
        }
        if constexpr (BIAS)
          if (b[e]) l += (double)a.bias[bb + b[e] - 1];
        if (c[e] | b[e]) v[e] = (float)l;
      }
    }
    if (masked) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = none ? NAN : (ok >> e & 1) ? v[e] : -INFINITY;
    }
    if (whole) *reinterpret_cast<f32x4*>(dst + i) = v;
    else
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (id + e >= 0 && id + e < n) dst[i + e] = v[e];
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
