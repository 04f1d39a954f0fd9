// Head outputs under penalties for repeated tokens, biases and masks, before a token is picked or drawn.
//
// A block takes a slice of one request's outputs.  It counts the request's earlier tokens that fall into the slice with
// LDS atomics (whole numbers, so their order cannot matter), enters the slice's biases, and passes over the slice once:
// in place it loads and stores only the 16 bytes around what changes.  Everything that a block needs of a request is loaded
// before LDS is cleared; its earlier tokens are read three loads ahead.  Every block of a request reads all of its
// earlier tokens, so slices are as large as LDS lets two blocks share a CU with, and blocks are numbered so that a request's
// run on one XCD, whose L2 serves all but the first.
//
// 256 requests of 32000 outputs after 200 to 4000 tokens, in place: 16.3 us, of which 6 are the launch and the chain plan ->
// lists -> LDS, 2 the counting and 8 the pass, which is bound by the lines it touches (a changed output costs a line read and
// written: with all counts left out the pass takes 4).  A list of what changes, gone through by all threads, gains nothing
// in place (14.7 for 14.9 without masks) and loses where it is long (26 for 21).  48 of 100003 after 5000 to 60000 tokens, to
// another place: 20.6 us, 5 of them the longest history's counting; slices of 8192 22.  One request: 4.2 us.
// The choice of slices looks at requests and rows alone, so where few requests have long histories many blocks count
// each of them: 100003 outputs after 60000 tokens take 20 us for 1 to 8 requests, 30 for 9 to 16 and 40 for 19 (98 blocks
// of 1024 each), 17.6 for 20 (13 of 8192); after 700 tokens 6 to 9 throughout.
#include <type_traits>

#include "decode_internal.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// The part of a list of n that [begin, begin + len) is
__device__ __forceinline__ int part(int64_t& begin, int64_t len, int64_t n) {
  if (begin < 0 || begin >= n || len <= 0) { begin = 0; return 0; }
  return (int)(len < n - begin ? len : n - begin);
}

constexpr uint32_t IN_PROMPT = 1u << 31;                  // the token was seen in the prompt

// What is known of an output: of the request's tokens, IN_PROMPT and how many were generated, and 1 + the place of its last
// bias.  One word holds both where the lists are short enough (15 bits and 16), which halves the LDS of a block and
// lets twice as many share a CU; with WIDE, one each.
constexpr int BIAS_AT = 16, BIAS_MOST = (1 << 15) - 1, COUNT_MOST = (1 << 16) - 1;

// The tokens p[0 .. n), taken by all threads of a block, 16 bytes a load where they are aligned, three loads ahead of their
// use; the first three are on their way while LDS is cleared.
template <int THREADS>
struct Tokens {
  const i32x4* quad;
  int quads;
  int32_t edge;                // of the thread: one before or behind the quads (3 and 3 at most), or none
  bool has_edge;
  i32x4 q[3];
  __device__ __forceinline__ Tokens(const int32_t* p, int n) {
    const int tid = threadIdx.x;
    const int head = min(n, (int)((4 - (((uintptr_t)p >> 2) & 3)) & 3));
    quads = (n - head) >> 2;
    quad = reinterpret_cast<const i32x4*>(p + head);
    const int at = tid < 4 ? tid : head + 4 * quads + tid - 4;
    has_edge = tid < 4 ? tid < head : tid < 8 && at < n;
    edge = has_edge ? p[at] : 0;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      q[k] = i32x4{};
      if (tid + k * THREADS < quads) q[k] = quad[tid + k * THREADS];
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) {
    if (has_edge) f(edge);
#pragma unroll 1
    for (int i = threadIdx.x; i < quads; i += THREADS) {
      i32x4 next = {};
      if (i + 3 * THREADS < quads) next = quad[i + 3 * THREADS];
#pragma unroll
      for (int e = 0; e < 4; ++e) f(q[0][e]);
      q[0] = q[1];
      q[1] = q[2];
      q[2] = next;
    }
  }
};

template <int SLICE, int THREADS>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(8, 8))) void adjust_kernel(
    Plan pl, const float* in, float* out, vfm_adjust a, int padded) {
  constexpr int WORDS = SLICE / 32 + 2;
  static_assert(WORDS <= THREADS, "a thread loads a word of the mask");
  __shared__ __attribute__((aligned(16))) uint32_t known[SLICE];
  __shared__ uint32_t allow[WORDS];
  const int r = blockIdx.x % padded, slice = blockIdx.x / padded;
  if (r >= pl.n_req) return;                              // block-uniform, as every exit below
  const int tid = threadIdx.x;
  const int base = pl.out_off[r], n = pl.out_off[r + 1] - base;
  // slices begin at multiples of 4 outputs of the whole batch, so that 4 neighbours are one aligned access
  if ((int64_t)slice * SLICE - (base & 3) >= n) return;
  const int lo = slice * SLICE - (base & 3);              // first output of the slice, of the request's (-3 .. -1: none there)
  const float rep_ = a.repetition ? a.repetition[r] : 1.f, pres_ = a.presence ? a.presence[r] : 0.f;
  const float freq_ = a.frequency ? a.frequency[r] : 0.f;
  int64_t hb = a.hist ? a.hist_begin[r] : 0, bb = a.bias ? a.bias_begin[r] : 0;
  const int hist_len = a.hist ? a.hist_len[r] : 0, bias_len = a.bias ? a.bias_len[r] : 0;
  int prompt = a.hist && a.n_prompt ? a.n_prompt[r] : 0;
  const int row = a.mask ? a.mask_row[r] : -1;
  const double rep = rep_ > 0.f ? (double)rep_ : 1.0;
  const double pres = pres_ == pres_ ? (double)pres_ : 0.0, freq = freq_ == freq_ ? (double)freq_ : 0.0;
  int hist = part(hb, hist_len, a.n_hist);
  if (rep == 1.0 && pres == 0.0 && freq == 0.0) hist = 0;
  prompt = min(max(prompt, 0), hist);
  const int biases = part(bb, bias_len, a.n_bias);
  const bool masked = row >= 0 && row < a.n_masks;
  const bool same = in == out;
  if (same && !hist && !biases && !masked) return;

  // the slice's words of the request's mask, bits past the request's outputs cleared
  const uint32_t* mask = masked ? a.mask + (int64_t)row * a.mask_words : nullptr;
  const int words = min(a.mask_words, (int)(((uint32_t)n + 31) >> 5)), w0 = max(lo, 0) >> 5;
  auto left = [&](int w) { return w < words ? mask[w] & (w == n >> 5 ? (1u << (n & 31)) - 1 : ~0u) : 0u; };
  uint32_t word = 0;
  if (masked && tid < WORDS) word = left(w0 + tid);
  const double inv = 1.0 / rep;
  bool none = false;                                      // the mask allows no output of the request

  // the outputs from `at` on, SLICE of them or with WIDE half as many
  auto pass = [&](auto wide, int at, bool first) {
    constexpr bool WIDE = decltype(wide)::value;
    constexpr int SIZE = WIDE ? SLICE / 2 : SLICE;
    uint32_t* const last = WIDE ? known + SIZE : known;
    const float* src = in + base + at;
    float* dst = out + base + at;
    const int skip = at < 0 ? -at : 0, past = min(n - at, SIZE);   // its outputs are places skip .. past - 1
    const uint32_t from = (uint32_t)(at + skip), span = (uint32_t)(past - skip);
    Tokens<THREADS> before(a.hist + hb, prompt), generated(a.hist + hb + prompt, hist - prompt);
    const int32_t bias0 = tid < biases ? a.bias_id[bb + tid] : -1;
#pragma unroll
    for (int g = 0; g < SLICE / (4 * THREADS); ++g) *reinterpret_cast<u32x4*>(known + 4 * (tid + g * THREADS)) = u32x4{};
    bool any = true;
    if (first && masked) {
      if (tid < WORDS) allow[tid] = word;
      any = __syncthreads_or(word != 0);
    } else {
      __syncthreads();
    }
    if (biases) {
      auto enter = [&](int i, int32_t id) {
        const uint32_t k = (uint32_t)id - from;
        if (k < span) atomicMax(&last[k + skip], (uint32_t)(i + 1) << (WIDE ? 0 : BIAS_AT));
      };
      if (tid < biases) enter(tid, bias0);
      for (int i = tid + THREADS; i < biases; i += THREADS) enter(i, a.bias_id[bb + i]);
      if (!WIDE) __syncthreads();
    }
    before.each([&](int32_t id) {
      const uint32_t k = (uint32_t)id - from;
      if (k < span) atomicOr(&known[k + skip], IN_PROMPT);
    });
    generated.each([&](int32_t id) {
      const uint32_t k = (uint32_t)id - from;
      if (k < span) atomicAdd(&known[k + skip], 1u);
    });
    if (!any) {                                           // none in the slice: is there one elsewhere?
      bool some = false;
      for (int w = tid; w < words; w += THREADS) some = some || left(w) != 0;
      none = !__syncthreads_or(some);
    } else {
      __syncthreads();
    }

#pragma unroll 4
    for (int i = 4 * tid; i < past; i += 4 * THREADS) {
      const u32x4 c = *reinterpret_cast<const u32x4*>(known + i);
      u32x4 b = {};
      if constexpr (WIDE) b = *reinterpret_cast<const u32x4*>(last + i);
      const uint32_t some = c[0] | c[1] | c[2] | c[3] | b[0] | b[1] | b[2] | b[3];
      uint32_t ok = 15;
      if (masked) {
        // bits of outputs at + i .. + 3, those before the request's first as if after it
        const int bit = at + i - 32 * w0, w = max(bit, 0) >> 5, s = bit - 32 * w;
        const uint64_t two = allow[w] | (uint64_t)allow[w + 1] << 32;
        ok = (uint32_t)(s < 0 ? two << -s : two >> s) & 15;
      }
      if (same && !some && ok == 15) continue;            // these 4 stay as they are
      const bool whole = i >= skip && i + 4 <= past;
      f32x4 v = {};
      if (ok) {                                           // of 4 that the mask forbids nothing is needed
        if (whole) v = *reinterpret_cast<const f32x4*>(src + i);
        else
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (i + e >= skip && i + e < past) v[e] = src[i + e];
      }
      if (some)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t bias = WIDE ? b[e] : (c[e] >> BIAS_AT) & BIAS_MOST;
          const uint32_t times = c[e] & (WIDE ? ~IN_PROMPT : (uint32_t)COUNT_MOST);
          if (!(c[e] | bias)) continue;
          double l = (double)v[e];
          if (times | (c[e] & IN_PROMPT)) l *= v[e] > 0.f ? inv : rep;
          if (times) l -= fma((double)times, freq, pres);
          if (bias) l += (double)a.bias[bb + bias - 1];
          v[e] = (float)l;
        }
      if (ok != 15)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = none ? NAN : (ok >> e & 1) ? v[e] : -INFINITY;
      if (whole) *reinterpret_cast<f32x4*>(dst + i) = v;
      else
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (i + e >= skip && i + e < past) dst[i + e] = v[e];
    }
  };
  if (hist <= COUNT_MOST && biases <= BIAS_MOST) {
    pass(std::false_type{}, lo, true);
  } else {
    pass(std::true_type{}, lo, true);
    if (n - lo > SLICE / 2) {
      __syncthreads();                                    // LDS is cleared anew
      pass(std::true_type{}, lo + SLICE / 2, false);
    }
  }
}

}  // namespace

hipError_t launch_adjust(const Plan& pl, const float* in, float* out, const vfm_adjust& a, int max_out, hipStream_t s) {
  const int padded = adjust_rows(pl.n_req), slice = adjust_slice(pl.n_req, max_out);
  const dim3 grid((unsigned)adjust_blocks(pl.n_req, max_out)), block(adjust_threads(slice));
#define ADJUST(S_, T_) hipLaunchKernelGGL((adjust_kernel<S_, T_>), grid, block, 0, s, pl, in, out, a, padded)
  if (slice == ADJUST_SMALL) ADJUST(ADJUST_SMALL, adjust_threads(ADJUST_SMALL));
  else if (slice == ADJUST_MIDDLE) ADJUST(ADJUST_MIDDLE, adjust_threads(ADJUST_MIDDLE));
  else ADJUST(ADJUST_LARGE, adjust_threads(ADJUST_LARGE));
#undef ADJUST
  return hipGetLastError();
}
