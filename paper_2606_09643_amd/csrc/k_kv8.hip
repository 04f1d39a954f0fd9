// A paged KV cache held in 8 bits: appending rotated keys and values to it, and attention of new rows over it.
//
// K and V are e4m3 codes; the 16 positions of a run (an aligned 16 of a page) share one scale per key head, a power of two
// 2^(e - 127) whose exponent byte e lies beside the other pool's: exps[run][key head][K, V].  A power of two, because a run
// fills up over several steps: when a later row needs a larger scale, the codes that are there move by their exponents
// and keep their mantissas (all but those that become subnormal), where a scale of any size would round them anew.
// It also is what gfx950's conversions multiply by for nothing: v_cvt_scalef32_pk_{bf16,f32}_fp8 give code 2^(e - 127)
// exactly, as e4m3 has 4 significant bits and bf16 8.
#include <type_traits>

#include "paged_device.h"

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// what the scale's exponent byte stands for, as the conversions take it (they look at the exponent field alone)
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e << 23); }

// 8 codes times their scale
__device__ __forceinline__ bf16x8 decode8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  const bf16x4 l = __builtin_shufflevector(a, b, 0, 1, 2, 3), h = __builtin_shufflevector(c, d, 0, 1, 2, 3);
  return __builtin_shufflevector(l, h, 0, 1, 2, 3, 4, 5, 6, 7);
}
// 4 codes times their scale
__device__ __forceinline__ f32x4 decode4(uint32_t w, float scale) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
  return f32x4{a[0], a[1], b[0], b[1]};
}
// 4 values of at most 448 as codes, ties to even
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// ---------------------------------------------------------------------------
// Append.  A block takes a run of new rows (those of one request in one aligned 16 positions) and some of its heads: the
// launch's first blocks each request's first run, the others the further runs that begin in 16 rows of the batch.  A wave
// takes a head of the whole run, so the run's largest magnitude is found by lane exchanges and the codes are written from
// the registers that hold the rotated values.  A single row (decode) leaves most of such a wave idle: there it takes
// 64 / (DH / 16) heads at once; with head dim 128 up to 8 rows are half a run's work (200 requests of 2 to 4 rows: 28 us,
// 38 as whole runs).
//
// Rotation in fp64, of operands that fp64 holds exactly: a code is one rounding of the rotated value, and scale and code
// do not depend on how the angle's last bits came out.  The value goes through fp32 rounded to odd (cut, the last
// bit set if anything was lost), after which rounding to 4 or 8 bits is as if from the fp64 value, and a comparison with a
// number of few bits comes out the same.  Below 2^-126 fp32 has fewer bits and rounds that to the nearest: bf16 queries
// stay so (off by up to 2^-149 before their own rounding: 2^-150 cut, 2^-150 rounded); a code feels it where the run's
// scale is among the smallest 11, and such a head is taken again with the last bit put where fp32 has it, behind the
// others and out of their way (40 requests of 40 to 60 rows: 22.1 us, 21.7 without, 22.6 with the queries' smallest
// magnitude looked at too).
//
// Bound by its bytes: 32 prompts of 128 to 1024 tokens, 32 heads of 128 on 32, take 162 us, 4.8 TB/s (a copy of 2 GiB runs
// at 4.95).  The blocks that share a run's heads are neighbours in the launch, so its rows are read at once: 191 us with
// them far apart.  4 heads a wave; 6 take 164, 12 190 (a long last round), and loading a head ahead 205 for 191 (3
// waves on a SIMD in place of 4).  One row: 4.4 us, all latency.  A block per row, most of which find no run, took 42 us for 40
// requests of 40 to 60 rows, 22 now, and a block for all runs of 16 rows 100 for 3000 single rows, 31 now.
// ---------------------------------------------------------------------------
constexpr float TOP8 = 3.19014718988379809e38f;          // 1.875 2^127: larger magnitudes would round to 2^128

template <bool TINY>
__device__ __forceinline__ float to_odd(double d) {
  if (TINY && fabs(d) < 0x1p-126) {                       // fp32 counts in 2^-149 there, whatever the value's own bits
    const double n = fabs(d) * 0x1p149;
    const uint32_t w = (uint32_t)n;
    return copysignf(__uint_as_float(w | ((double)w != n ? 1 : 0)), (float)d);
  }
  u32x2 w;
  __builtin_memcpy(&w, &d, 8);
  w[0] = (w[0] & 0xE0000000u) | ((w[0] & 0x1FFFFFFFu) ? 0x20000000u : 0u);
  double r;
  __builtin_memcpy(&r, &w, 8);
  return (float)r;
}
__device__ __forceinline__ bool finite(double d) { return (__double2hiint(d) & 0x7FF00000) != 0x7FF00000; }

template <typename T> struct Half8;                       // 8 elements of a row
template <> struct Half8<bf16> {
  bf16x8 v;
  __device__ __forceinline__ float get(int i) const { return (float)v[i]; }
  __device__ __forceinline__ void put(int i, float f) { v[i] = (bf16)f; }
};
template <> struct Half8<float> {
  f32x4 v[2];
  __device__ __forceinline__ float get(int i) const { return v[i >> 2][i & 3]; }
  __device__ __forceinline__ void put(int i, float f) { v[i >> 2][i & 3] = f; }
};

struct Append8 {
  int H, KH, rotate, split;          // blocks that share the heads of a run
  double log2_theta;
  int64_t ld, ldq, slots;
  uint8_t *k, *v, *exps;
  KvPages kp;
};

// How a wave holds rows of a run's head(s), a lane pairs (i, i + DH/2) of 8 of the dims: one head of up to ROWS rows, or
// with ROWS = 1 a single row of 64 / PER heads.
template <typename T, int DH, int ROWS>
struct Held {
  static constexpr int HALF = DH / 2, PER = HALF / 8;     // lanes of a row
  static constexpr bool ONE = ROWS == 1;
  static constexpr int RPP = ONE ? 1 : 64 / PER;          // rows at a time
  static constexpr int NI = ONE ? 1 : ROWS / RPP;
  Half8<T> x[NI], y[NI];
  __device__ __forceinline__ static int head_of(int unit) {
    return ONE ? unit * (64 / PER) + (int)(threadIdx.x & 63) / PER : unit;
  }
  __device__ __forceinline__ static int row0() { return ONE ? 0 : (int)(threadIdx.x & 63) / PER; }
  __device__ __forceinline__ void load(const T* qkv, int64_t ld, int n_heads, int unit, int r0, int nr) {
    const int head = min(head_of(unit), n_heads - 1), ch = (threadIdx.x & 63) % PER;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int r = min(row0() + i * RPP, nr - 1);        // rows past the last: copies of it
      const T* p = qkv + (int64_t)(r0 + r) * ld + (int64_t)head * DH + ch * 8;
      x[i] = *reinterpret_cast<const Half8<T>*>(p);
      y[i] = *reinterpret_cast<const Half8<T>*>(p + HALF);
    }
  }
};

// The run's nr rows from row r0 at position pos0, slot slot0.  Without TINY, where keys below 2^-126 could have other codes
// nothing is written and the answer is true.
template <bool TINY, typename T, int DH, int ROWS>
__device__ __forceinline__ bool append_heads(const Append8& a, Held<T, DH, ROWS>& in, T* q_out, int unit,
                                             int r0, int nr, int pos0, int64_t slot0, const double2* cs) {
  using In = Held<T, DH, ROWS>;
  constexpr int HALF = In::HALF, PER = In::PER, RPP = In::RPP, NI = In::NI;
  constexpr bool ONE = In::ONE;
  Half8<T>(&x)[NI] = in.x;
  Half8<T>(&y)[NI] = in.y;
  const int lane = threadIdx.x & 63, ch = lane % PER, row0 = in.row0(), head = in.head_of(unit);
  const int n_heads = a.H + 2 * a.KH;
  if (ONE && head >= n_heads) return false;               // whole groups of PER lanes, which alone exchange values
  const bool is_q = head < a.H, rot = a.rotate && head < a.H + a.KH;
  if (is_q && q_out == nullptr) return false;
  float u[NI][16];                                        // the rotated pairs' first halves, then the second ones
  float big = 0.f;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int r = min(row0 + i * RPP, nr - 1);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float f = x[i].get(j), g = y[i].get(j);
      bool ff = true, gf = true;
      if (rot) {
        const double2 c = cs[(r * 8 + j) * PER + ch + r * PER];
        const double p = f, q = g, s = fma(p, c.x, -(q * c.y)), t = fma(p, c.y, q * c.x);
        const bool last = sizeof(T) == 4 && is_q;         // fp32 is where the value stays
        f = last ? (float)s : to_odd<TINY>(s);
        g = last ? (float)t : to_odd<TINY>(t);
        ff = finite(s);
        gf = finite(t);
      } else if (!is_q) {
        ff = fabsf(f) < INFINITY;
        gf = fabsf(g) < INFINITY;
      }
      if (!is_q) {
        f = ff ? fminf(fmaxf(f, -TOP8), TOP8) : NAN;
        g = gf ? fminf(fmaxf(g, -TOP8), TOP8) : NAN;
        big = fmaxf(big, fmaxf(fabsf(f), fabsf(g)));      // fmaxf passes over NaN
      }
      u[i][j] = f;
      u[i][8 + j] = g;
    }
  }
  if (is_q) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int r = row0 + i * RPP;
      if (r >= nr) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[i].put(j, u[i][j]);
        y[i].put(j, u[i][8 + j]);
      }
      T* p = q_out + (int64_t)(r0 + r) * a.ldq + (int64_t)head * DH + ch * 8;
      *reinterpret_cast<Half8<T>*>(p) = x[i];
      *reinterpret_cast<Half8<T>*>(p + HALF) = y[i];
    }
    return false;
  }
#pragma unroll
  for (int m = 1; m < (ONE ? PER : 64); m <<= 1) big = fmaxf(big, __shfl_xor(big, m, 64));
  // the least e >= 1 with big <= 448 2^(e - 127) = 1.75 2^(e - 119)
  const uint32_t bits = __float_as_uint(big);
  int e = (int)(bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0);
  e = big > 0.f && e > 1 ? e : 1;
  if (!TINY && rot && e < 12) return true;                // from 12 on such a magnitude is less than half the smallest code
  const bool is_v = head >= a.H + a.KH;
  const int kh = head - a.H - (is_v ? a.KH : 0);
  uint8_t* pool = (is_v ? a.v : a.k) + ((int64_t)kh * a.slots + slot0) * DH;      // the run's first new row
  uint8_t* ex = a.exps + (((slot0 >> 4) * a.KH + kh) << 1) + (is_v ? 1 : 0);
  const int older = pos0 & 15;
  if (older) {                                            // rows of earlier steps keep the run's scale at least as large
    const int was = *ex;
    if (was >= e) {
      e = was;
    } else {
      // their codes times 2^(was - e), 16 bytes at a time; a shift of 2^-18 and less leaves zeros
      const float down = scale_of(127 - min(e - was, 60));
      constexpr int BPR = DH / 16;
      for (int i = ONE ? ch : lane; i < older * BPR; i += ONE ? PER : 64) {
        u32x4* p = reinterpret_cast<u32x4*>(pool - (int64_t)(older - i / BPR) * DH + (i % BPR) * 16);
        u32x4 w = *p;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 f = decode4(w[j], 1.f) * down;
          w[j] = encode4(f[0], f[1], f[2], f[3]);
        }
        *p = w;
      }
    }
  }
  // every lane of the head has read the byte: its loads are before the store in program order
  if ((ONE ? ch : lane) == 0) *ex = (uint8_t)e;
  const float inv = e < 254 ? scale_of(254 - e) : 1.f / scale_of(e);
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int r = row0 + i * RPP;
    if (r >= nr) continue;
    const float* w = u[i];
    uint8_t* p = pool + (int64_t)r * DH + ch * 8;
    *reinterpret_cast<u32x2*>(p) = u32x2{encode4(w[0] * inv, w[1] * inv, w[2] * inv, w[3] * inv),
                                         encode4(w[4] * inv, w[5] * inv, w[6] * inv, w[7] * inv)};
    *reinterpret_cast<u32x2*>(p + HALF) = u32x2{encode4(w[8] * inv, w[9] * inv, w[10] * inv, w[11] * inv),
                                                encode4(w[12] * inv, w[13] * inv, w[14] * inv, w[15] * inv)};
  }
  return false;
}

template <typename T, int DH>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4, 4))) void append8_kernel(Plan pl, Append8 a, const T* qkv, T* q_out) {
  constexpr int HALF = DH / 2, PER = HALF / 8;
  // cosine and sine of row r, pair 8 ch + j at (r * 8 + j) * PER + ch + r * PER: lanes of a row read neighbours, rows
  // differ in banks
  __shared__ double2 cs[16 * 9 * PER];
  const int split = a.split, share = (int)blockIdx.x % split, i = (int)blockIdx.x / split;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // revolutions per position of the pair whose angles this thread takes
  const int pair = threadIdx.x % HALF;
  const double inv = a.rotate ? exp2(-(2.0 * (double)pair / (double)DH) * a.log2_theta) * 0.15915494309189535 : 0.0;
  const int n_heads = a.H + 2 * a.KH, step = 4 * split, unit0 = share * 4 + wave;
  auto heads = [&](auto most, int units, int r0, int nr, int pos0, int64_t slot0) {
    using Rows = Held<T, DH, decltype(most)::value>;
    for (int unit = unit0; unit < units;) {
      const int begin = unit;
      uint32_t again = 0;                                 // heads to be taken with TINY, of up to 32
      for (int k = 0; k < 32 && unit < units; ++k, unit += step) {
        Rows rows;
        rows.load(qkv, a.ld, n_heads, unit, r0, nr);
        if (append_heads<false>(a, rows, q_out, unit, r0, nr, pos0, slot0, cs)) again |= 1u << k;
      }
      if (__builtin_expect(__any(again != 0), 0)) {
#pragma unroll 1
        for (int k = 0; k < 32; ++k)
          if (again >> k & 1) {
            Rows rows;
            rows.load(qkv, a.ld, n_heads, begin + k * step, r0, nr);
            append_heads<true>(a, rows, q_out, begin + k * step, r0, nr, pos0, slot0, cs);
          }
      }
    }
  };
  const int first = i < pl.n_req ? uniform(pl.cu_seqlens[i]) : (i - pl.n_req) * 16;
  const int end = i < pl.n_req ? first + 1 : min(first + 16, pl.T);
  for (int r0 = first, next; r0 < end; r0 = next) {
    const int pos0 = uniform(pl.pos[r0]), p = i < pl.n_req ? i : uniform(pl.row_req[r0]);
    const int begin = uniform(pl.cu_seqlens[p]), past = uniform(pl.cu_seqlens[p + 1]);
    next = min(past, r0 + 16 - (pos0 & 15));
    if (i >= pl.n_req && (r0 == begin || (pos0 & 15))) continue;   // a request's first run, or inside one
    const int nr = next - r0;
    const int64_t slot0 = page_slot(row_of(a.kp, uniform(pl.order[p])), a.kp.log2_page, pos0);
    if (a.rotate) {
      if (r0 != first) __syncthreads();                   // block-uniform; the run before has been rotated
      for (int r = threadIdx.x / HALF; r < nr; r += 256 / HALF) {
        const double rev = (double)(pos0 + r) * inv;
        double sine, cosine;
        sincospi(2.0 * (rev - rint(rev)), &sine, &cosine);
        cs[(r * 8 + (pair & 7)) * PER + (pair >> 3) + r * PER] = double2{cosine, sine};
      }
      __syncthreads();
    }
    if (nr == 1) heads(std::integral_constant<int, 1>{}, (n_heads + 64 / PER - 1) / (64 / PER), r0, nr, pos0, slot0);
    else if (64 / PER < 16 && nr <= 64 / PER) heads(std::integral_constant<int, 64 / PER>{}, n_heads, r0, nr, pos0, slot0);
    else heads(std::integral_constant<int, 16>{}, n_heads, r0, nr, pos0, slot0);
  }
}

// ---------------------------------------------------------------------------
// Attention, bf16 queries: one block per 16 packed queries of one request and key head and chunk of its keys; each of the 4
// waves streams every 4th 32-key tile of the chunk on its own and the waves' partial softmax sums are merged through
// LDS at the end (as in the bf16 cache's few-row kernel, k_paged.hip).  Codes become bf16 in registers: K on the way to
// the MFMA, V on the way to a wave-private LDS tile that the transposing LDS read turns into the V^T operand.
// A lane's 16-byte load of a K row holds 16 consecutive head dims, two MFMA steps of 8; the queries' fragments take the
// same dims, as a dot product does not mind their order.
// Weights are rounded to bf16 for the product with V, which the matrix cores take at 16 times fp32's rate: by up to 2^-8 of
// each, as the output is by its own rounding; their sum and maximum are fp32.  Against 64 bits the output is off by 1.0
// to 1.1 times what the fp32 form rounded once is.
// Memory bound: 256 requests with up to 1028 visible keys, 32 heads of 128 on 32: 305 us, 6.2 TB/s (at most 6.5 here); 8
// requests of 32768 to 131072, 32 heads on 8: 205 us, 6.2 TB/s.  One row after 300 keys: 8 us, the latency of a few
// dependent loads.
// NB tiles' registers: with few blocks, or long ones, the loads of two tiles are in flight while one is computed (head dim
// 128: 204 registers, two blocks on a CU; 64: one tile ahead and three).  Otherwise one tile at a time, and four blocks on a CU
// (64: five) hide each other's loads and starts.  With head dim 128, one tile and three: 256 rows of 30 to 60 keys 39 us and
// 64, of 256 to 2048 440 and 519, 8 of 32768 to 131072 216 and 205, one of 30000 21.2 and 19.4; with head dim 64, one and
// two: 256 of 30 to 60 15.4 and 16.9, 256 of 200 to 2000 110 and 114, 16 of 130 to 400 8.3 and 7.6.
// ---------------------------------------------------------------------------
// The last request whose blocks begin at id or before it (the first one's at 0), by whole waves: 64 places are looked at
// at once, as each step of a search waits for its load.  5 prompts of 40 to 250 rows and 19 single ones after 64 to
// 2000 keys, 16 heads of 64: 40.8 us, by halves 42.4.
template <typename F>
__device__ __forceinline__ int last_request(int n_req, int id, F begin) {
  int lo = 0;
  for (int n = n_req; n > 1;) {
    const int step = (n + 63) >> 6, at = (int)(threadIdx.x & 63) * step;
    const int k = __popcll(__ballot(at < n && begin(lo + min(at, n - 1)) <= id)) - 1;
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

// The exponent bytes of K (low) and V (high) of two runs, even lanes the first's and odd lanes the second's.  (A load from
// the same address in every lane would be made a scalar at once, and waited for before anything after it is issued.)
__device__ __forceinline__ uint32_t runs_exps(const uint8_t* exps, int64_t slot0, int64_t slot1, int KH, int h) {
  const int64_t slot = threadIdx.x & 1 ? slot1 : slot0;
  return reinterpret_cast<const uint16_t*>(exps)[(slot >> 4) * KH + h];
}
__device__ __forceinline__ float k_scale(uint32_t ex, int run) { return scale_of(__builtin_amdgcn_readlane(ex, run) & 0xFF); }
__device__ __forceinline__ float v_scale(uint32_t ex, int run) { return scale_of(__builtin_amdgcn_readlane(ex, run) >> 8); }

__device__ __forceinline__ bool is_nan8(uint32_t code) { return (code & 0x7F) == 0x7F; }

// A lane converts 16 consecutive head dims of a V (or K) row, two 16-byte chunks of bf16.  In LDS the rows' first chunks lie
// beside each other, then the second ones, so that the lanes of a store fill whole runs of banks: logical chunk c holds
// head dims from here on.  Odd rows of 128 bytes have the two halves swapped, as two of them make such a run.
template <int DH>
__device__ __forceinline__ constexpr int dims_of(int c) { return 16 * (c % (DH / 16)) + 8 * (c / (DH / 16)); }
template <int DH>
__device__ __forceinline__ int odd_rows(int r) { return DH == 64 ? (r & 1) << 2 : 0; }   // to a chunk's number by xor

// Swizzle of the 32-byte segments of a V row in a few-row tile: the 8 rows that a half of a transposing read touches, one
// segment each, lie in different banks.
template <int DH>
__device__ __forceinline__ int few_vswz(int r) { return DH == 128 ? r & 7 : (r >> 1) & 3; }

template <int DH, int NB, bool TABLE>
__device__ __forceinline__ void few_block8(const Plan& pl, const PagedAttn& a, const uint8_t* __restrict__ exps, int id, char* smem) {
  constexpr int LPR = DH / 16;         // lanes per K / V row (16 bytes each)
  constexpr int RPI = 64 / LPR;        // rows per wave-wide load
  constexpr int VI = 32 / RPI;         // V loads per lane and tile
  constexpr int KL = DH / 64;          // K loads per lane and 16 keys
  constexpr int KS = DH / 32;          // MFMA steps over the head dims
  constexpr int ND = DH / 16;          // output tiles
  __shared__ float sm[4][16], sl[4][16];

  Work w;
  if constexpr (TABLE) {
    const table_t parts = table_of(pl, a, TAB_FEW);
    w.p = last_request(pl.n_req, id, [&](int p) { return parts[p]; });
    id -= parts[w.p];
  } else {
    w.h = id % a.KH; id /= a.KH;
    w.c = id % a.few_chunks; id /= a.few_chunks;
    w.qt = id % a.qtiles;
    w.p = id / a.qtiles;
  }
  const int R0 = uniform(pl.cu_seqlens[w.p]), m = uniform(pl.cu_seqlens[w.p + 1]) - R0, ctx = uniform(pl.ctx[w.p]);
  const int request = uniform(pl.order[w.p]);            // with them, not behind what they decide
  if (!few_rows(VFM_BF16, m, a.G)) return;              // block-uniform, as every exit below
  const int qn = m * a.G;
  if (!TABLE && w.qt * 16 >= qn) return;
  const Chunks ck = request_chunks(VFM_BF16, m, ctx, a.G, a.KH, a.window, a.n_sink, true);
  if constexpr (TABLE) {
    w.h = id % a.KH; id /= a.KH;
    w.c = id % ck.n;
    w.qt = id / ck.n;
  } else if (w.c >= ck.n) {
    return;
  }
  const Vis vis = visible_runs<4>(ctx, ctx + m - 1, a.window, a.n_sink);
  const int t0 = w.c * ck.tiles, t1 = min(t0 + ck.tiles, (vis.n + 1) / 2);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = lane & 15, g = lane >> 4;
  const int qi = min(w.qt * 16 + x, qn - 1);
  const int jq = ctx + qi / a.G;
  const int j0 = ctx + w.qt * 16 / a.G, j1 = ctx + min(w.qt * 16 + 15, qn - 1) / a.G;
  int head;
  const int64_t row = out_row(a, R0, w.h, qi, head);
  bf16x8 qf[KS];
  {
    const bf16* qr = (const bf16*)a.q + row * a.ldq + head * DH + 16 * g;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qr + 64 * (s >> 1) + 8 * (s & 1));
  }
  const page_row prow = row_of(a.kp, request);
  const int lp = a.kp.log2_page;
  const uint8_t* kh = (const uint8_t*)a.k + (int64_t)w.h * a.slots * DH;
  const uint8_t* vh = (const uint8_t*)a.v + (int64_t)w.h * a.slots * DH;
  bf16* Vs = reinterpret_cast<bf16*>(smem) + wave * 32 * DH;

  // a tile's two runs (one page each, as a page holds a multiple of 16 positions); runs past the last re-read it, unseen
  auto run_pos = [&](int t, int e) { return 16 * vis.run(min(2 * t + e, vis.n - 1)); };
  u32x4 kf[NB][2][KL], vf[NB][VI];
  uint32_t ex[NB];
  int page[2], in_page[2];
  auto look_up = [&](int t) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int k = run_pos(t, e);
      page[e] = prow[k >> lp];
      in_page[e] = k & ((1 << lp) - 1);
    }
  };
  // The tile's runs are the two sub-tiles of keys, so that a load's run, and with it its base and scale, is the wave's.
  const uint32_t koff = x * DH + 16 * g, voff = (lane / LPR & 15) * DH + 16 * (lane % LPR);
  auto load = [&](int b) {
    const uint8_t *kr[2], *vr[2];
    int slot[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      slot[e] = (page[e] << lp) + in_page[e];
      kr[e] = kh + (int64_t)slot[e] * DH;
      vr[e] = vh + (int64_t)slot[e] * DH;
    }
    ex[b] = runs_exps(exps, slot[0], slot[1], a.KH, w.h);
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int s = 0; s < KL; ++s)
        kf[b][e][s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kr[e] + (koff + 64 * s)));
#pragma unroll
    for (int i = 0; i < VI; ++i)
      vf[b][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vr[(RPI * i) >> 4] + (voff + ((RPI * i) & 15) * DH)));
  };

  f32x4 o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = LOWEST, l_run = 0.f;

  // where a lane's two chunks of row RPI i + vst_row go, for i = 0 (the swizzle is the same for all of them)
  const int vst_row = lane / LPR, vst_swz = few_vswz<DH>(vst_row) << 1 ^ odd_rows<DH>(vst_row);
  char* const vst[2] = {reinterpret_cast<char*>(Vs + vst_row * DH) + 16 * ((lane % LPR) ^ vst_swz),
                        reinterpret_cast<char*>(Vs + vst_row * DH) + 16 * ((lane % LPR + LPR) ^ vst_swz)};
  const int vrow = 4 * g + (x >> 2);
  const int vbase = vrow * DH * 2 + ((few_vswz<DH>(vrow) << 5) ^ (odd_rows<DH>(vrow) << 4)) + (x & 3) * 8;
  // head dims of the lane's outputs of tile d: chunk 2 d + g / 2, from 4 (g % 2) on
  auto out_dims = [&](int d) { return dims_of<DH>(2 * d + (g >> 1)) + 4 * (g & 1); };

  auto compute = [&](int b, int t) {
    const int p0 = run_pos(t, 0);
    const int p1 = 2 * t + 1 < vis.n ? run_pos(t, 1) : INT32_MAX - 64;   // no second run: unseen
    const bool full = p1 == p0 + 16 && seen_by_all(j0, j1, p0, p0 + 31, a.window, a.n_sink);
    bool poison = false;
    // V to LDS
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      const int r = RPI * i + vst_row;
      const float scale = v_scale(ex[b], (RPI * i) >> 4);
      bf16x8 v[2] = {decode8(vf[b][i][0], vf[b][i][1], scale), decode8(vf[b][i][2], vf[b][i][3], scale)};
      if (!full) {
        const int k = (((RPI * i) >> 4) ? p1 : p0) + (r & 15);
        if (!seen_by_any(j0, j1, k, a.window, a.n_sink)) {
          v[0] = v[1] = bf16x8{};
        } else if (j0 != j1 && !seen_by_all(j0, j1, k, k, a.window, a.n_sink)) {
          v[0] = drop_nonfinite(v[0], poison);
          v[1] = drop_nonfinite(v[1], poison);
        }
      }
      *reinterpret_cast<bf16x8*>(vst[0] + RPI * i * DH * 2) = v[0];
      *reinterpret_cast<bf16x8*>(vst[1] + RPI * i * DH * 2) = v[1];
    }
    wave_lds_order();
    // S^T
    float s[8];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float kscale = k_scale(ex[b], e);
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        const u32x4& c = kf[b][e][st >> 1];
        acc = mfma16(decode8(c[2 * (st & 1)], c[2 * (st & 1) + 1], kscale), qf[st], acc);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * e + i] = acc[i];
    }
    if (!full) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        s[i] = sees(jq, (i < 4 ? p0 : p1) + 4 * g + (i & 3), a.window, a.n_sink) ? s[i] : -INFINITY;
    }
    float mb = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    mb = max_x32(max_x16(mb));
    if (__any(mb > m_run)) {                              // elsewhere the factor is 1
      const float m_new = fmaxf(m_run, mb);
      const float alpha = fast_exp2((m_run - m_new) * a.scale_log2);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int i = 0; i < ND; ++i) o[i] *= alpha;
    }
    float e8[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e8[i] = fast_exp2((s[i] - m_run) * a.scale_log2);
      l_run += e8[i];
    }
    const bf16x8 pf = pack8(e8[0], e8[1], e8[2], e8[3], e8[4], e8[5], e8[6], e8[7]);
    int vb = vbase;
    asm volatile("" : "+v"(vb));                          // the ND addresses made here, not held over the loop
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      const char* vp = reinterpret_cast<const char*>(Vs) + (vb ^ (d << 5));
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vp));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vp + 16 * DH * 2));
      bf16x8 f;
      __builtin_memcpy(&f, &lo, 8);
      __builtin_memcpy(reinterpret_cast<char*>(&f) + 8, &hi, 8);
      o[d] = mfma16(f, pf, o[d]);
    }
    wave_lds_order();
    if (__any(poison)) {                                  // rare: re-read the tile's V rows from memory
      for (int r = 0; r < 32; ++r) {
        const int k = (r < 16 ? p0 : p1) + (r & 15);
        if (!seen_by_any(j0, j1, k, a.window, a.n_sink) || seen_by_all(j0, j1, k, k, a.window, a.n_sink)) continue;
        const uint8_t* vr = vh + (int64_t)page_slot(prow, lp, k) * DH;
        const bool see = sees(jq, k, a.window, a.n_sink);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const uint32_t c = *reinterpret_cast<const uint32_t*>(vr + out_dims(d));
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (see && is_nan8(c >> (8 * i))) o[d][i] = NAN;
          __builtin_amdgcn_sched_barrier(0);              // no registers for more loads in flight
        }
      }
    }
  };

  // tiles t0 + wave, + 4, ...: the loads of NB - 1 tiles in flight while one is computed, page lookups a tile ahead of them
  int t = t0 + wave;
  if (t < t1) {
    constexpr int AHEAD = 4 * (NB - 1);
    look_up(t);
#pragma unroll
    for (int b = 0; b < NB - 1; ++b)
      if (t + 4 * b < t1) { load(b); if (t + 4 * b + 4 < t1) look_up(t + 4 * b + 4); }
    auto step = [&](int b) {
      if (t + AHEAD < t1) { load((b + NB - 1) % NB); if (t + AHEAD + 4 < t1) look_up(t + AHEAD + 4); }
      compute(b, t);
      t += 4;
      return t < t1;
    };
    if constexpr (NB == 1) while (step(0)) {}
    else if constexpr (NB == 2) while (step(0) && step(1)) {}
    else while (step(0) && step(1) && step(2)) {}
  }
  l_run = sum_x32(sum_x16(l_run));

  // merge the four waves
  __syncthreads();
  float* so = reinterpret_cast<float*>(smem);             // [4][16][DH]
  if (lane < 16) { sm[wave][x] = m_run; sl[wave][x] = l_run; }
#pragma unroll
  for (int d = 0; d < ND; ++d)
    *reinterpret_cast<f32x4*>(so + (wave * 16 + x) * DH + (out_dims(d) ^ (x << 2))) = o[d];   // queries in different banks
  __syncthreads();
  const int nq = min(16, qn - w.qt * 16);
  for (int e = tid; e < nq * DH / 4; e += 256) {
    const int q = e / (DH / 4), d = (e % (DH / 4)) * 4;
    const float M = fmaxf(fmaxf(sm[0][q], sm[1][q]), fmaxf(sm[2][q], sm[3][q]));
    float L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float wt = fast_exp2((sm[i][q] - M) * a.scale_log2);
      L += sl[i][q] * wt;
      // a wave without any visible key has weight 0 and zeros
      acc += *reinterpret_cast<const f32x4*>(so + (i * 16 + q) * DH + (d ^ (q << 2))) * wt;
    }
    int hd;
    const int64_t r = out_row(a, R0, w.h, w.qt * 16 + q, hd);
    if (ck.n == 1) {
      const float inv = 1.f / L;
      bf16x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (bf16)(acc[i] * inv);
      *reinterpret_cast<bf16x4*>((bf16*)a.out + r * a.ldo + hd * DH + d) = v;
    } else {
      const int64_t rec = record_of<TABLE>(pl, a, w.p, R0, ck.n, r, hd) + w.c;
      *reinterpret_cast<f32x4*>(a.rec_o + rec * DH + d) = acc;
      if (d == 0) a.rec_ml[rec] = make_float2(M, L);
    }
  }
}

// ---------------------------------------------------------------------------
// Many rows (prompts and chunks), bf16: one block per 128 packed queries of one request and key head (and chunk of the keys
// where the request has few blocks), waves of 32 queries, 64-key tiles in two LDS stages by turns, as in the bf16 cache's
// many-row kernel (k_paged.hip).  Codes go through registers: a thread loads 16 of a K and of a V row ahead and stores
// them as bf16 a step later, so each is converted once per block.
// 4 chunks of 1900 to 2048 rows after 3000 to 9000, window 4096, 32 heads of 128 on 8: 550 to 565 us by machine, 940 to 960
// TFLOP/s of visible products, as over a bf16 cache (a large matrix product: 1370): the matrix cores are busy for 47% of the
// cycles, the vector ALU for 47, LDS for 36.  Blocks of 8 waves, which halve the conversions per query, give 1%; V's
// conversion beside the products in place of the scores loses 2.  The matrix cores' own 8-bit products (a query as the
// sum of two codes) would need no conversion of K, but their sums hold 16 bits (1.6e-5 of random rows' products of 64).
// Weights are rounded to bf16 as above, and summed so: 1.28 times the error of the fp32 form rounded once.  With head dim 64 the
// softmax weighs more: 8 prompts of 4096, window 1024, 16 heads on 4, 209 to 222 us, the vector ALU busy for 51% of the
// cycles, the matrix cores for 28, 29% of the waves' time waiting.
// ---------------------------------------------------------------------------
template <int DH, bool TABLE>
__device__ __forceinline__ void rows_block8(const Plan& pl, const PagedAttn& a, const uint8_t* __restrict__ exps, int id, bf16* stage0, bf16* stage1) {
  constexpr int NW = 4;                  // waves
  constexpr int LPR = DH / 16;           // lanes per row of codes (16 bytes each)
  constexpr int CH = DH / 8;             // 16-byte chunks per row of a stage
  constexpr int RPI = 64 / LPR;          // rows per wave-wide load
  constexpr int NI = 64 / (NW * RPI);    // K (and V) loads per wave and tile
  constexpr int KS = DH / 16;            // MFMA steps over the head dims
  constexpr int ND = DH / 32;            // output tiles
  // Stage j: K of a tile t with t mod 2 = j, then V of tile t - 1 (a step reads K a tile ahead of V).
  constexpr int TE = 64 * DH;
  auto stage = [&](auto b) -> bf16* {
    if constexpr (b == 0) return stage0;
    else return stage1;
  };
  __shared__ int s_poison;

  const int rb = rows_per_block(a.G);
  Work w;
  if constexpr (TABLE) {
    const table_t parts = table_of(pl, a, TAB_ROWS);
    w.p = last_request(pl.n_req, id, [&](int p) { return parts[p]; });
    id -= parts[w.p];
  } else {
    w.h = id % a.KH; id /= a.KH;
    w.c = id % a.rows_chunks; id /= a.rows_chunks;
    // request p's blocks start at cu[p] / rb + p: at least ceil(m / rb) before the next request's
    w.p = last_request(pl.n_req, id, [&](int p) { return pl.cu_seqlens[p] / rb + p; });
  }
  const int R0 = uniform(pl.cu_seqlens[w.p]), m = uniform(pl.cu_seqlens[w.p + 1]) - R0, ctx = uniform(pl.ctx[w.p]);
  const int request = uniform(pl.order[w.p]);            // with them, not behind what they decide
  // a request's last rows see the most keys: they come first
  const int nb = (m + rb - 1) / rb;
  int bi = id - (R0 / rb + w.p);
  if (few_rows(VFM_BF16, m, a.G) || (!TABLE && bi >= nb)) return;   // block-uniform, as every exit below
  const Chunks ck = request_chunks(VFM_BF16, m, ctx, a.G, a.KH, a.window, a.n_sink, true);
  if constexpr (TABLE) {
    w.h = id % a.KH; id /= a.KH;
    w.c = id % ck.n;
    bi = id / ck.n;
  } else if (w.c >= ck.n) {
    return;
  }
  const int r0 = (nb - 1 - bi) * rb, nr = min(rb, m - r0);
  const int j0 = ctx + r0, j1 = j0 + nr - 1, qn = nr * a.G;
  const Vis vis = visible_runs<6>(j0, j1, a.window, a.n_sink);
  const int tpc = (vis.n + ck.n - 1) / ck.n;
  const int t0 = w.c * tpc, t1 = min(t0 + tpc, vis.n);    // may be empty: an empty record
  const int lo_any = a.window > 0 ? max(0, j0 - a.window + 1) : 0;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = lane & 31, h2 = lane >> 5;
  const int qi = min(wave * 32 + x, qn - 1);
  const int jq = j0 + qi / a.G;
  // the wave's rows
  const int wj0 = j0 + min(wave * 32, qn - 1) / a.G, wj1 = j0 + min(wave * 32 + 31, qn - 1) / a.G;
  int head;
  const int64_t row = out_row(a, R0 + r0, w.h, qi, head);
  bf16x8 qf[KS];
  {
    const bf16* qr = (const bf16*)a.q + row * a.ldq + head * DH;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qr + dims_of<DH>(2 * s + h2));
  }
  const page_row prow = row_of(a.kp, request);
  const int lp = a.kp.log2_page;
  const uint8_t* kh = (const uint8_t*)a.k + (int64_t)w.h * a.slots * DH;
  const uint8_t* vh = (const uint8_t*)a.v + (int64_t)w.h * a.slots * DH;
  if (tid == 0) s_poison = -1;

  f32x16 o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  float m_run = LOWEST, l_run = 0.f;

  // A lane's load i of a tile: 16 codes of row RPI (NW i + wave) + lane / LPR, from dim 16 (lane % LPR).
  const int lrow = RPI * wave + lane / LPR;               // mod 16: the row in its run
  const uint32_t off = (lrow & 15) * DH + (lane % LPR) * 16;   // from the run's first row, which is a scalar
  // Pages of the wave's runs of a tile (scalar loads, a step ahead of their use) and where the runs
  // start in them.  A run that no row sees reads a seen one instead: its page may not exist.
  int page[NI], in_page[NI];
  auto look_up = [&](int t) {
    const int kb = 64 * vis.run(min(t, vis.n - 1));
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      int k = min(kb + (RPI * (NW * i + wave) & ~15), j1 & ~15);
      if (k + 15 < lo_any && k >= a.n_sink) k = lo_any & ~15;
      page[i] = prow[k >> lp];
      in_page[i] = k & ((1 << lp) - 1);
    }
  };
  // Loads K of the tile looked up last and V of the one looked up before it; looks `next` up.  Past the last tile that one
  // is loaded again, into stages that nothing reads any more: the loop needs no branch.
  int vslot[NI] = {};
  u32x4 kr[NI], vr[NI];
  uint32_t kx = 0, vx = 0;
  auto load = [&](int next) {
    int kslot[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) kslot[i] = (page[i] << lp) + in_page[i];
    look_up(next);
    vx = kx;
    kx = runs_exps(exps, kslot[0], kslot[NI - 1], a.KH, w.h);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      kr[i] = *reinterpret_cast<const u32x4*>(kh + (int64_t)kslot[i] * DH + off);
      vr[i] = *reinterpret_cast<const u32x4*>(vh + (int64_t)vslot[i] * DH + off);
      vslot[i] = kslot[i];
    }
  };
  // where the two chunks that a lane's codes become go in a stage's K and V, for i = 0: row RPI NW i + lrow has the same
  // swizzle for every i
  const int seg = lane % LPR, flip = odd_rows<DH>(lrow), row_at = lrow * DH;
  const int k_at[2] = {row_at + 8 * rows_kswz<DH>(lrow, seg ^ flip), row_at + 8 * rows_kswz<DH>(lrow, (seg + LPR) ^ flip)};
  const int v_at[2] = {row_at + 8 * rows_vswz<DH>(lrow, seg ^ flip), row_at + 8 * rows_vswz<DH>(lrow, (seg + LPR) ^ flip)};
  // what was loaded, as bf16 into stage b
  auto store = [&](auto b, bool with_v) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const float ks = k_scale(kx, i), vs = v_scale(vx, i);
      bf16* to = stage(b) + RPI * NW * i * DH;
      *reinterpret_cast<bf16x8*>(to + k_at[0]) = decode8(kr[i][0], kr[i][1], ks);
      *reinterpret_cast<bf16x8*>(to + k_at[1]) = decode8(kr[i][2], kr[i][3], ks);
      if (with_v) {
        *reinterpret_cast<bf16x8*>(to + TE + v_at[0]) = decode8(vr[i][0], vr[i][1], vs);
        *reinterpret_cast<bf16x8*>(to + TE + v_at[1]) = decode8(vr[i][2], vr[i][3], vs);
      }
    }
  };
  // every wave's LDS accesses have finished
  auto meet = [&]() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // V rows of a tile that some row of the block does not see: zeros where none sees them, no
  // infinities or NaN where some do
  auto mend = [&](auto b, int t) {
    const int kb = 64 * vis.run(t);
#pragma unroll 1
    for (int i = 0; i < NI; ++i) {
      const int k = kb + RPI * NW * i + lrow;
      bf16* v = stage(b) + TE + RPI * NW * i * DH;
      bf16x8 *lo = reinterpret_cast<bf16x8*>(v + v_at[0]), *hi = reinterpret_cast<bf16x8*>(v + v_at[1]);
      if (!seen_by_any(j0, j1, k, a.window, a.n_sink)) {
        *lo = *hi = bf16x8{};
      } else if (!seen_by_all(j0, j1, k, k, a.window, a.n_sink)) {
        bool found = false;
        const bf16x8 l = drop_nonfinite(*lo, found), h = drop_nonfinite(*hi, found);
        if (found) { *lo = l; *hi = h; s_poison = t; }
      }
    }
  };

  // fragment addresses (bytes): K row x of a 32-key half, chunk 2 s + h2;
  // V: the transposing read takes 4 keys x 16 dims per 16 lanes, lane (x & 15)
  // bringing key (x & 15) / 4, dims 4 (x & 3).  Its rows differ from the lane's
  // first by multiples of 8, which leave the swizzle alone.
  const int kq = x & 15, gq = x >> 4;
  const int kaddr = x * DH * 2 + (rows_kswz<DH>(x, h2 ^ odd_rows<DH>(x)) << 4);
  const int vaddr = (4 * h2 + (kq >> 2)) * DH * 2 + (rows_vswz<DH>(kq >> 2, odd_rows<DH>(kq >> 2)) << 4) + gq * 32 + (kq & 3) * 8;
  // head dims of the lane's outputs 4 j .. of tile d: chunk 4 d + j, from 4 h2 on
  auto out_dims = [&](int d, int j) { return dims_of<DH>(4 * d + j) + 4 * h2; };

  // S^T of a tile: two 32-key halves; lane half h2, register i: key 8 (i / 4) + 4 h2 + i % 4
  auto scores = [&](auto b, f32x16 (&st)[2]) {
    const char* kp = reinterpret_cast<const char*>(stage(b));
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      f32x16 acc;
#pragma unroll
      for (int j = 0; j < 16; ++j) acc[j] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const bf16x8 f = *reinterpret_cast<const bf16x8*>(kp + kt * 32 * DH * 2 + (kaddr ^ (s << 5)));
        acc = mfma32(f, qf[s], acc);
      }
      st[kt] = acc;
    }
  };
  auto mask = [&](int t, f32x16 (&st)[2]) {
    const int kb = 64 * vis.run(t);
    if (seen_by_all(wj0, wj1, kb, kb + 63, a.window, a.n_sink)) return;
    // made anew in each masked tile: held over the loop, the compares' lane masks would fill the scalar registers
    int d0 = jq - kb - 4 * h2, n0 = a.n_sink - kb - 4 * h2;     // of the lane's key 0
    asm volatile("" : "+v"(d0), "+v"(n0));
    const int win = a.window > 0 ? a.window : INT32_MAX;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int k = 32 * kt + 8 * (i >> 2) + (i & 3);
        const bool see = (d0 >= k) & ((d0 - k < win) | (k < n0));
        st[kt][i] = see ? st[kt][i] : -INFINITY;
      }
  };
  // largest score of the lane's query
  auto largest = [&](const f32x16 (&st)[2]) {
    float mb = st[0][0];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) mb = fmaxf(mb, st[kt][i]);
    return max_x32(mb);
  };
  // The running maximum follows the scores only where one passes it by 8 (a factor of 256, which
  // neither fp32 sums nor bf16 weights mind): with 32 queries a wave, some maximum grows in most
  // tiles, and the products would be rescaled that often.
  auto follow = [&](float mb) {
    if (__any((mb - m_run) * a.scale_log2 > 8.f)) {
      const float m_new = fmaxf(m_run, mb);
      const float alpha = fast_exp2((m_run - m_new) * a.scale_log2);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int i = 0; i < ND; ++i) o[i] *= alpha;
    }
  };
  // A weight is one fma here, 2^(s scale - m scale): the rest that m scale's rounding leaves is a factor common
  // to all of a query's weights, below 2^(1/16) while |m scale| < 2^20.  Beyond (m at its start, too) the
  // tile's scores are made differences from m first.  (Differences throughout: 579 us for the 564 of 4 chunks.)
  float neg_m = 0.f;
  auto settle = [&](f32x16 (&st)[2]) {
    neg_m = -m_run * a.scale_log2;
    if (__any(!(fabsf(neg_m) < 1048576.f))) {
      neg_m = 0.f;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) st[kt][i] -= m_run;
    }
  };
  // P^T of 16 keys u of a tile, 8 of them in this lane
  auto weights = [&](const f32x16 (&st)[2], int u, bf16x8 (&pf)[4]) {
    float e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = fast_exp2(fmaf(st[u >> 1][8 * (u & 1) + i], a.scale_log2, neg_m));
    pf[u] = pack8(e[0], e[1], e[2], e[3], e[4], e[5], e[6], e[7]);
  };
  // Their sum, of the weights rounded to bf16 that the products use (two to an instruction; and what rounding
  // adds to all weights of a row divides out), and the products
  auto products = [&](auto b, const bf16x8 (&pf)[4]) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        l_run = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pf[u][2 * i], pf[u][2 * i + 1]}, bf16x2{(bf16)1.f, (bf16)1.f}, l_run, false);
    const char* vp = reinterpret_cast<const char*>(stage(b) + TE);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const char* q = vp + (vaddr ^ (d << 6)) + u * 16 * DH * 2;
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(q));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(q + 8 * DH * 2));
        bf16x8 f;
        __builtin_memcpy(&f, &lo, 8);
        __builtin_memcpy(reinterpret_cast<char*>(&f) + 8, &hi, 8);
        o[d] = mfma32(f, pf[u], o[d]);
      }
  };
  // the NaN that `mend` took out of tile t
  auto add_nonfinite = [&](int t) {
    const int kb = 64 * vis.run(t);
#pragma unroll 1
    for (int r = 0; r < 64; ++r) {
      const int k = kb + r;
      if (!seen_by_any(j0, j1, k, a.window, a.n_sink) || seen_by_all(j0, j1, k, k, a.window, a.n_sink)) continue;
      const uint8_t* vrow = vh + (int64_t)(page_slot(prow, lp, k)) * DH;
      if (sees(jq, k, a.window, a.n_sink)) {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t c = *reinterpret_cast<const uint32_t*>(vrow + out_dims(d, j));
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (is_nan8(c >> (8 * i))) o[d][4 * j + i] = NAN;
            __builtin_amdgcn_sched_barrier(0);            // rare: no registers for loads in flight
          }
      }
    }
  };

  // While the weights of tile t are computed (vector ALU), the matrix cores already take the scores
  // of tile t + 1; while they take the products of t, its largest scores are found.  K of tile t + 1
  // and V of tile t were stored a step ago from what had been loaded in the step before;
  // the barrier makes every wave's part visible, and frees K of tile t and V of tile t - 1.
  if (t0 < t1) {
    f32x16 sa[2], sb[2];
    look_up(t0);
    load(t0 + 1);
    store(std::integral_constant<int, 0>{}, false);
    load(t0 + 2);
    store(std::integral_constant<int, 1>{}, true);
    load(t0 + 3);
    meet();
    scores(std::integral_constant<int, 0>{}, sa);
    mask(t0, sa);
    follow(largest(sa));
    settle(sa);
    // tile t, t mod 2 = j: its scores st, the next one's sn (behind the last tile: of what the stage
    // holds, and not used)
    auto step = [&](auto j, int t, f32x16 (&st)[2], f32x16 (&sn)[2]) {
      constexpr auto jn = std::integral_constant<int, 1 - j>{};   // holds K of tile t + 1, V of tile t
      meet();
      const int kb = 64 * vis.run(t);
      if (!seen_by_all(j0, j1, kb, kb + 63, a.window, a.n_sink)) {
        mend(jn, t);
        meet();
      }
      bf16x8 pf[4];
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);                       // before the other wave of the SIMD: 1%
      // Scores of t + 1 (2 KS MFMAs) beside the first half of t's weights, the conversion of what was loaded and the next
      // loads; a fragment is read four ahead of its MFMA.
      store(j, true);
      load(t + 4);
      scores(jn, sn);
      weights(st, 0, pf);
      weights(st, 1, pf);
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int s = 0; s < 2 * KS; ++s) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x402, 96 / (2 * KS), 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        if (s % 2) __builtin_amdgcn_sched_group_barrier(0x200, 4 * NI * 2 / (2 * KS), 0);
        if (s % (2 * KS / 8) == 1) __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) asm volatile("" : "+v"(pf[u]));   // not put off behind the mask
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(0);
      if (t + 1 < t1) mask(t + 1, sn);
      __builtin_amdgcn_sched_barrier(0);
      // products of t (4 ND MFMAs) beside the second half of its weights and the largest scores of t + 1
      weights(st, 2, pf);
      weights(st, 3, pf);
      products(jn, pf);
      const float mb = largest(sn);
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int s = 0; s < 4 * ND; ++s) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x402, 96 / (4 * ND), 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (s_poison == t) add_nonfinite(t);
      if (t + 1 >= t1) return false;
      follow(mb);
      settle(sn);
      return true;
    };
    for (int t = t0;; t += 2) {
      if (!step(std::integral_constant<int, 0>{}, t, sa, sb)) break;
      if (!step(std::integral_constant<int, 1>{}, t + 1, sb, sa)) break;
    }
  }
  l_run = sum_x32(l_run);
  if (wave * 32 + x >= qn) return;
  if (ck.n == 1) {
    const float inv = 1.f / l_run;
    bf16* orow = (bf16*)a.out + row * a.ldo + head * DH;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (bf16)(o[d][4 * j + i] * inv);
        *reinterpret_cast<bf16x4*>(orow + out_dims(d, j)) = v;
      }
  } else {
    const int64_t rec = record_of<TABLE>(pl, a, w.p, R0, ck.n, row, head) + w.c;
    float* ro = a.rec_o + rec * DH;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4*>(ro + out_dims(d, j)) =
            f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
    if (h2 == 0) a.rec_ml[rec] = make_float2(m_run, l_run);
  }
}

// ROWS / FEW as in the bf16 cache's kernel (k_paged.hip): the blocks of a step's many-row requests, then those of its few-row
// ones, in one launch.
template <int DH, bool ROWS, int NB, int WAVES, bool TABLE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(WAVES, WAVES))) void attn8_bf16_kernel(
    Plan pl, PagedAttn a, const uint8_t* __restrict__ exps, int rows_blocks) {
  __shared__ __attribute__((aligned(16))) bf16 stage0[128 * DH], stage1[ROWS ? 128 * DH : 8];
  if constexpr (NB > 0)
    if ((int)blockIdx.x >= rows_blocks) {
      few_block8<DH, NB, TABLE>(pl, a, exps, (int)blockIdx.x - rows_blocks, reinterpret_cast<char*>(stage0));
      return;
    }
  if constexpr (ROWS) rows_block8<DH, TABLE>(pl, a, exps, blockIdx.x, stage0, stage1);
}

// ---------------------------------------------------------------------------
// fp32 queries of one row on a key head, at most 4 of them (single_row).  The 4 x 4 MFMA takes 16 independent products at a time: lane
// 4 b + i brings key i of the block's 4 (a wave's 64) and query i, and gets its query's scores with the 4 keys.  Those are
// just what the product with V takes, a key of each block at a time, lane 4 b + i bringing a quarter of the head dims of its
// V row; so each lane has a softmax of its own until the end, and nothing is exchanged before it.
// K of the next tile is loaded once the scores have taken this one's, V once the products have.
// 64 rows after 2000 keys, 16 heads of 64: 61 us, 4.3 TB/s (16 x 16 x 4 products, 15 of 16 of them for nothing: 100); of 128 123
// and 182; 8 rows after 30000, 32 heads of 128 on 8, 122 and 166.  Bound by its products and conversions; with head dim 64 three
// blocks share a CU, four of them spill (66).
// ---------------------------------------------------------------------------
template <int DH>
__device__ __forceinline__ void single_row8(const PagedAttn& a, const uint8_t* __restrict__ exps, page_row prow, const uint8_t* kh, const uint8_t* vh,
                                            const float* q, int h, const Vis& vis, int t0, int t1, int jq, float* sq,
                                            float (*sm)[16], float (*sl)[16], float (*so)[16][DH]) {
  constexpr int NV = DH / 4, KL = DH / 16, VL = DH / 64, QS = DH + 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j = lane & 3, lp = a.kp.log2_page;
  auto mfma = [](float p, float q, const f32x4& c) { return __builtin_amdgcn_mfma_f32_4x4x1f32(p, q, c, 0, 0, 0); };
  for (int i = tid; i < DH; i += 256) {                   // queries past the group's: copies of its last
    const int r = i / (DH / 4), d = i % (DH / 4) * 4;
    *reinterpret_cast<f32x4*>(sq + r * QS + d) = *reinterpret_cast<const f32x4*>(q + min(r, a.G - 1) * DH + d);
  }
  __syncthreads();
  f32x4 o[NV];
#pragma unroll
  for (int c = 0; c < NV; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = LOWEST, l_run = 0.f;
  // the slot of the lane's key of the 4 runs from run t on; runs past the last re-read it, unseen
  auto slot_of = [&](int t) {
    const int k = 16 * vis.run(min(t + (lane >> 4), t1 - 1));
    return (prow[k >> lp] << lp) + (k & ((1 << lp) - 1)) + (lane & 15);
  };
  u32x4 kc[KL], vc[4][VL];
  uint32_t ex;
  auto load_k = [&](int slot) {
    ex = reinterpret_cast<const uint16_t*>(exps)[(int64_t)(slot >> 4) * a.KH + h];
    const uint8_t* r = kh + (int64_t)slot * DH;
#pragma unroll
    for (int c = 0; c < KL; ++c) kc[c] = *reinterpret_cast<const u32x4*>(r + 16 * c);
  };
  auto load_v = [&](int slot) {
    const uint8_t* r = vh + (int64_t)(slot - j) * DH + j * (DH / 4);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < VL; ++c) vc[i][c] = *reinterpret_cast<const u32x4*>(r + i * DH + 16 * c);
  };
  int t = t0 + 4 * wave;
  if (t < t1) {
    int slot = slot_of(t);
    load_k(slot);
    load_v(slot);
    slot = slot_of(t + 16);
    for (; t < t1; t += 16) {
      f32x4 s2[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      const float kscale = scale_of(ex & 0xFF);
      float vscale = scale_of(ex >> 8);
      int at = j * QS;
      asm volatile("" : "+v"(at));                        // the queries are read anew, not held over the loop
#pragma unroll
      for (int c = 0; c < KL; ++c)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const f32x4 kf = decode4(kc[c][w], kscale), qf = *reinterpret_cast<const f32x4*>(sq + at + 16 * c + 4 * w);
#pragma unroll
          for (int e = 0; e < 4; ++e) s2[w & 1] = mfma(kf[e], qf[e], s2[w & 1]);
        }
      if (t + 16 < t1) load_k(slot);
      f32x4 s = s2[0] + s2[1];
      // the block's 4 keys
      const int run = t + (lane >> 4), k0 = 16 * vis.run(min(run, t1 - 1)) + (lane & 12);
      bool see[4], all = true, any = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        see[i] = run < t1 && sees(jq, k0 + i, a.window, a.n_sink);
        all = all && see[i];
        any = any || see[i];
      }
      if (__any(!all)) {
        if (!any) vscale = 1.f;                           // of a run that may have none
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[i] = see[i] ? s[i] : -INFINITY;
#pragma unroll
          for (int c = 0; c < VL; ++c) vc[i][c] = see[i] ? vc[i][c] : u32x4{};
        }
      }
      const float mb = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
      if (__any(mb > m_run)) {
        const float m_new = fmaxf(m_run, mb), alpha = exp2f((m_run - m_new) * a.scale_log2);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int c = 0; c < NV; ++c) o[c] *= alpha;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = exp2f((s[i] - m_run) * a.scale_log2);
        l_run += e;
#pragma unroll
        for (int c = 0; c < NV; c += 4) {
          const f32x4 v = decode4(vc[i][c / 16][c / 4 % 4], vscale);
#pragma unroll
          for (int d = 0; d < 4; ++d) o[c + d] = mfma(v[d], e, o[c + d]);
        }
      }
      if (t + 16 < t1) { load_v(slot); slot = slot_of(t + 32); }
    }
  }
  // the 16 blocks' softmaxes as one; of the outputs, each lane keeps half of what it and its partner hold
  float M = m_run;
#pragma unroll
  for (int x = 4; x < 64; x <<= 1) M = fmaxf(M, __shfl_xor(M, x, 64));
  const float wt = exp2f((m_run - M) * a.scale_log2);
  l_run *= wt;
#pragma unroll
  for (int x = 4; x < 64; x <<= 1) l_run += __shfl_xor(l_run, x, 64);
#pragma unroll
  for (int c = 0; c < NV; ++c) o[c] *= wt;
  int c0 = 0;
#pragma unroll
  for (int x = 32, n = NV / 2; x >= 4; x >>= 1, n >>= 1) {
    const bool upper = lane & x;
    c0 += upper ? n : 0;
#pragma unroll
    for (int c = 0; c < n; ++c) {
      f32x4 mine = upper ? o[c + n] : o[c], other = upper ? o[c] : o[c + n];
#pragma unroll
      for (int i = 0; i < 4; ++i) mine[i] += __shfl_xor(other[i], x, 64);
      o[c] = mine;
    }
  }
#pragma unroll
  for (int c = 0; c < NV / 16; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) so[wave][j][NV * i + c0 + c] = o[c][i];
  if (lane < 4) { sm[wave][j] = M; sl[wave][j] = l_run; }
}

// ---------------------------------------------------------------------------
// Other fp32 queries, any number of rows: as the fp32 cache's kernel (k_paged.hip), the codes made fp32 in registers.  A lane
// loads 16 consecutive head dims of its key's K row (its queries' registers hold the same ones), and DH / 16 consecutive
// ones of V rows, which give as many MFMAs a row each.  8 chunks of 512 rows after 1000, 16 heads of 64, take 231 to 237 us,
// 91 TFLOP/s of visible products (a large matrix product: 154): the matrix cores are busy for 60% of the cycles and the
// vector ALU for 37, by turns (each wave converts its own K and V); of 128 439 us, 64 and 31.
// SINGLE, OTHER: which requests the step has.  With both, all blocks have the single rows' registers (head dim 64: 134 for 85, 128:
// 232 for 141): one single row beside those chunks makes 237 us 240 and 439 464.
// ---------------------------------------------------------------------------
template <int DH, bool SINGLE, bool OTHER, bool TABLE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void attn8_f32_kernel(
    Plan pl, PagedAttn a, const uint8_t* __restrict__ exps) {
  constexpr int NC = DH / 16, KL = DH / 64, NV = DH / 16;
  __shared__ float sm[4][16], sl[4][16];
  __shared__ __attribute__((aligned(16))) float so[4][16][DH];
  auto mfma = [](float p, float q, const f32x4& c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(p, q, c, 0, 0, 0); };
  Work w;
  int id = blockIdx.x;
  if constexpr (TABLE) {
    const table_t parts = table_of(pl, a, TAB_FEW);
    w.p = last_request(pl.n_req, id, [&](int p) { return parts[p]; });
    id -= parts[w.p];
  } else {
    w.h = id % a.KH; id /= a.KH;
    w.c = id % a.few_chunks; id /= a.few_chunks;
    // request p's query tiles start at cu[p] G / 16 + p
    auto begin = [&](int p) { return (int)((int64_t)pl.cu_seqlens[p] * a.G / 16 + p); };
    w.p = last_request(pl.n_req, id, begin);
    w.qt = id - uniform(begin(w.p));
  }
  const int R0 = uniform(pl.cu_seqlens[w.p]), m = uniform(pl.cu_seqlens[w.p + 1]) - R0, ctx = uniform(pl.ctx[w.p]);
  const int request = uniform(pl.order[w.p]);            // with them, not behind what they decide
  const int qn = m * a.G;
  if (!TABLE && w.qt * 16 >= qn) return;      // block-uniform, as every exit below
  const Chunks ck = request_chunks(VFM_F32, m, ctx, a.G, a.KH, a.window, a.n_sink, true);
  if constexpr (TABLE) {
    w.h = id % a.KH; id /= a.KH;
    w.c = id % ck.n;
    w.qt = id / ck.n;
  } else if (w.c >= ck.n) {
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j0 = ctx + w.qt * 16 / a.G, j1 = ctx + min(w.qt * 16 + 15, qn - 1) / a.G;
  // the tile's own runs, dealt over the request's chunks
  const Vis vis = visible_runs<4>(j0, j1, a.window, a.n_sink);
  const int rpc = (vis.n + ck.n - 1) / ck.n;
  const int t0 = w.c * rpc, t1 = min(t0 + rpc, vis.n);
  const page_row prow = row_of(a.kp, request);
  const int lp = a.kp.log2_page;
  const uint8_t* kh = (const uint8_t*)a.k + (int64_t)w.h * a.slots * DH;
  const uint8_t* vh = (const uint8_t*)a.v + (int64_t)w.h * a.slots * DH;
  if (SINGLE && (!OTHER || single_row(m, a.G, vis.n))) {         // block-uniform
    int head;
    const int64_t row = out_row(a, R0, w.h, 0, head);
    __shared__ __attribute__((aligned(16))) float sq[4 * (DH + 4)];
    single_row8<DH>(a, exps, prow, kh, vh, (const float*)a.q + row * a.ldq + head * DH, w.h, vis, t0, t1, j0, sq, sm, sl, so);
  } else if constexpr (OTHER) {
    const int x = lane & 15, g = lane >> 4;
    const int qi = min(w.qt * 16 + x, qn - 1);
    const int jq = ctx + qi / a.G;
    int head;
    const int64_t row = out_row(a, R0, w.h, qi, head);
    f32x4 q[NC], o[NV];
#pragma unroll
    for (int c = 0; c < NC; ++c)
      q[c] = *reinterpret_cast<const f32x4*>((const float*)a.q + row * a.ldq + head * DH + 64 * (c >> 2) + 16 * g + 4 * (c & 3));
#pragma unroll
    for (int c = 0; c < NV; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = LOWEST, l_run = 0.f;
    // a run's codes, loaded while the one before is computed
    struct Run {
      int slot;
      uint32_t ex, vc[4][NV / 4];
      u32x4 kc[KL];
    } next;
    auto load = [&](int t) {
      const int slot = page_slot(prow, lp, 16 * vis.run(t));
      next.slot = slot;
      next.ex = runs_exps(exps, slot, slot, a.KH, w.h);
      const uint8_t *kr = kh + (int64_t)slot * DH, *vr = vh + (int64_t)slot * DH;
#pragma unroll
      for (int c = 0; c < KL; ++c) next.kc[c] = *reinterpret_cast<const u32x4*>(kr + (x * DH + 64 * c + 16 * g));
#pragma unroll
      for (int j = 0; j < 4; ++j) __builtin_memcpy(next.vc[j], __builtin_assume_aligned(vr + ((4 * g + j) * DH + NV * x), NV), NV);
    };
    if (t0 + wave < t1) load(t0 + wave);
    for (int t = t0 + wave; t < t1; t += 4) {
      const int p0 = 16 * vis.run(t);
      const bool full = seen_by_all(j0, j1, p0, p0 + 15, a.window, a.n_sink);
      const Run now = next;
      if (t + 4 < t1) load(t + 4);
      const int64_t slot = now.slot;
      const u32x4(&kc)[KL] = now.kc;
      const uint32_t(&vc)[4][NV / 4] = now.vc;
      const float kscale = k_scale(now.ex, 0), vscale = v_scale(now.ex, 0);
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const f32x4 kf = decode4(kc[c >> 2][c & 3], kscale);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = mfma(kf[e], q[c][e], s);
      }
      f32x4 vf[4][NV / 4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int c = 0; c < NV / 4; ++c) vf[j][c] = decode4(vc[j][c], vscale);
      bool poison = false;
      if (!full) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int k = p0 + 4 * g + j;
          s[j] = sees(jq, k, a.window, a.n_sink) ? s[j] : -INFINITY;
          const bool any = seen_by_any(j0, j1, k, a.window, a.n_sink);
          const bool some = any && !seen_by_all(j0, j1, k, k, a.window, a.n_sink);
#pragma unroll
          for (int c = 0; c < NV; ++c) {
            const bool bad = some && nonfinite(vf[j][c >> 2][c & 3]);
            poison = poison || bad;
            vf[j][c >> 2][c & 3] = !any || bad ? 0.f : vf[j][c >> 2][c & 3];
          }
        }
      }
      float mb = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
      mb = max_x32(max_x16(mb));
      const float m_new = fmaxf(m_run, mb);
      const float alpha = exp2f((m_run - m_new) * a.scale_log2);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int c = 0; c < NV; ++c) o[c] *= alpha;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = exp2f((s[j] - m_run) * a.scale_log2);
        l_run += e;
#pragma unroll
        for (int c = 0; c < NV; ++c) o[c] = mfma(vf[j][c >> 2][c & 3], e, o[c]);
      }
      if (__any(poison)) {                                  // rare: see the bf16 kernel
        for (int r = 0; r < 16; ++r) {
          const int k = p0 + r;
          if (!seen_by_any(j0, j1, k, a.window, a.n_sink) || seen_by_all(j0, j1, k, k, a.window, a.n_sink)) continue;
          const bool see = sees(jq, k, a.window, a.n_sink);
#pragma unroll
          for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (see && is_nan8(vh[(slot + r) * DH + NV * (4 * g + i) + c])) o[c][i] = NAN;
        }
      }
    }
    l_run = sum_x32(sum_x16(l_run));
    if (lane < 16) { sm[wave][x] = m_run; sl[wave][x] = l_run; }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < NV; c += 4)
        *reinterpret_cast<f32x4*>(&so[wave][x][NV * (4 * g + i) + c]) = f32x4{o[c][i], o[c + 1][i], o[c + 2][i], o[c + 3][i]};
  }
  __syncthreads();
  const int nq = min(16, qn - w.qt * 16);
  for (int e = tid; e < nq * DH / 4; e += 256) {
    const int qq = e / (DH / 4), d = (e % (DH / 4)) * 4;
    const float M = fmaxf(fmaxf(sm[0][qq], sm[1][qq]), fmaxf(sm[2][qq], sm[3][qq]));
    float L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float wt = exp2f((sm[i][qq] - M) * a.scale_log2);
      L += sl[i][qq] * wt;
      acc += *reinterpret_cast<const f32x4*>(&so[i][qq][d]) * wt;
    }
    int hd;
    const int64_t r = out_row(a, R0, w.h, w.qt * 16 + qq, hd);
    if (ck.n == 1) {
      *reinterpret_cast<f32x4*>((float*)a.out + r * a.ldo + hd * DH + d) = acc / L;
    } else {
      const int64_t rec = record_of<TABLE>(pl, a, w.p, R0, ck.n, r, hd) + w.c;
      *reinterpret_cast<f32x4*>(a.rec_o + rec * DH + d) = acc;
      if (d == 0) a.rec_ml[rec] = make_float2(M, L);
    }
  }
}

template <int DH, bool TABLE>
void launch_blocks8(int dtype, const Plan& pl, const PagedAttn& a, const uint8_t* exps, unsigned nf, unsigned nr, bool deep, bool single, bool other, hipStream_t s) {
  const dim3 block(256), grid(nf + nr);
#define F32(S_, O_) hipLaunchKernelGGL((attn8_f32_kernel<DH, S_, O_, TABLE>), grid, block, 0, s, pl, a, exps)
  if (dtype != VFM_BF16) { if (!single) F32(false, true); else if (other) F32(true, true); else F32(true, false); }
#undef F32
#define BF16(R_, N_, W_) hipLaunchKernelGGL((attn8_bf16_kernel<DH, R_, N_, W_, TABLE>), grid, block, 0, s, pl, a, exps, (int)nr)
  else if (nr && nf) BF16(true, 2, 2);
  else if (nr) BF16(true, 0, 2);
  else if (deep) BF16(false, (DH == 64 ? 2 : 3), (DH == 64 ? 3 : 2));
  else BF16(false, 1, (DH == 64 ? 5 : 4));
#undef BF16
}

}  // namespace

hipError_t launch_append8(int dtype, const Plan& pl, int H, int KH, int head_dim, float theta, const void* qkv, int64_t ld,
                          void* q_out, int64_t ldq, const Pool8& pool, const KvPages& kp, hipStream_t s) {
  Append8 a = {};
  a.H = H; a.KH = KH; a.rotate = theta > 0.f; a.log2_theta = theta > 0.f ? log2((double)theta) : 0.0;
  a.ld = ld; a.ldq = ldq; a.slots = pool.slots; a.k = pool.k; a.v = pool.v; a.exps = pool.exps; a.kp = kp;
  // single rows: a wave has 64 / (head_dim / 16) heads at a time, otherwise one
  const int n_heads = H + 2 * KH, units = pl.max_seqlen > 1 ? n_heads : (n_heads + 1024 / head_dim - 1) / (1024 / head_dim);
  const int blocks = pl.n_req + (pl.max_seqlen > 1 ? (pl.T + 15) / 16 : 0);
  // A wave takes 4 heads of a run, so that the blocks come to several rounds over the chip and the last one is short; where
  // blocks are few, less: up to 1024 blocks are resident.  (Each share takes the run's angles anew.)
  const int most = (units + 3) / 4;
  int split = (units + 15) / 16;
  if ((int64_t)blocks * split < 1024) split = (1024 + blocks - 1) / blocks;
  if (split > most) split = most;
  if (split > APPEND8_MAX_BLOCKS / blocks) split = APPEND8_MAX_BLOCKS / blocks;
  a.split = split;
#define APPEND(T_, D_)                                                                                             \
  hipLaunchKernelGGL((append8_kernel<T_, D_>), dim3((unsigned)(blocks * a.split)), dim3(256), 0, s, pl, a, (const T_*)qkv, (T_*)q_out)
  if (dtype == VFM_BF16) { if (head_dim == 64) APPEND(bf16, 64); else APPEND(bf16, 128); }
  else { if (head_dim == 64) APPEND(float, 64); else APPEND(float, 128); }
#undef APPEND
  return hipGetLastError();
}

hipError_t launch_attention8(int dtype, int head_dim, const Plan& pl, const PagedAttn& a, const uint8_t* exps, int64_t few_blocks,
                             int64_t rows_blocks, int64_t joins, bool deep, bool single, bool other, bool table, hipStream_t s) {
  if (table) launch_attention_table(dtype, pl, a, s);
  const int pi = prof_begin(VFM_PROF_ATTN, s);
  const unsigned nf = (unsigned)few_blocks, nr = (unsigned)rows_blocks;
  if (head_dim == 64) {
    if (table) launch_blocks8<64, true>(dtype, pl, a, exps, nf, nr, deep, single, other, s);
    else launch_blocks8<64, false>(dtype, pl, a, exps, nf, nr, deep, single, other, s);
  } else if (table) {
    launch_blocks8<128, true>(dtype, pl, a, exps, nf, nr, deep, single, other, s);
  } else {
    launch_blocks8<128, false>(dtype, pl, a, exps, nf, nr, deep, single, other, s);
  }
  prof_end(pi, s);
  if (joins) launch_attention_joins(dtype, head_dim, pl, a, (int)joins, table, s);
  return hipGetLastError();
}
