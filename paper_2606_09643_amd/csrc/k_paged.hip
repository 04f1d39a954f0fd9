// Appending to a paged KV cache and attention of new rows over it, with a
// sliding window and first tokens that stay visible, for any number of query
// heads per key head.
//
// A request's m rows times the G query heads of one key head are its packed
// queries (row-major: neighbours share the row, so a tile's queries see nearly
// the same keys); all of them read the same K and V.  Every kernel computes
// S^T = K Q^T, keys in the MFMA's A slot and packed queries in the B slot, so
// a lane holds several keys of ONE query: the softmax's maximum and sum are
// in-lane plus one or two lane swaps, and exp(S^T) already lies as the B operand
// of O^T = V^T P^T.
//
// A weight is 2^((s - m) scale), m the running maximum of the scores s as they are: with s scale
// rounded for m alone, a score of 2^33 would leave a rest of hundreds in the exponent.  The difference is
// 0 for the largest score whatever its size, so every finite score has its weight.  m starts at the
// lowest number; sums of nothing (and their weight in a merge) are 0 beside any m.
//
// Unseen keys.  Scores of unseen keys become -inf by a select, so what K holds
// there does not matter.  V rows that no query of the tile sees are staged as
// zeros.  Where some queries of a tile see a key and others do not, a zero
// weight would still turn an infinity or a NaN of its V row into a NaN: such
// tiles look for those values while staging, put zeros in their place and add
// them afterwards to the queries that see them (add_nonfinite below).
#include <type_traits>

#include "decode_internal.h"

namespace {

constexpr float LOWEST = -3.40282347e38f;   // below or at every finite score

typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 2^x, x <= 0 or -inf: the hardware exponential (1 ulp; no range reduction)
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ bf16x8 pack8(float a, float b, float c, float d, float e, float f, float g, float h) {
  const bf16x2 p0 = __builtin_convertvector(f32x2{a, b}, bf16x2), p1 = __builtin_convertvector(f32x2{c, d}, bf16x2);
  const bf16x2 p2 = __builtin_convertvector(f32x2{e, f}, bf16x2), p3 = __builtin_convertvector(f32x2{g, h}, bf16x2);
  const bf16x4 lo = __builtin_shufflevector(p0, p1, 0, 1, 2, 3), hi = __builtin_shufflevector(p2, p3, 0, 1, 2, 3);
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// v of lane ^ 32 and of lane ^ 16 combined with the lane's own (gfx950 lane swaps)
__device__ __forceinline__ float max_x32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_x16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_x32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum_x16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// v combined over the 16 lanes of a row (rotations within it), in every lane
template <int CTRL>
__device__ __forceinline__ float rotated(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float max_row(float v) {
  v = fmaxf(v, rotated<0x128>(v));
  v = fmaxf(v, rotated<0x124>(v));
  v = fmaxf(v, rotated<0x122>(v));
  return fmaxf(v, rotated<0x121>(v));
}
__device__ __forceinline__ float sum_row(float v) {
  v += rotated<0x128>(v);
  v += rotated<0x124>(v);
  v += rotated<0x122>(v);
  return v + rotated<0x121>(v);
}

// A wave's own LDS accesses complete in order; only the compiler must keep them.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// whether the row at position j sees position k
__device__ __forceinline__ bool sees(int j, int k, int window, int n_sink) {
  return k <= j && (window == 0 || j - k < window || k < n_sink);
}
// whether any of the rows at positions j0 .. j1 sees position k
__device__ __forceinline__ bool seen_by_any(int j0, int j1, int k, int window, int n_sink) {
  return k <= j1 && (window == 0 || j0 - k < window || k < n_sink);
}
// whether all of them see every position of [k0, k1]
__device__ __forceinline__ bool seen_by_all(int j0, int j1, int k0, int k1, int window, int n_sink) {
  return k1 <= j0 && (window == 0 || j1 - k0 < window || k1 < n_sink);
}

// bf16 pairs with an infinity or a NaN replaced by zeros; `found` is set if any
__device__ __forceinline__ bf16x8 drop_nonfinite(const bf16x8& v, bool& found) {
  u32x4 w;
  __builtin_memcpy(&w, &v, 16);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (w[i] & 0x7F80u) == 0x7F80u, hi = (w[i] & 0x7F800000u) == 0x7F800000u;
    found = found || lo || hi;
    w[i] &= (lo ? 0xFFFF0000u : 0xFFFFFFFFu) & (hi ? 0x0000FFFFu : 0xFFFFFFFFu);
  }
  bf16x8 r;
  __builtin_memcpy(&r, &w, 16);
  return r;
}
__device__ __forceinline__ bool nonfinite(float v) { return !(fabsf(v) < INFINITY); }

// A value that every lane of the wave holds, as a scalar.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A request's page row.  Nothing writes it during the kernel: positions that are
// uniform over a wave are looked up with scalar loads, beside the vector loads
// that are in flight.
typedef const int32_t __attribute__((address_space(4)))* page_row;
__device__ __forceinline__ page_row row_of(const KvPages& kp, int request) {
  return (page_row)(uintptr_t)(kp.table + (int64_t)request * kp.max_pages);
}
// Slot of position k.
__device__ __forceinline__ int page_slot(page_row prow, int lp, int k) {
  return (prow[k >> lp] << lp) + (k & ((1 << lp) - 1));
}

// ---------------------------------------------------------------------------
// Append: rotate-half of the q and k heads, q to q_out, k and v to their slots.
// One block per row; a thread takes 8 pairs (i, i + dh/2) of one head with
// 16-byte accesses (32 for fp32) and writes them after it has read both halves,
// so q_out may be the queries' own place.  Bound by its bytes: every element is read and
// written once.  The row's dh/2 angles go through LDS: revolutions in fp64
// (position times theta^(-2i/dh) / 2 pi loses nothing up to 2^30 positions),
// their fraction in fp32.
// 32 prompts of 128 to 1024 tokens, 32 heads of 128 on 32: 178 us, 5.2 TB/s (a
// copy of 2 GiB runs at 4.95).  Blocks of 8 rows by 12 heads, which write longer
// runs into a page, take the same.  One row: 2.8 us by kernel trace, all latency.
// ---------------------------------------------------------------------------
template <typename T> struct Vec8;
template <> struct Vec8<bf16> { bf16x8 v; };
template <> struct Vec8<float> { f32x4 v[2]; };
__device__ __forceinline__ float get(const Vec8<bf16>& x, int i) { return (float)x.v[i]; }
__device__ __forceinline__ float get(const Vec8<float>& x, int i) { return x.v[i >> 2][i & 3]; }
__device__ __forceinline__ void put(Vec8<bf16>& x, int i, float f) { x.v[i] = (bf16)f; }
__device__ __forceinline__ void put(Vec8<float>& x, int i, float f) { x.v[i >> 2][i & 3] = f; }

template <typename T, int DH>
__global__ __launch_bounds__(APPEND_THREADS) void kv_append_kernel(Plan pl, int H, int KH, int rotate, double log2_theta,
                                                        const T* qkv, int64_t ld, T* q_out, int64_t ldq,
                                                        T* __restrict__ kc, T* __restrict__ vc, int64_t slots,
                                                        KvPages kp) {
  constexpr int HALF = DH / 2, PER = HALF / 8;
  __shared__ float cs[HALF], sn[HALF];
  const int r = blockIdx.x;
  const int pos = pl.pos[r];
  if (rotate && (int)threadIdx.x < HALF) {
    const double inv = exp2(-(2.0 * (double)threadIdx.x / (double)DH) * log2_theta) * 0.15915494309189535;
    const double rev = (double)pos * inv;
    float s, c;
    sincospif((float)(2.0 * (rev - rint(rev))), &s, &c);
    cs[threadIdx.x] = c;
    sn[threadIdx.x] = s;
  }
  const int64_t slot = kv_slot(pl, kp, pl.row_req[r], pos);
  __syncthreads();
  const T* row = qkv + (int64_t)r * ld;
  const int first = q_out != nullptr ? 0 : H * PER;
  for (int w = first + threadIdx.x; w < (H + 2 * KH) * PER; w += APPEND_THREADS) {
    const int hh = w / PER, i0 = (w % PER) * 8;
    Vec8<T> a = *reinterpret_cast<const Vec8<T>*>(row + hh * DH + i0);
    Vec8<T> b = *reinterpret_cast<const Vec8<T>*>(row + hh * DH + HALF + i0);
    if (rotate && hh < H + KH) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = get(a, j), y = get(b, j), c = cs[i0 + j], s = sn[i0 + j];
        put(a, j, x * c - y * s);
        put(b, j, x * s + y * c);
      }
    }
    T* dst = hh < H ? q_out + (int64_t)r * ldq + hh * DH
                    : (hh < H + KH ? kc + ((int64_t)(hh - H) * slots + slot) * DH
                                   : vc + ((int64_t)(hh - H - KH) * slots + slot) * DH);
    *reinterpret_cast<Vec8<T>*>(dst + i0) = a;
    *reinterpret_cast<Vec8<T>*>(dst + HALF + i0) = b;
  }
}

// ---------------------------------------------------------------------------
// Where a block of the attention kernels works.
// ---------------------------------------------------------------------------
struct Work {
  int h, c, qt, p;    // key head, chunk, query tile, plan position
};

// The table's sum `which` (it is written by a kernel before this one).
typedef const int32_t __attribute__((address_space(4)))* table_t;
__device__ __forceinline__ table_t table_of(const Plan& pl, const PagedAttn& a, int which) {
  return (table_t)(uintptr_t)(a.table + (int64_t)which * (pl.n_req + 1));
}
// The request that place id of a sum falls to, the last one whose part begins at or before it; id becomes the place
// in its part.
__device__ __forceinline__ int request_at(table_t t, int n_req, int& id) {
  int lo = 0, hi = n_req - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t[mid] <= id) lo = mid; else hi = mid - 1;
  }
  id -= t[lo];
  return lo;
}
// The first record of a row and head, in a request p whose rows begin at R0 and whose keys are cut in n.
template <bool TABLE>
__device__ __forceinline__ int64_t record_of(const Plan& pl, const PagedAttn& a, int p, int R0, int n, int64_t row,
                                             int head) {
  if constexpr (TABLE) return table_of(pl, a, TAB_RECS)[p] + ((row - R0) * a.H + head) * n;
  else return (row * a.H + head) * a.nchunk;
}

// Output of packed query `qi` (of the request's first row R0): the row's head.
__device__ __forceinline__ int64_t out_row(const PagedAttn& a, int R0, int h, int qi, int& head) {
  const int i = qi / a.G;
  head = h * a.G + (qi - i * a.G);
  return (int64_t)R0 + i;
}

// ---------------------------------------------------------------------------
// Few rows (decode and short chunks), bf16: one block per 16 packed queries of
// one request and key head and chunk of its keys; each of the 4 waves streams
// every 4th 32-key tile of the chunk on its own (no barrier in the loop) and
// the waves' partial softmax sums are merged through LDS at the end.
// Memory bound: each visible K / V row is read once per query tile.  K fragments
// go straight to registers (lane: one key's row, 16 bytes per MFMA step), V
// through a wave-private LDS tile that the transposing LDS read turns into the
// V^T operand; a tile's loads are issued while the tile before is computed, which
// takes half the registers (see SINGLE below for where it does not pay).
// A weight is rounded to bf16, by at most 2^-8 of itself, for the product alone; the
// sum that divides is of the weights as they are, which costs nothing here.
// 256 requests with up to 1028 visible keys, 32 heads of 128 on 32: 598 us, 6.3
// TB/s; 8 requests of 32768 to 131072, 32 heads on 8: 388 us, 6.5 TB/s.  One row
// after 300 keys: 8.9 us, the latency of a few dependent loads.
// ---------------------------------------------------------------------------
__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// V rows of a few-row tile lie in LDS as [32][DH], their segments swizzled by vswz.

// smem: 256 DH bytes, V tiles, then the waves' outputs.  SINGLE: one tile at a time in registers, with head dim
// 128 the wave's only one.
template <int DH, bool SINGLE, bool TABLE>
__device__ __forceinline__ void few_block(const Plan& pl, const PagedAttn& a, int id, char* smem) {
  constexpr int LPR = DH / 8;          // lanes per K / V row (16 bytes each)
  constexpr int RPI = 64 / LPR;        // rows per wave-wide load
  constexpr int VI = 32 / RPI;         // V loads per lane and tile
  constexpr int KS = DH / 32;          // MFMA steps over the head dims
  constexpr int ND = DH / 16;          // output tiles
  __shared__ float sm[4][16], sl[4][16];

  Work w;
  if constexpr (TABLE) {
    w.p = request_at(table_of(pl, a, TAB_FEW), pl.n_req, id);
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
  const Chunks ck = request_chunks(VFM_BF16, m, ctx, a.G, a.KH, a.window, a.n_sink);
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
  // this lane's query; the tile's rows' positions
  const int qi = min(w.qt * 16 + x, qn - 1);
  const int jq = ctx + qi / a.G;
  const int j0 = ctx + w.qt * 16 / a.G, j1 = ctx + min(w.qt * 16 + 15, qn - 1) / a.G;
  int head;
  const int64_t row = out_row(a, R0, w.h, qi, head);
  bf16x8 qf[KS];
  {
    const bf16* qr = (const bf16*)a.q + row * a.ldq + head * DH + 8 * g;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qr + 32 * s);
  }
  const page_row prow = row_of(a.kp, request);
  const int lp = a.kp.log2_page;
  const bf16* kh = (const bf16*)a.k + (int64_t)w.h * a.slots * DH;
  const bf16* vh = (const bf16*)a.v + (int64_t)w.h * a.slots * DH;
  bf16* Vs = reinterpret_cast<bf16*>(smem) + wave * 32 * DH;

  // positions and slots of a tile's two 16-position runs (one page each, as a
  // page holds a multiple of 16); runs past the last re-read it, unseen
  auto run_pos = [&](int t, int e) { return 16 * vis.run(min(2 * t + e, vis.n - 1)); };
  bf16x8 kf[2][2][KS], vf[2][VI];
  int slot[2];
  auto look_up = [&](int t) {
    slot[0] = page_slot(prow, lp, run_pos(t, 0));
    slot[1] = page_slot(prow, lp, run_pos(t, 1));
  };
  // keys of sub-tile e in rows x: 8 (x / 4) + x % 4 + 4 e, so that after the MFMA
  // a lane holds the 8 consecutive keys 8 g .. 8 g + 7 over both sub-tiles
  const int key0 = 8 * (x >> 2) + (x & 3);
  auto load = [&](int b) {
    const int64_t ks = (int64_t)(x < 8 ? slot[0] : slot[1]) + (key0 & 15);
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int s = 0; s < KS; ++s)
        kf[b][e][s] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(kh + (ks + 4 * e) * DH + 8 * g + 32 * s));
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      const int64_t vs = (int64_t)slot[(RPI * i) >> 4] + ((RPI * i) & 15) + lane / LPR;
      vf[b][i] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(vh + vs * DH + 8 * (lane % LPR)));
    }
  };

  f32x4 o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = LOWEST, l_run = 0.f;

  const int vst_ch = lane % LPR, vst_row = lane / LPR;
  const int vrow = 8 * g + (x >> 2);
  const int vbase = vrow * DH * 2 + (vswz<DH>(vrow) << 5) + (x & 3) * 8;

  auto compute = [&](int b, int t) {
    const int p0 = run_pos(t, 0);
    const int p1 = 2 * t + 1 < vis.n ? run_pos(t, 1) : INT32_MAX - 64;   // no second run: unseen
    const bool full = p1 == p0 + 16 && seen_by_all(j0, j1, p0, p0 + 31, a.window, a.n_sink);
    bool poison = false;
    // V to LDS
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      const int r = RPI * i + vst_row;
      bf16x8 v = vf[b][i];
      if (!full) {
        const int k = (((RPI * i) >> 4) ? p1 : p0) + (r & 15);
        if (!seen_by_any(j0, j1, k, a.window, a.n_sink)) v = bf16x8{};
        else if (j0 != j1 && !seen_by_all(j0, j1, k, k, a.window, a.n_sink)) v = drop_nonfinite(v, poison);
      }
      *reinterpret_cast<bf16x8*>(Vs + r * DH + ((((vst_ch >> 1) ^ vswz<DH>(r)) << 1) | (vst_ch & 1)) * 8) = v;
    }
    wave_lds_order();
    // S^T
    float s[8];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < KS; ++st) acc = mfma16(kf[b][e][st], qf[st], acc);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * e + i] = acc[i];
    }
    if (!full) {
      const int kb = (g < 2 ? p0 : p1) + 8 * (g & 1);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] = sees(jq, kb + i, a.window, a.n_sink) ? s[i] : -INFINITY;
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
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      const char* vp = reinterpret_cast<const char*>(Vs) + (vbase ^ (d << 5));
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vp));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vp + 4 * DH * 2));
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
        const bf16* vr = vh + (int64_t)page_slot(prow, lp, k) * DH + 4 * g;
        const bool see = sees(jq, k, a.window, a.n_sink);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float v = (float)vr[16 * d + i];
            if (see && nonfinite(v)) o[d][i] += v;
          }
          __builtin_amdgcn_sched_barrier(0);              // no registers for more loads in flight
        }
      }
    }
  };

  // tiles t0 + wave, + 4, ...: one at a time, its page lookups a tile ahead, or (not SINGLE) a tile's loads
  // in flight while the one before is computed, its page lookups a tile before that
  int t = t0 + wave;
  if (t < t1) {
    look_up(t);
    if constexpr (SINGLE && DH == 128) {                  // the caller has seen that there is no other
      load(0);
      compute(0, t);
    } else if constexpr (SINGLE) {
      for (; t < t1; t += 4) {
        load(0);
        if (t + 4 < t1) look_up(t + 4);
        compute(0, t);
      }
    } else {
      load(0);
      if (t + 4 < t1) look_up(t + 4);
      for (;;) {
        if (t + 4 < t1) { load(1); if (t + 8 < t1) look_up(t + 8); }
        compute(0, t);
        t += 4;
        if (t >= t1) break;
        if (t + 4 < t1) { load(0); if (t + 8 < t1) look_up(t + 8); }
        compute(1, t);
        t += 4;
        if (t >= t1) break;
      }
    }
  }
  l_run = sum_x32(sum_x16(l_run));

  // merge the four waves
  __syncthreads();
  float* so = reinterpret_cast<float*>(smem);             // [4][16][DH]
  if (lane < 16) { sm[wave][x] = m_run; sl[wave][x] = l_run; }
  // all 16 queries, those past the last (copies of it) among them: their outputs lie at wave, query, dim
#pragma unroll
  for (int d = 0; d < ND; ++d)
    *reinterpret_cast<f32x4*>(so + (wave * 16 + x) * DH + 16 * d + 4 * g) = o[d];
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
      acc += *reinterpret_cast<const f32x4*>(so + (i * 16 + q) * DH + d) * wt;
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
// Many rows (prompts and chunks), bf16: one block per 128 packed queries of one
// request and key head (and chunk of the keys where the request has few blocks);
// waves of 32 queries on v_mfma_f32_32x32x16_bf16, so a K or V fragment read from
// LDS feeds 32 queries.  64-key tiles of K and V go from memory straight into two
// LDS stages by turns (global_load_lds, one barrier per tile).  A wave-wide load
// takes whole rows of one 16-position run, whose page it looks up as a scalar, a
// tile ahead of the load.
// No unit is at its limit: by counters (head dim 128) the matrix cores are busy for 45% of
// the cycles, the vector ALU for 38 and LDS for 23 (no bank conflicts), and 28% of the
// waves' time is waiting.  Two waves per SIMD, all that the registers of head dim 128
// allow, take the two pipes by turns more than side by side.  Blocks of 8 waves, which
// halve the fills, gain nothing (587 us for 585, 169 for 151 with head dim 64); 64
// queries per wave, which would halve the LDS reads, do not fit the registers.  With head
// dim 64 four stages take longer than two (250 us for 240); its 160 registers would
// let a third wave onto a SIMD, which the kernel's attribute does not.
// 4 chunks of 1900 to 2048 rows after 3000 to 9000, window 4096, 32 heads of 128 on
// 8: 575 us, 920 TFLOP/s of visible products (a large matrix product: 1370).  8 prompts
// of 4096, window 1024, 16 heads of 64 on 4: 200 us, 600 TFLOP/s.
// ---------------------------------------------------------------------------
typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;

__device__ __forceinline__ f32x16 mfma32(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// The stages swizzle their rows: physical 16-byte chunk of logical chunk c of K
// row r: the 16 rows that one phase of a fragment read touches lie in different
// banks.  (An involution: it maps physical to logical chunks as well.)
template <int DH>
__device__ __forceinline__ int rows_kswz(int r, int c) {
  return DH == 128 ? (c ^ (r & 15)) : (c ^ ((r >> 1) & 7));
}
// V by 64-byte segments: the 4 rows that one half of a transposing read touches
// lie in different banks
template <int DH>
__device__ __forceinline__ int rows_vswz(int r, int c) {
  return c ^ ((DH == 128 ? (r & 3) : ((r >> 1) & 1)) << 2);
}

// wait until at most n loads of the wave are outstanding and its LDS accesses have finished
template <int N>
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14)); }

template <int DH, bool TABLE>
__device__ __forceinline__ void rows_block(const Plan& pl, const PagedAttn& a, int id, bf16* stage0, bf16* stage1) {
  constexpr int NW = 4;                  // waves
  constexpr int CH = DH / 8;             // 16-byte chunks per row
  constexpr int RPI = 64 / CH;           // rows per wave-wide load
  constexpr int NI = 64 / (NW * RPI);    // K (and V) loads per wave and tile
  constexpr int KS = DH / 16;            // MFMA steps over the head dims
  constexpr int ND = DH / 32;            // output tiles
  // Stage j: K of a tile t with t mod 2 = j, then V of tile t - 1 (a step reads K a tile ahead of V).
  // A variable per stage, so that the compiler can tell the one that is read from the one being
  // filled and does not wait for its loads.
  constexpr int TE = 64 * DH;
  auto stage = [&](auto b) -> bf16* {
    if constexpr (b == 0) return stage0;
    else return stage1;
  };
  __shared__ int s_poison;

  const int rb = rows_per_block(a.G);
  Work w;
  if constexpr (TABLE) {
    w.p = request_at(table_of(pl, a, TAB_ROWS), pl.n_req, id);
  } else {
    w.h = id % a.KH; id /= a.KH;
    w.c = id % a.rows_chunks; id /= a.rows_chunks;
    // request p's blocks start at cu[p] / rb + p: at least ceil(m / rb) before the next request's
    int lo = 0, hi = pl.n_req - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (uniform(pl.cu_seqlens[mid]) / rb + mid <= id) lo = mid; else hi = mid - 1;
    }
    w.p = lo;
  }
  const int R0 = uniform(pl.cu_seqlens[w.p]), m = uniform(pl.cu_seqlens[w.p + 1]) - R0, ctx = uniform(pl.ctx[w.p]);
  const int request = uniform(pl.order[w.p]);            // with them, not behind what they decide
  // a request's last rows see the most keys: they come first
  const int nb = (m + rb - 1) / rb;
  int bi = id - (R0 / rb + w.p);
  if (few_rows(VFM_BF16, m, a.G) || (!TABLE && bi >= nb)) return;   // block-uniform, as every exit below
  const Chunks ck = request_chunks(VFM_BF16, m, ctx, a.G, a.KH, a.window, a.n_sink);
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
    const bf16* qr = (const bf16*)a.q + row * a.ldq + head * DH + 8 * h2;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qr + 16 * s);
  }
  const page_row prow = row_of(a.kp, request);
  const int lp = a.kp.log2_page;
  const bf16* kh = (const bf16*)a.k + (int64_t)w.h * a.slots * DH;
  const bf16* vh = (const bf16*)a.v + (int64_t)w.h * a.slots * DH;
  if (tid == 0) s_poison = -1;

  f32x16 o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  float m_run = LOWEST, l_run = 0.f;

  // A lane's load i of a tile: row RPI (NW i + wave) + lane / CH, physical chunk lane % CH;
  // within its 16-position run the row, and with it the swizzle, is the same for every i.
  const int lrow = RPI * wave + lane / CH;                // mod 16: the row in its run
  // Byte offsets from the run's first row, which is a scalar.
  const uint32_t koff = 2 * ((lrow & 15) * DH + rows_kswz<DH>(lrow, lane % CH) * 8);
  const uint32_t voff = 2 * ((lrow & 15) * DH + rows_vswz<DH>(lrow, lane % CH) * 8);
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
  // K of the tile looked up last and V of the one looked up before it into stage b; looks `next` up.  Past the last tile that one is loaded again, into stages that nothing reads any
  // more: the loop needs no branch, and the count of loads in flight is always the same.
  int64_t vrun[NI] = {};
  auto issue = [&](auto b, int next, auto with_v) {
    int64_t krun[NI], prun[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      krun[i] = (int64_t)((page[i] << lp) + in_page[i]) * DH;
      prun[i] = vrun[i];
      vrun[i] = krun[i];
    }
    look_up(next);
#pragma unroll
    for (int i = 0; i < NI; ++i)
      __builtin_amdgcn_global_load_lds((gptr_t)((const char*)(kh + krun[i]) + koff), (lptr_t)(stage(b) + RPI * (NW * i + wave) * DH), 16, 0, 0);
    if constexpr (with_v)
#pragma unroll
      for (int i = 0; i < NI; ++i)
        __builtin_amdgcn_global_load_lds((gptr_t)((const char*)(vh + prun[i]) + voff),
                                         (lptr_t)(stage(b) + TE + RPI * (NW * i + wave) * DH), 16, 0, 0);
  };
  // V rows of a tile that some row of the block does not see: zeros where none sees them, no
  // infinities or NaN where some do
  auto mend = [&](auto b, int t) {
    const int kb = 64 * vis.run(t);
#pragma unroll 1
    for (int i = 0; i < NI; ++i) {
      const int r = RPI * NW * i + lrow, k = kb + r;
      bf16x8* at = reinterpret_cast<bf16x8*>(stage(b) + TE + r * DH + (lane % CH) * 8);
      if (!seen_by_any(j0, j1, k, a.window, a.n_sink)) *at = bf16x8{};
      else if (!seen_by_all(j0, j1, k, k, a.window, a.n_sink)) {
        bool found = false;
        const bf16x8 v = drop_nonfinite(*at, found);
        if (found) { *at = v; s_poison = t; }
      }
    }
  };

  // fragment addresses (bytes): K row x of a 32-key half, chunk 2 s + h2;
  // V: the transposing read takes 4 keys x 16 dims per 16 lanes, lane (x & 15)
  // bringing key (x & 15) / 4, dims 4 (x & 3).  Its rows differ from the lane's
  // first by multiples of 8, which leave the swizzle alone.
  const int kq = x & 15, gq = x >> 4;
  const int kaddr = x * DH * 2 + (rows_kswz<DH>(x, h2) << 4);
  const int vaddr = (4 * h2 + (kq >> 2)) * DH * 2 + (rows_vswz<DH>(kq >> 2, 0) << 4) + gq * 32 + (kq & 3) * 8;

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
  // the infinities and NaN that `mend` took out of tile t
  auto add_nonfinite = [&](int t) {
    const int kb = 64 * vis.run(t);
#pragma unroll 1
    for (int r = 0; r < 64; ++r) {
      const int k = kb + r;
      if (!seen_by_any(j0, j1, k, a.window, a.n_sink) || seen_by_all(j0, j1, k, k, a.window, a.n_sink)) continue;
      const bf16* vrow = vh + (int64_t)(page_slot(prow, lp, k)) * DH + 4 * h2;
      if (sees(jq, k, a.window, a.n_sink)) {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float v = (float)vrow[32 * d + 8 * (i >> 2) + (i & 3)];
            o[d][i] += nonfinite(v) ? v : 0.f;
            if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // rare: no registers for loads in flight
          }
      }
    }
  };

  // While the weights of tile t are computed (vector ALU), the matrix cores already take the scores
  // of tile t + 1; while they take the products of t, its largest scores are found.  K of tile t + 1
  // and V of tile t were asked for a step ago, and nothing later has been;
  // the barrier makes every wave's part visible, and frees K of tile t and V of tile t - 1.
  if (t0 < t1) {
    f32x16 sa[2], sb[2];
    look_up(t0);
    auto fill = [&](auto j) { issue(j, t0 + j + 1, std::bool_constant<(j > 0)>{}); };
    fill(std::integral_constant<int, 0>{});
    fill(std::integral_constant<int, 1>{});
    wait_loads<2 * NI>();
    __builtin_amdgcn_s_barrier();
    scores(std::integral_constant<int, 0>{}, sa);
    mask(t0, sa);
    follow(largest(sa));
    settle(sa);
    // tile t, t mod 2 = j: its scores st, the next one's sn (behind the last tile: of what the stage
    // holds, and not used)
    auto step = [&](auto j, int t, f32x16 (&st)[2], f32x16 (&sn)[2]) {
      constexpr auto jn = std::integral_constant<int, 1 - j>{};   // holds K of tile t + 1, V of tile t
      wait_loads<0>();
      __builtin_amdgcn_s_barrier();
      const int kb = 64 * vis.run(t);
      if (!seen_by_all(j0, j1, kb, kb + 63, a.window, a.n_sink)) {
        mend(jn, t);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
      }
      bf16x8 pf[4];
      __builtin_amdgcn_sched_barrier(0);
      // Scores of t + 1 (2 KS MFMAs) beside the first half of t's weights and the next loads (32 KB
      // take the CU 512 cycles to address); a fragment is read four ahead of its MFMA.
      scores(jn, sn);
      weights(st, 0, pf);
      weights(st, 1, pf);
      issue(j, t + 3, std::true_type{});
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int s = 0; s < 2 * KS; ++s) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x402, 64 / (2 * KS), 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        if (s % (2 * KS / (2 * NI)) == 1) __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) asm volatile("" : "+v"(pf[u]));   // not put off behind the mask
      __builtin_amdgcn_sched_barrier(0);
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
    wait_loads<0>();                                      // nothing still writes to LDS when the block ends
  }
  l_run = sum_x32(l_run);
  if (wave * 32 + x >= qn) return;
  if (ck.n == 1) {
    const float inv = 1.f / l_run;
    bf16* orow = (bf16*)a.out + row * a.ldo + head * DH + 4 * h2;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (bf16)(o[d][4 * j + i] * inv);
        *reinterpret_cast<bf16x4*>(orow + 32 * d + 8 * j) = v;
      }
  } else {
    const int64_t rec = record_of<TABLE>(pl, a, w.p, R0, ck.n, row, head) + w.c;
    float* ro = a.rec_o + rec * DH + 4 * h2;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4*>(ro + 32 * d + 8 * j) =
            f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
    if (h2 == 0) a.rec_ml[rec] = make_float2(m_run, l_run);
  }
}

// rows_blocks blocks of the many-row kind (ROWS), then, with FEW, those of the few-row kind: a step's
// single rows run beside its prompts, on the CUs that these leave free.  24 requests of 64 to 2000
// positions, 5 of them with up to 250 rows, 16 heads of 64: 28.5 us (31.5 when two launches took 45.7).
// SINGLE (no rows): without registers for a second tile 4 blocks share a CU instead of 2, and other blocks'
// work hides a block's start and its loads.  It is taken where no few-row request has more than 128 keys
// (a tile per wave): 256 rows of 70 to 120 keys, 32 heads of 128: 72 us, else 108; of 30 to 60 keys: 60 and
// 80; one row of 100 keys: 7.5 and 7.4.  With head dim 64 also where the launch has more blocks than 2 per CU,
// those that find no work among them, as they take places, too: 16 heads, 256 rows of 200 to 2000 keys
// 177 us and 206, 64 of 8000 331 and 333, 3 of 80 to 200 beside one of 60000 47 and 67; 16 of 60000, the worst
// found, 597 and 585.  With few blocks the loads in flight count: 16 rows of 130 to 400 keys (256 blocks) would
// take 8.8 instead of 8.0.  With head dim 128 a loop of single tiles spills at 4 blocks (954 us for 598)
// and gains nothing at 3.  The order of a row's sums is the same in both.
template <int DH, bool ROWS, bool FEW, bool SINGLE, bool TABLE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(SINGLE ? 4 : 2, SINGLE ? 4 : 2))) void attn_bf16_kernel(
    Plan pl, PagedAttn a, int rows_blocks) {
  __shared__ __attribute__((aligned(16))) bf16 stage0[128 * DH], stage1[ROWS ? 128 * DH : 8];
  if constexpr (FEW)
    if ((int)blockIdx.x >= rows_blocks) {
      few_block<DH, SINGLE, TABLE>(pl, a, (int)blockIdx.x - rows_blocks, reinterpret_cast<char*>(stage0));
      return;
    }
  if constexpr (ROWS) rows_block<DH, TABLE>(pl, a, blockIdx.x, stage0, stage1);
}

// ---------------------------------------------------------------------------
// fp32, any number of rows (v_mfma_f32_16x16x4_f32): 16 packed queries per
// block, the chunk's 16-key runs dealt to the 4 waves, operands from memory
// straight into registers.  A 16-byte load of K or Q holds 4 consecutive head
// dims, MFMA e taking component e of both; P^T is the B operand of the PV
// products as it lies (MFMA j takes keys 4 g + j), and a lane that loads dims
// 4 x .. 4 x + 3 of its key's V row gives MFMA c row x of tile c = head dim
// 4 x + c, which leaves a lane with 16 consecutive head dims of its query.
// Every K and V element is read once per 16 queries, from L2 for the later ones.
// 64 rows after 2000 keys, 16 heads of 64: 188 us, 5.6 TB/s.  8 chunks of 512 rows
// after 1000: 225 us, 94 TFLOP/s (a large fp32 matrix product: 154): each 16 queries
// load all of their K and V from L2, which no other block's queries share through LDS.
// ---------------------------------------------------------------------------
template <int DH, bool TABLE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void attn_f32_kernel(Plan pl, PagedAttn a) {
  constexpr int NC = DH / 16, NH = DH / 64;
  __shared__ float sm[4][16], sl[4][16];
  __shared__ __attribute__((aligned(16))) float so[4][16][DH];
  auto mfma = [](float p, float q, const f32x4& c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(p, q, c, 0, 0, 0); };
  Work w;
  int id = blockIdx.x;
  if constexpr (TABLE) {
    w.p = request_at(table_of(pl, a, TAB_FEW), pl.n_req, id);
  } else {
    w.h = id % a.KH; id /= a.KH;
    w.c = id % a.few_chunks; id /= a.few_chunks;
    // request p's query tiles start at cu[p] G / 16 + p
    int lo = 0, hi = pl.n_req - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((int64_t)uniform(pl.cu_seqlens[mid]) * a.G / 16 + mid <= id) lo = mid; else hi = mid - 1;
    }
    w.p = lo;
    w.qt = id - (int)((int64_t)uniform(pl.cu_seqlens[lo]) * a.G / 16 + lo);
  }
  const int R0 = uniform(pl.cu_seqlens[w.p]), m = uniform(pl.cu_seqlens[w.p + 1]) - R0, ctx = uniform(pl.ctx[w.p]);
  const int request = uniform(pl.order[w.p]);            // with them, not behind what they decide
  const int qn = m * a.G;
  if (!TABLE && w.qt * 16 >= qn) return;      // block-uniform, as every exit below
  const Chunks ck = request_chunks(VFM_F32, m, ctx, a.G, a.KH, a.window, a.n_sink);
  if constexpr (TABLE) {
    w.h = id % a.KH; id /= a.KH;
    w.c = id % ck.n;
    w.qt = id / ck.n;
  } else if (w.c >= ck.n) {
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = lane & 15, g = lane >> 4;
  const int qi = min(w.qt * 16 + x, qn - 1);
  const int jq = ctx + qi / a.G;
  const int j0 = ctx + w.qt * 16 / a.G, j1 = ctx + min(w.qt * 16 + 15, qn - 1) / a.G;
  // the tile's own runs, dealt over the request's chunks
  const Vis vis = visible_runs<4>(j0, j1, a.window, a.n_sink);
  const int rpc = (vis.n + ck.n - 1) / ck.n;
  const int t0 = w.c * rpc, t1 = min(t0 + rpc, vis.n);
  int head;
  const int64_t row = out_row(a, R0, w.h, qi, head);
  const page_row prow = row_of(a.kp, request);
  const int lp = a.kp.log2_page;
  const float* kh = (const float*)a.k + (int64_t)w.h * a.slots * DH;
  const float* vh = (const float*)a.v + (int64_t)w.h * a.slots * DH;
  f32x4 q[NC], o[NH][4];
#pragma unroll
  for (int c = 0; c < NC; ++c)
    q[c] = *reinterpret_cast<const f32x4*>((const float*)a.q + row * a.ldq + head * DH + 16 * c + 4 * g);
#pragma unroll
  for (int hh = 0; hh < NH; ++hh)
#pragma unroll
    for (int c = 0; c < 4; ++c) o[hh][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = LOWEST, l_run = 0.f;
  for (int t = t0 + wave; t < t1; t += 4) {
    const int p0 = 16 * vis.run(t);
    const int64_t slot = page_slot(prow, lp, p0);
    const bool full = seen_by_all(j0, j1, p0, p0 + 15, a.window, a.n_sink);
    f32x4 kf[NC], vf[4][NH];
#pragma unroll
    for (int c = 0; c < NC; ++c)
      kf[c] = *reinterpret_cast<const f32x4*>(kh + (slot + x) * DH + 16 * c + 4 * g);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int hh = 0; hh < NH; ++hh)
        vf[j][hh] = *reinterpret_cast<const f32x4*>(vh + (slot + 4 * g + j) * DH + 64 * hh + 4 * x);
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = mfma(kf[c][e], q[c][e], s);
    bool poison = false;
    if (!full) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = p0 + 4 * g + j;
        s[j] = sees(jq, k, a.window, a.n_sink) ? s[j] : -INFINITY;
        const bool any = seen_by_any(j0, j1, k, a.window, a.n_sink);
        const bool some = any && !seen_by_all(j0, j1, k, k, a.window, a.n_sink);
#pragma unroll
        for (int hh = 0; hh < NH; ++hh)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const bool bad = some && nonfinite(vf[j][hh][c]);
            poison = poison || bad;
            vf[j][hh][c] = !any || bad ? 0.f : vf[j][hh][c];
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
    for (int hh = 0; hh < NH; ++hh)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[hh][c] *= alpha;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float e = exp2f((s[j] - m_run) * a.scale_log2);
      l_run += e;
#pragma unroll
      for (int hh = 0; hh < NH; ++hh)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[hh][c] = mfma(vf[j][hh][c], e, o[hh][c]);
    }
    if (__any(poison)) {                                  // rare: see add_nonfinite of the bf16 kernel
      for (int r = 0; r < 16; ++r) {
        const int k = p0 + r;
        if (!seen_by_any(j0, j1, k, a.window, a.n_sink) || seen_by_all(j0, j1, k, k, a.window, a.n_sink)) continue;
        const bool see = sees(jq, k, a.window, a.n_sink);
#pragma unroll
        for (int hh = 0; hh < NH; ++hh)
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float v = vh[(slot + r) * DH + 64 * hh + 16 * g + 4 * i + c];
              if (see && nonfinite(v)) o[hh][c][i] += v;
            }
      }
    }
  }
  l_run = sum_x32(sum_x16(l_run));
  if (lane < 16) { sm[wave][x] = m_run; sl[wave][x] = l_run; }
#pragma unroll
  for (int hh = 0; hh < NH; ++hh)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4*>(&so[wave][x][64 * hh + 16 * g + 4 * i]) =
          f32x4{o[hh][0][i], o[hh][1][i], o[hh][2][i], o[hh][3][i]};
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

// ---------------------------------------------------------------------------
// Joins the chunks' partial sums of rows whose keys were cut: a wave per row and
// head, o = sum_c w_c o_c / sum_c w_c l_c with w_c = 2^((m_c - M) scale), chunks in order.
// Bound by its launch: 5 to 7 us for 256 rows of 32 heads in up to 8 chunks.
// ---------------------------------------------------------------------------
template <typename T, int DH, bool TABLE>
__global__ __launch_bounds__(256) void attn_join_kernel(Plan pl, PagedAttn a, int joins) {
  constexpr int DT = std::is_same<T, bf16>::value ? VFM_BF16 : VFM_F32;
  constexpr int E = DH / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int id = (int)blockIdx.x * 4 + wave;                    // the launch has fewer than 2^26
  if (id >= joins) return;
  int r, p;
  if constexpr (TABLE) {
    p = request_at(table_of(pl, a, TAB_JOIN), pl.n_req, id);
    r = uniform(pl.cu_seqlens[p]) + id / a.H;
  } else {
    r = id / a.H;
    p = uniform(pl.row_req[r]);
  }
  const int head = id % a.H;
  const int R0 = uniform(pl.cu_seqlens[p]), m = uniform(pl.cu_seqlens[p + 1]) - R0, ctx = uniform(pl.ctx[p]);
  const int n = request_chunks(DT, m, ctx, a.G, a.KH, a.window, a.n_sink).n;
  if (n <= 1) return;
  const int64_t rec = record_of<TABLE>(pl, a, p, R0, n, r, head);
  const float2* ml = a.rec_ml + rec;
  const float* ro = a.rec_o + rec * DH + E * lane;
  float M = LOWEST;
  for (int c = lane; c < n; c += 64) M = fmaxf(M, ml[c].x);
  M = max_x32(max_x16(max_row(M)));
  float L = 0.f, acc[E] = {};
  for (int c0 = 0; c0 < n; c0 += 64) {
    float wt = 0.f;
    if (c0 + lane < n) {
      const float2 v = ml[c0 + lane];
      wt = exp2f((v.x - M) * a.scale_log2);
      L += wt * v.y;
    }
    const int cn = min(64, n - c0);
    int c = 0;
    for (; c + 4 <= cn; c += 4) {
      float v[4][E];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) v[j][e] = ro[(int64_t)(c0 + c + j) * DH + e];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float wc = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wt), c + j));
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(wc, v[j][e], acc[e]);
      }
    }
    for (; c < cn; ++c) {
      const float wc = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wt), c));
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(wc, ro[(int64_t)(c0 + c) * DH + e], acc[e]);
    }
  }
  L = sum_x32(sum_x16(sum_row(L)));
  T* dst = (T*)a.out + (int64_t)r * a.ldo + head * DH + E * lane;
#pragma unroll
  for (int e = 0; e < E; ++e) dst[e] = from_f32<T>(acc[e] / L);
}

// ---------------------------------------------------------------------------
// The prefix sums of a.table: one block, 256 requests at a time.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void attn_table_kernel(Plan pl, PagedAttn a, int dtype, int32_t* table) {
  __shared__ int64_t part[4][4];                          // sums of a wave's requests
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int64_t base[4] = {};
  for (int p0 = 0; p0 < pl.n_req; p0 += 256) {
    const int p = p0 + tid;
    AttnCounts c = {};
    if (p < pl.n_req) {
      const int m = pl.cu_seqlens[p + 1] - pl.cu_seqlens[p];
      c = request_counts(dtype, m, a.H, a.KH, request_chunks(dtype, m, pl.ctx[p], a.G, a.KH, a.window, a.n_sink).n);
    }
    int64_t sum[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum[i] = c.v[i];
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int64_t o = __shfl_up(sum[i], d, 64);
        sum[i] += lane >= d ? o : 0;
      }
      if (lane == 63) part[i][wave] = sum[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      for (int w = 0; w < 4; ++w) {
        if (w < wave) sum[i] += part[i][w];
      }
      if (p < pl.n_req) table[(int64_t)i * (pl.n_req + 1) + p + 1] = (int32_t)(base[i] + sum[i]);
      for (int w = 0; w < 4; ++w) base[i] += part[i][w];
    }
    __syncthreads();
  }
  if (tid < 4) table[(int64_t)tid * (pl.n_req + 1)] = 0;
}

}  // namespace

hipError_t launch_kv_append(int dtype, const Plan& pl, int H, int KH, int head_dim, float theta, const void* qkv,
                            int64_t ld, void* q_out, int64_t ldq, void* k, void* v, int64_t slots, const KvPages& kp,
                            hipStream_t s) {
  const int rotate = theta > 0.f;
  const double l2 = rotate ? log2((double)theta) : 0.0;
#define APPEND(T_, D_)                                                                                     \
  hipLaunchKernelGGL((kv_append_kernel<T_, D_>), dim3(pl.T), dim3(APPEND_THREADS), 0, s, pl, H, KH, rotate, l2, (const T_*)qkv, ld, \
                     (T_*)q_out, ldq, (T_*)k, (T_*)v, slots, kp)
  if (dtype == VFM_BF16) { if (head_dim == 64) APPEND(bf16, 64); else APPEND(bf16, 128); }
  else { if (head_dim == 64) APPEND(float, 64); else APPEND(float, 128); }
#undef APPEND
  return hipGetLastError();
}

namespace {

template <int DH, bool TABLE>
void launch_attention_blocks(int dtype, const Plan& pl, const PagedAttn& a, unsigned nf, unsigned nr, bool one,
                             hipStream_t s) {
  const dim3 block(256), grid(nf + nr);
  if (dtype != VFM_BF16) hipLaunchKernelGGL((attn_f32_kernel<DH, TABLE>), grid, block, 0, s, pl, a);
#define BF16(R_, F_, O_) hipLaunchKernelGGL((attn_bf16_kernel<DH, R_, F_, O_, TABLE>), grid, block, 0, s, pl, a, (int)nr)
  else if (nr && nf) BF16(true, true, false);
  else if (nr) BF16(true, false, false);
  else if (one || (DH == 64 && nf > 512)) BF16(false, true, true);
  else BF16(false, true, false);
#undef BF16
}

template <int DH, bool TABLE>
void launch_attention_join(int dtype, const Plan& pl, const PagedAttn& a, int joins, hipStream_t s) {
  const dim3 block(256), grid((unsigned)((joins + 3) / 4));
  if (dtype == VFM_BF16) hipLaunchKernelGGL((attn_join_kernel<bf16, DH, TABLE>), grid, block, 0, s, pl, a, joins);
  else hipLaunchKernelGGL((attn_join_kernel<float, DH, TABLE>), grid, block, 0, s, pl, a, joins);
}

}  // namespace

hipError_t launch_attention_paged(int dtype, int head_dim, const Plan& pl, const PagedAttn& a, int64_t few_blocks,
                                  int64_t rows_blocks, int64_t joins, bool one, bool table, hipStream_t s) {
#define BY(F_, ...)                                                                       \
  do {                                                                                    \
    if (table) { if (head_dim == 64) F_<64, true>(__VA_ARGS__); else F_<128, true>(__VA_ARGS__); } \
    else if (head_dim == 64) F_<64, false>(__VA_ARGS__);                                  \
    else F_<128, false>(__VA_ARGS__);                                                     \
  } while (0)
  if (table) {
    const int pi = prof_begin(VFM_PROF_OTHER, s);
    hipLaunchKernelGGL(attn_table_kernel, dim3(1), dim3(256), 0, s, pl, a, dtype, const_cast<int32_t*>(a.table));
    prof_end(pi, s);
  }
  int pi = prof_begin(VFM_PROF_ATTN, s);
  BY(launch_attention_blocks, dtype, pl, a, (unsigned)few_blocks, (unsigned)rows_blocks, one, s);
  prof_end(pi, s);
  if (joins) {
    pi = prof_begin(VFM_PROF_OTHER, s);
    BY(launch_attention_join, dtype, pl, a, (int)joins, s);
    prof_end(pi, s);
  }
#undef BY
  return hipGetLastError();
}
