// What the attention kernels over paged caches share: softmax steps across lanes, what a row sees, page lookups, the
// place of a block's work, and the MFMA tiles' layouts.
#pragma once

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
// MFMA tiles, and the stages of the many-row kernels.
// ---------------------------------------------------------------------------
__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

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

}  // namespace
