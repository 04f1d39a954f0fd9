// Declarations of the bounded-cache decoding kernels (k_paged.hip, k_sample.hip).
#pragma once

#include <initializer_list>

#include "vfm_decode.h"
#include "vfm_internal.h"
#include "vfm_kv8.h"

// One attention over a paged cache, as the kernels take it.
struct PagedAttn {
  int16_t H, KH;               // query heads, key heads (at most 1024)
  int G;                       // query heads per key head
  int kv8;                     // the cache is held in 8 bits
  int window, n_sink;          // window 0: none
  float scale_log2;            // scale * log2(e)
  const void* q; int64_t ldq;
  const void* k; const void* v; int64_t slots;   // slots per head
  KvPages kp;
  void* out; int64_t ldo;
  // partial results of rows whose keys are cut, a record per row, head and chunk
  float* rec_o;                // [records][head_dim] outputs
  float2* rec_ml;              // [records] largest score, sum
  union {                      // (a longer argument list costs a call of one row 0.2 us of 8.9)
    struct {                   // blocks and records in rectangles over the largest counts:
      int few_chunks, rows_chunks;   // chunks of a few-row and of a many-row request (1 if none)
      int nchunk;              // the larger of the two (the records' stride)
      int qtiles;              // query tiles of a few-row request
    };
    const int32_t* table;      // or where each request's own begin
  };
};

// The table: four prefix sums over the batch's requests in plan order, [4][n_req + 1]: blocks of the many-row kind, of the
// few-row kind, records, and rows times heads that are joined.  A request's blocks are in the order of tile, chunk
// and head, its records in that of row, head and chunk, its joins in that of row and head.  A kernel before the
// attention writes the table where rectangles would be mostly empty (plan_attention has the rule).
enum { TAB_ROWS = 0, TAB_FEW = 1, TAB_RECS = 2, TAB_JOIN = 3 };
struct AttnCounts { int64_t v[4]; };

// What one request's rows see, in runs of 2^SH positions: ns runs from position
// 0 (the sinks), then the runs from run `base` up to the last row's own.
struct Vis {
  int ns, base, n;             // n: runs in all
  __host__ __device__ int run(int i) const { return i < ns ? i : i - ns + base; }
};
template <int SH>
__host__ __device__ inline Vis visible_runs(int first_pos, int last_pos, int window, int n_sink) {
  Vis v;
  const int end = last_pos + 1;
  const int lo = window > 0 && first_pos - window + 1 > 0 ? first_pos - window + 1 : 0;
  v.base = lo >> SH;
  const int sk = n_sink < end ? n_sink : end;
  v.ns = (sk + (1 << SH) - 1) >> SH;
  if (v.ns >= v.base) { v.ns = 0; v.base = 0; }
  v.n = v.ns + ((end + (1 << SH) - 1) >> SH) - v.base;
  return v;
}

// A request's keys are cut into chunks of whole tiles, one block each, as far
// as the request alone then fills the chip: 256 blocks with the `par` (key
// heads x query tiles) that it has uncut, and at least min_tiles tiles each.
// Nothing but the request's own sizes and the head layout goes into it, so a
// row's bits do not depend on the batch.
struct Chunks { int n, tiles; };   // chunks, tiles per chunk
__host__ __device__ inline Chunks key_chunks(int tiles, int par, int min_tiles) {
  int want = 256 / par;
  const int most = tiles / min_tiles;
  if (want > most) want = most;
  if (want < 1) want = 1;
  Chunks c;
  c.tiles = (tiles + want - 1) / want;
  c.n = (tiles + c.tiles - 1) / c.tiles;
  return c;
}

constexpr int FEW_QUERIES = 32;      // packed queries (rows x group) up to which a request takes the few-row kernel
// The fewest tiles of a chunk, so long as a request has them. A chunk costs its block's start and its share
// of the join; uncut, a request alone uses few CUs. 32 heads of 128 on 32 of keys. Few-row kernel, 32-key
// tiles: one row after 1500 keys takes 14.4 us with 8 tiles, 17.0 with 12, 26.5 with 24; one row of each of 256
// requests with up to 2048 keys under a window of 1024 654, 597, 582. Many-row kernel, 64-key tiles: 100 rows
// after 1500 keys take 26.3 us with 8 and 32.3 with 16; 512 rows after none 21.2 with 8 and 30.6 with 4.
constexpr int FEW_MIN_TILES = 12;
constexpr int ROWS_MIN_TILES = 8;
// bf16 over a cache in 8 bits, whose tiles are read in half the time: 256 rows under a window of 1024, 32 heads of 128 on 32,
// take 321 us with 12 and 305 with 18 (uncut), 128 rows after 1000 keys, 64 heads of 64 on 8, 32 and 24; one row after 1500 takes
// 14.2 and 15.9.
constexpr int FEW_MIN_TILES8 = 18;
// fp32 over 8 bits where single_row holds: 64 rows after 2000 keys, 16 heads of 64, take 78 us with 12, 61 with 24 and 54 with 32
// (uncut), one after 3000, 16 heads on 4, 11.6, 15.3 and 18.7.
constexpr int SINGLE_MIN_TILES8 = 24;

// few-row kernel (bf16; fp32: every request): 16 packed queries per block
__host__ __device__ inline bool few_rows(int dtype, int m, int G) { return dtype != VFM_BF16 || (int64_t)m * G <= FEW_QUERIES; }
// fp32 over a cache in 8 bits: one row of at most 4 queries on a key head, which sees more than 8 runs of 16 keys (256 rows of
// 30 to 60, 8 heads of 64: 20.2 us with the single rows' kernel, 16.2 without; 4 of 176 to 322, 4 heads of 128: 11.5 and 12.1)
__host__ __device__ inline bool single_row(int m, int G, int runs) { return m == 1 && G <= 4 && runs > 8; }
__host__ __device__ inline int64_t few_qtiles(int m, int G) { return ((int64_t)m * G + 15) / 16; }
// many-row kernel (bf16): blocks of 128 packed queries, 32 a wave
__host__ __device__ inline int rows_per_block(int G) { return 128 / G; }

// chunks of the request with m rows after ctx cached tokens
__host__ __device__ inline Chunks request_chunks(int dtype, int m, int ctx, int G, int KH, int window, int n_sink,
                                                 bool kv8 = false) {
  if (few_rows(dtype, m, G)) {
    const int runs = visible_runs<4>(ctx, ctx + m - 1, window, n_sink).n, tiles = (runs + 1) / 2;
    const int64_t qt = few_qtiles(m, G);
    const int par = KH * (qt > 256 ? 256 : (int)qt);
    const int few_min = !kv8 ? FEW_MIN_TILES : dtype == VFM_BF16 ? FEW_MIN_TILES8
                        : single_row(m, G, runs) ? SINGLE_MIN_TILES8 : FEW_MIN_TILES;
    return key_chunks(tiles, par > 256 ? 256 : par, few_min);
  }
  const int rb = rows_per_block(G);
  const int64_t par = (int64_t)KH * ((m + rb - 1) / rb);
  const int m1 = m < rb ? m : rb;     // a block sees at most this many tiles more or fewer than another
  const int tiles = visible_runs<6>(ctx + m - m1, ctx + m - 1, window, n_sink).n;
  return key_chunks(tiles, par > 256 ? 256 : (int)par, ROWS_MIN_TILES);
}

// what a request of m rows and n chunks adds to the table
__host__ __device__ inline AttnCounts request_counts(int dtype, int m, int H, int KH, int n) {
  const int G = H / KH;
  const bool few = few_rows(dtype, m, G);
  const int rb = rows_per_block(G);
  AttnCounts c;
  c.v[TAB_ROWS] = few ? 0 : (int64_t)KH * n * (((int64_t)m + rb - 1) / rb);
  c.v[TAB_FEW] = few ? KH * n * few_qtiles(m, G) : 0;
  c.v[TAB_RECS] = n > 1 ? (int64_t)m * H * n : 0;
  c.v[TAB_JOIN] = n > 1 ? (int64_t)m * H : 0;
  return c;
}

constexpr int APPEND_THREADS = 256;  // a block per row

// q_out: rows ldq apart; qkv itself (ldq = ld) to rotate the queries in place, NULL for keys and values only.
hipError_t launch_kv_append(int dtype, const Plan& pl, int H, int KH, int head_dim, float theta, const void* qkv,
                            int64_t ld, void* q_out, int64_t ldq, void* k, void* v, int64_t slots, const KvPages& kp,
                            hipStream_t s);

// few_blocks, rows_blocks, joins: the grids (few rows, many rows) and the rows times heads to join; one: no few-row
// request has more than a tile per wave.  table: a.table is there, and is written first.
hipError_t launch_attention_paged(int dtype, int head_dim, const Plan& pl, const PagedAttn& a, int64_t few_blocks,
                                  int64_t rows_blocks, int64_t joins, bool one, bool table, hipStream_t s);

// its parts: a.table written, and the chunks' records joined
void launch_attention_table(int dtype, const Plan& pl, const PagedAttn& a, hipStream_t s);
void launch_attention_joins(int dtype, int head_dim, const Plan& pl, const PagedAttn& a, int joins, bool table, hipStream_t s);

// ---- a cache held in 8 bits (k_kv8.hip) ----
struct Pool8 {
  uint8_t *k, *v;              // codes [n_kv_heads][slots][head_dim]
  uint8_t* exps;               // [slots / 16][n_kv_heads][2]
  int64_t slots;
};
constexpr int APPEND8_MAX_BLOCKS = (1 << 24) - 1;   // of 256 threads; requests and 16th rows together are at most as many
// q_out, ldq: as launch_kv_append
hipError_t launch_append8(int dtype, const Plan& pl, int H, int KH, int head_dim, float theta, const void* qkv, int64_t ld,
                          void* q_out, int64_t ldq, const Pool8& pool, const KvPages& kp, hipStream_t s);
// a.k, a.v: the pools' codes; deep: few blocks, or long ones (AttnPlan::deep); single, other: fp32 requests of a single row
// (single_row) and others; the other arguments as
// launch_attention_paged's
hipError_t launch_attention8(int dtype, int head_dim, const Plan& pl, const PagedAttn& a, const uint8_t* exps, int64_t few_blocks,
                             int64_t rows_blocks, int64_t joins, bool deep, bool single, bool other, bool table, hipStream_t s);

// max_out: the batch's longest row of head outputs; a block of that many threads per request
inline int sample_threads(int max_out) { return max_out <= 1024 ? 256 : 1024; }
hipError_t launch_sample(const Plan& pl, const float* out, const vfm_sampling& sp, const float* u, int32_t* ids,
                         float* logprob, int max_out, hipStream_t s);

// ---- penalties, biases and masks on head outputs (k_adjust.hip) ----
// Outputs that a block takes, 16 a thread (4 with the small ones): the largest with which there is a block for every CU, as
// each goes through all of a request's earlier tokens.
constexpr int ADJUST_LARGE = 16384, ADJUST_MIDDLE = 8192, ADJUST_SMALL = 1024;
constexpr int adjust_threads(int slice) { return slice == ADJUST_SMALL ? 256 : slice / 16; }
// blocks of slice s begin at s * adjust_rows: a multiple of 8, so a request's blocks share their number mod 8, the XCD
inline int adjust_rows(int n_req) { return (n_req + 7) & ~7; }
inline int64_t adjust_slices(int max_out, int slice) { return ((int64_t)max_out + 3 + slice - 1) / slice; }
inline int adjust_slice(int n_req, int max_out) {
  for (int slice : {ADJUST_LARGE, ADJUST_MIDDLE})
    if (max_out > ADJUST_SMALL && n_req * adjust_slices(max_out, slice) >= 256) return slice;
  return ADJUST_SMALL;
}
inline int64_t adjust_blocks(int n_req, int max_out) {
  return adjust_rows(n_req) * adjust_slices(max_out, adjust_slice(n_req, max_out));
}
hipError_t launch_adjust(const Plan& pl, const float* in, float* out, const vfm_adjust& a, int max_out, hipStream_t s);
