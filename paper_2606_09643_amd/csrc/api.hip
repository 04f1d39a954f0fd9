// C ABI entry points: argument validation, workspace carving and the launch
// sequence of one backbone layer over a mixed-task batch.
#include <algorithm>
#include <initializer_list>
#include <mutex>

#include "decode_internal.h"
#include "vfm_internal.h"

namespace {

constexpr size_t ALIGN = 256;
inline size_t align_up(size_t v) { return (v + ALIGN - 1) / ALIGN * ALIGN; }

inline size_t elem_size(int dtype) { return dtype == VFM_BF16 ? 2 : 4; }

int check_cfg(const vfm_cfg* c) {
  if (!c) return VFM_ERR_ARG;
  if (c->dtype != VFM_F32 && c->dtype != VFM_BF16) return VFM_ERR_ARG;
  if (c->norm != VFM_NORM_LAYER && c->norm != VFM_NORM_RMS) return VFM_ERR_ARG;
  if (c->mlp != VFM_MLP_GELU && c->mlp != VFM_MLP_SWIGLU) return VFM_ERR_ARG;
  if (c->attn < VFM_ATTN_BIDIR || c->attn > VFM_ATTN_MIXED) return VFM_ERR_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return VFM_ERR_UNSUPPORTED;
  if (c->n_heads < 1 || (int64_t)c->n_heads * c->head_dim != c->d_model) return VFM_ERR_SHAPE;
  if (c->d_model % 64 || c->d_model > 8192 || c->d_ff < 64 || c->d_ff % 64) return VFM_ERR_SHAPE;
  if (c->mlp == VFM_MLP_SWIGLU && c->has_bias) return VFM_ERR_UNSUPPORTED;
  if (!(c->norm_eps >= 0.f) || !(c->rope_theta >= 0.f)) return VFM_ERR_ARG;
  return VFM_OK;
}

int check_batch(const vfm_batch* b, Plan* out) {
  if (!b || !b->plan_host || !b->plan_dev) return VFM_ERR_ARG;
  if (b->n_ints < VFM_PLAN_HEADER) return VFM_ERR_SHAPE;
  const int32_t* h = b->plan_host;
  if (h[0] < 1 || h[1] < 1 || h[2] < h[0]) return VFM_ERR_SHAPE;
  if ((size_t)plan_offsets(h[0], h[1], h[2]).total > b->n_ints) return VFM_ERR_SHAPE;
  *out = make_plan(h, b->plan_dev);
  return VFM_OK;
}

// host-side view of the plan arrays (for validation of cache bounds)
inline const int32_t* host_arr(const vfm_batch* b, int64_t off) { return b->plan_host + off; }

int check_lora(const vfm_lora_table* l, const Plan& pl) {
  if (!l) return VFM_OK;
  if (l->n_tasks != pl.n_tasks) return VFM_ERR_SHAPE;
  if (l->max_rank < 0 || l->max_rank > VFM_MAX_RANK || l->max_rank % 8) return VFM_ERR_SHAPE;
  if (!l->rank || !l->scale) return VFM_ERR_ARG;
  for (int p = 0; p < VFM_NPROJ; ++p)
    if ((l->A[p] == nullptr) != (l->B[p] == nullptr)) return VFM_ERR_ARG;
  return VFM_OK;
}

inline int rpad_of(const vfm_lora_table* l) {
  if (!l || l->max_rank == 0) return 0;
  return l->max_rank <= 32 ? 32 : 64;
}

// Small bf16 batches take the split-K GEMM + separate shrink + finalize path.
inline bool use_skinny(const vfm_cfg& c, const Plan& pl) {
  return c.dtype == VFM_BF16 && pl.T < VFM_SMALL_BATCH_ROWS;
}

// Largest number of keys one request attends to (ctx + its rows), from the
// host copy of the plan.
int max_keys_of(const vfm_batch* b, const Plan& pl) {
  const PlanOffsets po = plan_offsets(pl.n_req, pl.n_tasks, pl.T);
  const int32_t* ctx = b->plan_host + po.ctx;
  const int32_t* cu = b->plan_host + po.cu_seqlens;
  int mk = 0;
  for (int p = 0; p < pl.n_req; ++p) mk = std::max(mk, ctx[p] + cu[p + 1] - cu[p]);
  return mk;
}

struct LayerWs {
  size_t h, big, attn, u, z, p, aws, total;
  int kchunks;
};

// attn_bytes: the windowed attention's workspace in place of the attention's over max_keys keys.
LayerWs layer_ws(const vfm_cfg& c, const Plan& pl, const vfm_lora_table* l, int max_keys, int64_t attn_bytes = -1) {
  const size_t es = elem_size(c.dtype);
  const size_t T = (size_t)pl.T;
  const int d = c.d_model, f = c.d_ff, rpad = rpad_of(l);
  LayerWs w;
  size_t off = 0;
  w.h = off;    off += align_up(T * d * es);
  w.big = off;  off += align_up(T * std::max<size_t>(3 * (size_t)d, f) * es);
  w.attn = off; off += align_up(T * d * es);
  w.u = off;    off += align_up(T * 8 * rpad * es);
  w.aws = off; off += align_up(attn_bytes >= 0 ? (size_t)attn_bytes : attention_workspace(c, pl, max_keys));
  w.z = w.p = off;
  w.kchunks = 0;
  if (use_skinny(c, pl)) {
    // fp32 split partials of the largest projection group
    auto zbytes = [&](int N, int K) { return (size_t)skinny_splits(N, K) * T * N * 4; };
    const int n_up = c.mlp == VFM_MLP_SWIGLU ? 2 * f : f;
    const size_t zmax = std::max(std::max(zbytes(3 * d, d), zbytes(d, d)),
                                 std::max(zbytes(n_up, d), zbytes(d, f)));
    w.z = off; off += align_up(zmax);
    if (rpad > 0) {
      w.kchunks = std::max(shrink_chunks(d), shrink_chunks(f));
      w.p = off; off += align_up((size_t)w.kchunks * T * 8 * rpad * 4);
    }
  }
  w.total = off;
  return w;
}

// pooled rows, then room for the MLP heads' hidden rows (hidden <= d)
size_t head_ws(const vfm_cfg& c, const Plan& pl) {
  return 2 * align_up((size_t)pl.n_req * c.d_model * elem_size(c.dtype));
}

inline int hip_status(hipError_t e) { return e == hipSuccess ? VFM_OK : VFM_ERR_HIP; }

#define VFM_TRY(expr)              \
  do {                             \
    int _st = (expr);              \
    if (_st != VFM_OK) return _st; \
  } while (0)
#define VFM_HIP(expr)                               \
  do {                                              \
    hipError_t _e = (expr);                         \
    if (_e != hipSuccess) return VFM_ERR_HIP;       \
  } while (0)
// a launch bracketed by the optional timing hooks
#define VFM_TIMED(cls, expr)                        \
  do {                                              \
    const int _pi = prof_begin((cls), s);           \
    hipError_t _e = (expr);                         \
    prof_end(_pi, s);                               \
    if (_e != hipSuccess) return VFM_ERR_HIP;       \
  } while (0)

}  // namespace

extern "C" const char* vfm_status_string(int status) {
  switch (status) {
    case VFM_OK: return "ok";
    case VFM_ERR_ARG: return "invalid argument (null pointer or bad enum)";
    case VFM_ERR_SHAPE: return "inconsistent or unsupported sizes";
    case VFM_ERR_TASK: return "task id out of range";
    case VFM_ERR_UNSUPPORTED: return "configuration not supported by the library";
    case VFM_ERR_WORKSPACE: return "workspace missing or too small";
    case VFM_ERR_HIP: return "HIP runtime error";
  }
  return "unknown status";
}

extern "C" int vfm_workspace_size(const vfm_cfg* cfg, const vfm_batch* batch,
                                  const vfm_lora_table* lora, size_t* bytes) {
  if (!bytes) return VFM_ERR_ARG;
  VFM_TRY(check_cfg(cfg));
  Plan pl;
  VFM_TRY(check_batch(batch, &pl));
  VFM_TRY(check_lora(lora, pl));
  size_t need = layer_ws(*cfg, pl, lora, max_keys_of(batch, pl)).total;
  need = std::max(need, head_ws(*cfg, pl));
  *bytes = need;
  return VFM_OK;
}

extern "C" int vfm_embed_forward(const vfm_cfg* cfg, const vfm_batch* batch, int32_t mode,
                                 const void* src, int32_t src_width, const void* table,
                                 const void* bias, float* x, void* stream) {
  VFM_TRY(check_cfg(cfg));
  Plan pl;
  VFM_TRY(check_batch(batch, &pl));
  if (!src || !x) return VFM_ERR_ARG;
  if (mode == VFM_EMBED_TOKENS) {
    if (!table) return VFM_ERR_ARG;
    if (src_width < 1) return VFM_ERR_SHAPE;
  } else if (mode == VFM_EMBED_PATCHES) {
    if (!table) return VFM_ERR_ARG;
    if (src_width < 1 || src_width > 64) return VFM_ERR_SHAPE;
  } else if (mode != VFM_EMBED_ROWS) {
    return VFM_ERR_ARG;
  }
  return hip_status(launch_embed(cfg->dtype, pl, mode, src, src_width, table, bias, cfg->d_model, x,
                                 (hipStream_t)stream));
}

namespace {

// A paged cache's pool and tables.
int check_pool(const vfm_kv_pages* kv) {
  if (!kv || !kv->k || !kv->v || !kv->table_host || !kv->table_dev) return VFM_ERR_ARG;
  const int ps = kv->page_size;
  if (ps < 16 || ps > 1024 || (ps & (ps - 1))) return VFM_ERR_ARG;
  if (kv->n_pages < 1 || kv->max_pages < 1 || kv->n_pages > ((int64_t)1 << 40) / ps) return VFM_ERR_SHAPE;
  return VFM_OK;
}

KvPages pages_of(const vfm_kv_pages* kv) {
  int lp = 0;
  while ((1 << lp) < kv->page_size) ++lp;
  return KvPages{kv->table_dev, kv->max_pages, lp};
}

// ---- decoding over a bounded cache (vfm_decode.h) ----------------------------
constexpr int kMaxPos = 1 << 30;
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1;   // of a launch

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// The stream belongs to the current device (the one the kernels' code is loaded on).
int check_stream(void* stream) {
  if (stream == nullptr) return VFM_OK;
  int dev = -1;
  hipDevice_t sdev = -1;
  if (hipGetDevice(&dev) != hipSuccess || hipStreamGetDevice((hipStream_t)stream, &sdev) != hipSuccess) {
    (void)hipGetLastError();               // reported here, not by the next launch
    return VFM_ERR_HIP;
  }
  return sdev == dev ? VFM_OK : VFM_ERR_ARG;
}

int check_attn(const vfm_attn* a) {
  if (!a) return VFM_ERR_ARG;
  if (a->dtype != VFM_F32 && a->dtype != VFM_BF16) return VFM_ERR_ARG;
  if (a->head_dim != 64 && a->head_dim != 128) return VFM_ERR_UNSUPPORTED;
  if (a->n_heads < 1 || a->n_heads > 1024 || a->n_kv_heads < 1 || a->n_heads % a->n_kv_heads) return VFM_ERR_SHAPE;
  if (a->n_heads / a->n_kv_heads > 64) return VFM_ERR_UNSUPPORTED;
  if (a->window < 0 || a->window > kMaxPos || a->n_sink < 0 || a->n_sink > kMaxPos) return VFM_ERR_ARG;
  if (!(a->scale >= 0.f && a->scale <= 1e30f) || !(a->rope_theta >= 0.f && a->rope_theta <= 1e30f)) return VFM_ERR_ARG;
  return VFM_OK;
}

// The pages that a step uses exist: those of each request's new positions
// (writes) and, with `reads`, those with a position that one of its rows sees.
int check_pages(const vfm_attn& a, const vfm_batch* batch, const Plan& pl, const vfm_kv_pages* kv, bool reads) {
  const int64_t ps = kv->page_size;
  if (!aligned16(kv->k) || !aligned16(kv->v)) return VFM_ERR_ARG;
  if (kv->n_pages * ps >= (int64_t)1 << 31) return VFM_ERR_SHAPE;
  const PlanOffsets po = plan_offsets(pl.n_req, pl.n_tasks, pl.T);
  const int32_t *ctx = host_arr(batch, po.ctx), *cu = host_arr(batch, po.cu_seqlens), *order = host_arr(batch, po.order);
  for (int p = 0; p < pl.n_req; ++p) {
    const int64_t end = (int64_t)ctx[p] + (cu[p + 1] - cu[p]);
    if (ctx[p] < 0 || end > kMaxPos) return VFM_ERR_SHAPE;
    const int64_t last = (end - 1) / ps;
    if (last >= kv->max_pages) return VFM_ERR_SHAPE;
    const int32_t* row = kv->table_host + (int64_t)order[p] * kv->max_pages;
    int64_t first = ctx[p];                               // the window's (or the new rows') first position
    if (reads) first = a.window > 0 ? std::max<int64_t>(0, (int64_t)ctx[p] - a.window + 1) : 0;
    for (int64_t j = first / ps; j <= last; ++j)
      if (row[j] < 0 || row[j] >= kv->n_pages) return VFM_ERR_SHAPE;
    if (reads && a.window > 0) {
      const int64_t sinks = std::min<int64_t>(a.n_sink, end);
      for (int64_t j = 0; j * ps < sinks; ++j)
        if (row[j] < 0 || row[j] >= kv->n_pages) return VFM_ERR_SHAPE;
    }
  }
  return VFM_OK;
}

// One request with a long context makes most blocks of a rectangle empty, and most of its records unused.  A table
// of where each request's own begin costs a launch before the attention's and a search per block: it pays from some
// 2500 empty blocks on where they are two in three.  Rows of 32 heads of 128 beside one of 30000 keys: 128 short
// ones on 32 key heads 216 us, with the table 187 (33024 blocks, 4352 of them with work), on 8 130 and 59
// (33024, 1280), on 1 of 8 heads 38 and 26 (9417, 201); 8 short ones and 8 of 8000 keys on 8 56.5 and 58.4 (2560, 1344),
// and 256 rows of 200 to 2000 keys, 16 heads of 64, 194 and 198 (20480, 10608).
// Records are kept to their own from 16 MB of unused ones on whatever the time (22.5 us and 24.7 for 300 rows beside
// one after 8000 keys and two shorter: 101 MB and 0.4).
constexpr int64_t TABLE_MIN_EMPTY = 2500;
constexpr int64_t TABLE_MIN_BYTES = 16 << 20;

// Launch facts of the paged attention over a batch.
struct AttnPlan {
  int few_chunks, rows_chunks, qtiles;
  bool one;                  // no few-row request has more than 4 tiles of keys
  bool single, other;        // requests of a single row (single_row), and others
  bool table;                // blocks and records where each request's own begin, not in rectangles
  int64_t few_blocks, rows_blocks, recs, joins;
  int64_t bytes;             // workspace
  int64_t few_own, few_tiles;    // few-row blocks with work, and the 32-key tiles of all of them
  int nchunk() const { return std::max(few_chunks, rows_chunks); }
  bool deep() const { return few_blocks <= 512 || few_tiles >= 64 * few_own; }
  size_t table_bytes(const Plan& pl) const { return table ? align_up((size_t)4 * (pl.n_req + 1) * sizeof(int32_t)) : 0; }
};

// kv8: over a cache in 8 bits
int plan_attention(const vfm_attn& a, const vfm_batch* batch, const Plan& pl, bool kv8, AttnPlan* out) {
  AttnPlan ap = {};
  ap.few_chunks = ap.rows_chunks = ap.qtiles = 1;
  ap.one = true;
  const int G = a.n_heads / a.n_kv_heads;
  const PlanOffsets po = plan_offsets(pl.n_req, pl.n_tasks, pl.T);
  const int32_t *ctx = host_arr(batch, po.ctx), *cu = host_arr(batch, po.cu_seqlens);
  int64_t own[4] = {};       // the requests' own blocks, records and joins
  for (int p = 0; p < pl.n_req; ++p) {
    const int m = cu[p + 1] - cu[p];
    if (ctx[p] < 0 || (int64_t)ctx[p] + m > kMaxPos) return VFM_ERR_SHAPE;
    const Chunks ck = request_chunks(a.dtype, m, ctx[p], G, a.n_kv_heads, a.window, a.n_sink, kv8);
    const int n = ck.n;
    const AttnCounts c = request_counts(a.dtype, m, a.n_heads, a.n_kv_heads, n);
    for (int i = 0; i < 4; ++i) own[i] += c.v[i];
    (single_row(m, G, visible_runs<4>(ctx[p], ctx[p] + m - 1, a.window, a.n_sink).n) ? ap.single : ap.other) = true;
    if (few_rows(a.dtype, m, G)) {
      ap.one = ap.one && n * ck.tiles <= 4;
      ap.few_own += c.v[TAB_FEW];
      ap.few_tiles += c.v[TAB_FEW] * ck.tiles;
      ap.few_chunks = std::max(ap.few_chunks, n);
      if (a.dtype == VFM_BF16) ap.qtiles = std::max(ap.qtiles, (int)few_qtiles(m, G));
    } else {
      ap.rows_chunks = std::max(ap.rows_chunks, n);
    }
  }
  const int64_t few_tiles = a.dtype == VFM_BF16 ? (int64_t)ap.qtiles * pl.n_req : (int64_t)pl.T * G / 16 + pl.n_req;
  const int64_t rows_tiles = (int64_t)pl.T / rows_per_block(G) + pl.n_req;
  ap.few_blocks = own[TAB_FEW] > 0 ? few_tiles * a.n_kv_heads * ap.few_chunks : 0;
  ap.rows_blocks = own[TAB_ROWS] > 0 ? rows_tiles * a.n_kv_heads * ap.rows_chunks : 0;
  const bool cut = own[TAB_RECS] > 0;
  ap.joins = cut ? (int64_t)pl.T * a.n_heads : 0;
  ap.recs = ap.joins * ap.nchunk();
  const int64_t most = kMaxThreads / 256;                 // blocks
  const int64_t rec_bytes = a.head_dim * 4 + 8;
  const int64_t blocks = ap.few_blocks + ap.rows_blocks, with_work = own[TAB_FEW] + own[TAB_ROWS];
  ap.table = blocks > most || (cut && ((blocks > 3 * with_work && blocks - with_work > TABLE_MIN_EMPTY) ||
                                       (ap.recs - 2 * own[TAB_RECS]) * rec_bytes > TABLE_MIN_BYTES ||
                                       ap.joins / 4 >= most));
  if (ap.table) {
    ap.few_blocks = own[TAB_FEW];
    ap.rows_blocks = own[TAB_ROWS];
    ap.recs = own[TAB_RECS];
    ap.joins = own[TAB_JOIN];
  }
  if (ap.few_blocks + ap.rows_blocks > most || ap.joins / 4 >= most || (ap.table && ap.recs > INT32_MAX)) return VFM_ERR_UNSUPPORTED;
  if (cut || ap.table)
    ap.bytes = (int64_t)ap.table_bytes(pl) + (int64_t)align_up((size_t)ap.recs * a.head_dim * 4) +
               (int64_t)align_up((size_t)ap.recs * 8);
  *out = ap;
  return VFM_OK;
}

// exps: k and v are codes with these exponents (vfm_kv8.h), or NULL
hipError_t run_attention(const vfm_attn& a, const Plan& pl, const AttnPlan& ap, const void* q, int64_t ldq, const void* k,
                         const void* v, const uint8_t* exps, int64_t slots, const KvPages& kp, void* out, int64_t ldo,
                         char* ws, hipStream_t s) {
  PagedAttn p = {};
  p.H = (int16_t)a.n_heads; p.KH = (int16_t)a.n_kv_heads; p.G = a.n_heads / a.n_kv_heads;
  p.kv8 = exps != nullptr;
  p.window = a.window; p.n_sink = a.window > 0 ? a.n_sink : 0;
  p.scale_log2 = (a.scale > 0.f ? a.scale : 1.f / sqrtf((float)a.head_dim)) * 1.4426950408889634f;
  p.q = q; p.ldq = ldq; p.k = k; p.v = v; p.slots = slots; p.kp = kp; p.out = out; p.ldo = ldo;
  if (ap.table) {
    p.table = (const int32_t*)ws;
  } else {
    p.few_chunks = ap.few_chunks; p.rows_chunks = ap.rows_chunks; p.nchunk = ap.nchunk(); p.qtiles = ap.qtiles;
  }
  if (ap.joins > 0) {
    p.rec_o = (float*)(ws + ap.table_bytes(pl));
    p.rec_ml = (float2*)((char*)p.rec_o + align_up((size_t)ap.recs * a.head_dim * 4));
  }
  if (exps != nullptr)
    return launch_attention8(a.dtype, a.head_dim, pl, p, exps, ap.few_blocks, ap.rows_blocks, ap.joins, ap.deep(), ap.single, ap.other, ap.table, s);
  return launch_attention_paged(a.dtype, a.head_dim, pl, p, ap.few_blocks, ap.rows_blocks, ap.joins, ap.one,
                                ap.table, s);
}

vfm_attn attn_of_layer(const vfm_cfg& c, int32_t window, int32_t n_sink) {
  vfm_attn a = {};
  a.dtype = c.dtype; a.n_heads = a.n_kv_heads = c.n_heads; a.head_dim = c.head_dim;
  a.window = window; a.n_sink = n_sink;
  return a;
}

// Checks shared by the layer entry points (everything but the cache).
int check_layer(const vfm_cfg* cfg, const vfm_layer_weights* w, const vfm_lora_table* lora,
                const vfm_batch* batch, const float* x, bool have_cache, Plan* pl, bool windowed = false) {
  VFM_TRY(check_cfg(cfg));
  VFM_TRY(check_batch(batch, pl));
  VFM_TRY(check_lora(lora, *pl));
  if (!w || !x) return VFM_ERR_ARG;
  if (!w->norm1_w || !w->norm2_w || !w->w_qkv || !w->w_o || !w->w_up || !w->w_down)
    return VFM_ERR_ARG;
  if (cfg->mlp == VFM_MLP_SWIGLU && !w->w_gate) return VFM_ERR_ARG;
  if (cfg->attn == VFM_ATTN_DECODE || cfg->attn == VFM_ATTN_MIXED) {
    if (!have_cache) return VFM_ERR_ARG;
  }
  if (cfg->attn == VFM_ATTN_DECODE && pl->max_seqlen != 1) return VFM_ERR_UNSUPPORTED;
  const PlanOffsets po = plan_offsets(pl->n_req, pl->n_tasks, pl->T);
  if (cfg->attn == VFM_ATTN_BIDIR || cfg->attn == VFM_ATTN_CAUSAL) {
    // these steps attend over a request's own rows only: cached tokens
    // before them would be ignored, so a request with ctx > 0 is refused
    const int32_t* ctx = host_arr(batch, po.ctx);
    for (int p = 0; p < pl->n_req; ++p)
      if (ctx[p] > 0) return VFM_ERR_UNSUPPORTED;
  }
  if (cfg->attn == VFM_ATTN_MIXED && cfg->dtype != VFM_BF16 && !windowed) {   // prompt chunks after cached tokens: bf16
    const int32_t* ctx = host_arr(batch, po.ctx);
    const int32_t* cu = host_arr(batch, po.cu_seqlens);
    for (int p = 0; p < pl->n_req; ++p)
      if (ctx[p] > 0 && cu[p + 1] - cu[p] != 1) return VFM_ERR_UNSUPPORTED;
  }
  return VFM_OK;
}

// win: attention over the paged cache with a window and sinks (vfm_layer_forward_windowed), or NULL; exps: with it, the
// cache is held in 8 bits under these exponents (vfm_layer_forward_q8).
int layer_impl(const vfm_cfg& c, const vfm_layer_weights* w, const vfm_lora_table* lora,
               const vfm_batch* batch, const Plan& pl, float* x, void* k_cache, void* v_cache,
               int64_t kv_slots, const KvPages& kp, void* workspace, size_t ws_bytes, void* stream,
               const vfm_attn* win = nullptr, uint8_t* exps = nullptr);

}  // namespace

namespace {

// Checks of the contiguous-cache layer call: check_layer plus the cache's
// bounds (host copy of the plan).
int check_layer_contiguous(const vfm_cfg* cfg, const vfm_layer_weights* w, const vfm_lora_table* lora,
                           const vfm_batch* batch, const float* x, const void* k_cache,
                           const void* v_cache, int64_t kv_slots, Plan* pl) {
  if ((k_cache != nullptr) != (v_cache != nullptr)) return VFM_ERR_ARG;
  VFM_TRY(check_layer(cfg, w, lora, batch, x, k_cache != nullptr, pl));
  if (k_cache) {
    const PlanOffsets po = plan_offsets(pl->n_req, pl->n_tasks, pl->T);
    const int32_t* ctx = host_arr(batch, po.ctx);
    const int32_t* kvs = host_arr(batch, po.kv_start);
    const int32_t* cu = host_arr(batch, po.cu_seqlens);
    for (int p = 0; p < pl->n_req; ++p) {
      const int64_t end = (int64_t)kvs[p] + ctx[p] + (cu[p + 1] - cu[p]);
      if (end > kv_slots) return VFM_ERR_SHAPE;
    }
  }
  return VFM_OK;
}

}  // namespace

extern "C" int vfm_layer_forward(const vfm_cfg* cfg, const vfm_layer_weights* w,
                                 const vfm_lora_table* lora, const vfm_batch* batch, float* x,
                                 void* k_cache, void* v_cache, int64_t kv_slots, void* workspace,
                                 size_t ws_bytes, void* stream) {
  Plan pl;
  VFM_TRY(check_layer_contiguous(cfg, w, lora, batch, x, k_cache, v_cache, kv_slots, &pl));
  return layer_impl(*cfg, w, lora, batch, pl, x, k_cache, v_cache, kv_slots, KvPages{nullptr, 0, 0},
                    workspace, ws_bytes, stream);
}

// ---- the allocation-free layer call ----------------------------------------
namespace {

// Workspace of vfm_layer_forward_noalloc.  Every GPU the library runs on
// holds its own copy of this array, at its own address, until the process
// ends.  In host code `scratch` names a host-side stand-in, not the device
// memory: host code uses only the device address hipGetSymbolAddress returns
// for the current device (kept per device below), never the name itself.
static __device__ __align__(256) unsigned char scratch[VFM_NOALLOC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_dev[kMaxDevices] = {};

// Device address of the current device's scratch array, looked up once per
// device (with that device current) on its first call.  The stream must
// belong to the current device, since the address is that device's.
int scratch_of_current_device(hipStream_t s, void** out) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return VFM_ERR_HIP;
  if (dev < 0 || dev >= kMaxDevices) return VFM_ERR_UNSUPPORTED;
  if (s != nullptr) {
    hipDevice_t sdev = -1;
    if (hipStreamGetDevice(s, &sdev) != hipSuccess) return VFM_ERR_HIP;
    if (sdev != dev) return VFM_ERR_ARG;
  }
  std::lock_guard<std::mutex> lk(g_scratch_mu);
  if (g_scratch_dev[dev] == nullptr) {
    void* p = nullptr;
    if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || p == nullptr) return VFM_ERR_HIP;
    g_scratch_dev[dev] = p;
  }
  *out = g_scratch_dev[dev];
  return VFM_OK;
}

}  // namespace

extern "C" int vfm_layer_forward_noalloc(const vfm_cfg* cfg, const vfm_layer_weights* w,
                                         const vfm_lora_table* lora, const vfm_batch* batch, float* x,
                                         void* k_cache, void* v_cache, int64_t kv_slots, void* stream) {
  Plan pl;
  VFM_TRY(check_layer_contiguous(cfg, w, lora, batch, x, k_cache, v_cache, kv_slots, &pl));
  // the batch's workspace must fit the fixed scratch array (checked on the
  // host, before the device is touched)
  if (layer_ws(*cfg, pl, lora, max_keys_of(batch, pl)).total > VFM_NOALLOC_SCRATCH_BYTES)
    return VFM_ERR_WORKSPACE;
  void* ws = nullptr;
  VFM_TRY(scratch_of_current_device((hipStream_t)stream, &ws));
  // nothing in the scratch array needs to start at zero: every kernel writes
  // the workspace regions it reads in the same call (stale bytes of an
  // earlier call are never read)
  return layer_impl(*cfg, w, lora, batch, pl, x, k_cache, v_cache, kv_slots, KvPages{nullptr, 0, 0}, ws,
                    VFM_NOALLOC_SCRATCH_BYTES, stream);
}

extern "C" int vfm_layer_forward_paged(const vfm_cfg* cfg, const vfm_layer_weights* w,
                                       const vfm_lora_table* lora, const vfm_batch* batch, float* x,
                                       const vfm_kv_pages* kv, void* workspace, size_t ws_bytes,
                                       void* stream) {
  VFM_TRY(check_pool(kv));
  const int ps = kv->page_size;
  Plan pl;
  VFM_TRY(check_layer(cfg, w, lora, batch, x, true, &pl));
  if (cfg->attn == VFM_ATTN_BIDIR) return VFM_ERR_UNSUPPORTED;
  // every page a request uses (ctx + len tokens) exists
  const PlanOffsets po = plan_offsets(pl.n_req, pl.n_tasks, pl.T);
  const int32_t* ctx = host_arr(batch, po.ctx);
  const int32_t* cu = host_arr(batch, po.cu_seqlens);
  const int32_t* order = host_arr(batch, po.order);
  for (int p = 0; p < pl.n_req; ++p) {
    const int64_t need = ((int64_t)ctx[p] + (cu[p + 1] - cu[p]) + ps - 1) / ps;
    if (need > kv->max_pages) return VFM_ERR_SHAPE;
    const int32_t* row = kv->table_host + (int64_t)order[p] * kv->max_pages;
    for (int64_t j = 0; j < need; ++j)
      if (row[j] < 0 || row[j] >= kv->n_pages) return VFM_ERR_SHAPE;
  }
  return layer_impl(*cfg, w, lora, batch, pl, x, kv->k, kv->v, kv->n_pages * ps, pages_of(kv), workspace, ws_bytes,
                    stream);
}

namespace {

int layer_impl(const vfm_cfg& c, const vfm_layer_weights* w, const vfm_lora_table* lora,
               const vfm_batch* batch, const Plan& pl, float* x, void* k_cache, void* v_cache,
               int64_t kv_slots, const KvPages& kp, void* workspace, size_t ws_bytes, void* stream,
               const vfm_attn* win, uint8_t* exps) {
  const int d = c.d_model, f = c.d_ff, T = pl.T;
  const int max_keys = max_keys_of(batch, pl);
  AttnPlan ap = {};
  if (win) VFM_TRY(plan_attention(*win, batch, pl, exps != nullptr, &ap));
  const LayerWs ws = win ? layer_ws(c, pl, lora, 0, ap.bytes) : layer_ws(c, pl, lora, max_keys);
  if (!workspace || ws_bytes < ws.total || ((uintptr_t)workspace % ALIGN)) return VFM_ERR_WORKSPACE;

  hipStream_t s = (hipStream_t)stream;
  char* base = (char*)workspace;
  void* h = base + ws.h;
  void* qkv = base + ws.big;
  void* act = base + ws.big;  // the MLP activation reuses the qkv region
  void* attn = base + ws.attn;
  void* U = base + ws.u;
  float* Z = (float*)(base + ws.z);
  float* P = (float*)(base + ws.p);
  const int rpad = rpad_of(lora);
  const int ldu = 8 * rpad;  // 7 projections + one spare slot
  const bool use_lora = lora && rpad > 0;

  const bool skinny = use_skinny(c, pl);
  const bool direct = c.attn == VFM_ATTN_BIDIR;   // see VFM_DIRECT_K

  auto has = [&](int p) { return use_lora && lora->A[p] != nullptr; };
  // One projection group: X [T, K] times the stacked weights (W, then W2
  // for SwiGLU), the per-task LoRA of `projs` (column slots of slot_width),
  // and the epilogue.
  // norm_into: for a residual projection, the pre-norm that follows it (its
  // output buffer); the small-batch path then fuses the two, and the caller
  // skips its own norm launch when `fused_norm` comes back true
  bool fused_norm = false;
  // set for the QKV projection of a small batch: the finalize applies RoPE
  // (and the cache write) itself
  FinRope fin_rope = {};
  // set for the QKV projection of a large bf16 batch: the GEMM applies RoPE
  GemmRope gemm_rope = {};
  auto project = [&](int cls, const void* X, int K, const void* W, const void* W2,
                     const void* bias, int N, int epi, void* out, int ldo,
                     std::initializer_list<int> projs, int slot_width, const void* norm_g = nullptr,
                     const void* norm_b = nullptr, void* norm_into = nullptr) -> int {
    fused_norm = false;
    bool any = false;
    for (int p : projs) any = any || has(p);
    // (with RoPE, the QKV projection of a small batch stays on the split path,
    // whose finalize rotates before the one rounding to bf16)
    if (!skinny || (direct && K <= VFM_DIRECT_K && !fin_rope.on)) {
      if (any) {
        ShrinkArgs a = {};
        a.X = X; a.ldx = K; a.K = K; a.U = U; a.ldu = ldu; a.rpad = rpad;
        a.rank = lora->rank; a.scale = lora->scale;
        a.nsub = std::min(std::max(1, (lora->max_rank + 15) / 16), rpad / 16);
        for (int p : projs) {
          if (!has(p)) continue;
          a.A[a.n_proj] = lora->A[p];
          a.ucol[a.n_proj] = p * rpad;
          a.n_proj++;
        }
        VFM_TIMED(VFM_PROF_SHRINK, launch_lora_shrink(c.dtype, pl, a, s));
      }
      GemmArgs g = {};
      g.X = X; g.ldx = K; g.W = W; g.W2 = W2; g.bias = bias;
      g.M = T; g.N = N; g.K = K; g.epi = epi; g.out = out; g.ldo = ldo;
      g.rope = gemm_rope;
      if (any) {
        GemmLora& L = g.lora;
        int i = 0;
        for (int p : projs) {
          if (has(p)) L.B[i] = lora->B[p];
          L.ucol[i] = p * rpad;
          ++i;
        }
        L.enabled = 1;
        L.U = U; L.ldu = ldu; L.slot_width = slot_width;
        L.rank = lora->rank; L.row_task = pl.row_task; L.seg_row = pl.seg_row;
        L.max_rank = lora->max_rank;
      }
      VFM_TIMED(cls, launch_gemm(c.dtype, g, s));
      return VFM_OK;
    }
    // small batch: split-K shrink, split-K GEMM into partial slices, then
    // the streaming sum, which also reduces the shrink partials and adds
    // each row's LoRA difference
    const bool sw = epi == EPI_SWIGLU;
    const int nz = sw ? 2 * N : N;
    SkinnyArgs k = {};
    k.X = X; k.ldx = K; k.W = W; k.W2 = W2; k.n_half = N;
    k.M = T; k.N = nz; k.K = K; k.Z = Z;
    k.nsplit = skinny_splits(nz, K);
    FinalizeArgs fa = {};
    fa.Z = Z; fa.nslices = skinny_slices(T, nz, K); fa.M = T; fa.N = N; fa.epi = epi; fa.bias = bias;
    fa.out = out; fa.ldo = ldo;
    fa.rope = fin_rope;
    if (any) {
      // the split shrink writes fp32 partials; the finalize pass sums them
      // into each row's U and adds U B_t^T to the row's columns
      ShrinkSplitArgs a = {};
      a.X = X; a.ldx = K; a.K = K; a.P = P; a.ldp = ldu; a.rpad = rpad;
      a.kchunk = SHRINK_CHUNK; a.kchunks = shrink_chunks(K); a.rank = lora->rank;
      a.nsub = std::min(std::max(1, (lora->max_rank + 15) / 16), rpad / 16);
      for (int p : projs) {
        if (!has(p)) continue;
        a.A[a.n_proj] = lora->A[p];
        a.ucol[a.n_proj] = p * rpad;
        a.n_proj++;
      }
      if (skinny_takes_shrink(T)) { k.sh = a; k.pl = pl; }
      else VFM_TIMED(VFM_PROF_SHRINK, launch_shrink_split(pl, a, s));
      FinLora& fl = fa.lora;
      fl.enabled = 1;
      fl.P = P; fl.ldp = ldu; fl.cstride = (int64_t)T * ldu; fl.kchunks = a.kchunks;
      int i = 0;
      for (int p : projs) {
        fl.ucol[i] = p * rpad;
        fl.B[i] = has(p) ? lora->B[p] : nullptr;
        ++i;
      }
      fl.n_slots = i; fl.rpad = rpad;
      fl.slot_width = sw ? N : slot_width;
      fl.scale = lora->scale; fl.rank = lora->rank; fl.max_rank = lora->max_rank;
      fl.row_task = pl.row_task;
    }
    const int pi = prof_begin(cls, s);
    hipError_t e = launch_gemm_skinny(k, s);
    const bool fuse = norm_into != nullptr && epi == EPI_RESID && c.dtype == VFM_BF16 && ldo == N && N <= 8192;
    if (e == hipSuccess)
      e = fuse ? launch_finalize_norm(c.dtype, fa, norm_g, norm_b, c.norm, c.norm_eps, norm_into, s)
               : launch_finalize(fa, s);
    prof_end(pi, s);
    fused_norm = fuse && e == hipSuccess;
    return hip_status(e);
  };

  // a2: pre-norm 1
  VFM_TIMED(VFM_PROF_NORM, launch_norm(c.dtype, x, T, d, w->norm1_w, w->norm1_b, c.norm, c.norm_eps, h, s));
  // a5 (small bf16 batches): the QKV finalize also applies the rotary
  // embedding of q and k and, with a KV cache, writes each row's rotated k
  // and its v to its slot
  // (large bf16 batches): the QKV GEMM's store pass rotates q and k, and the
  // cache write is the attention launcher's plain copy
  const bool cache_write = k_cache != nullptr && c.attn != VFM_ATTN_BIDIR;
  // (windowed: the append pass, whose angles hold at any position; see below)
  const bool rope_fusable = !win && c.dtype == VFM_BF16 && c.rope_theta > 0.f &&
                            (c.head_dim == 64 || c.head_dim == 128) && d % 256 == 0;
  const bool rope_in_finalize = skinny && rope_fusable;
  const bool rope_in_gemm = !skinny && rope_fusable && T >= 1024 &&
                            (int64_t)T * d < ((int64_t)1 << 31) && (int64_t)3 * d * d < ((int64_t)1 << 31);
  const bool rope_writes_kv = !win && c.rope_theta > 0.f && cache_write && !rope_in_gemm;
  if (rope_in_gemm) {
    gemm_rope.on = 1; gemm_rope.d = d; gemm_rope.head_dim = c.head_dim;
    gemm_rope.log2_theta = log2f(c.rope_theta); gemm_rope.pos = pl.pos;
  }
  if (rope_in_finalize) {
    fin_rope.on = 1; fin_rope.d = d; fin_rope.head_dim = c.head_dim; fin_rope.log2_theta = log2f(c.rope_theta);
    fin_rope.pl = pl; fin_rope.kp = kp; fin_rope.kv_slots = kv_slots;
    fin_rope.kc = rope_writes_kv ? (bf16*)k_cache : nullptr;
    fin_rope.vc = rope_writes_kv ? (bf16*)v_cache : nullptr;
  }
  // a3 + a4: shared QKV projection with the per-task LoRA of q, k, v
  VFM_TRY(project(VFM_PROF_GEMM_QKV, h, d, w->w_qkv, nullptr, w->b_qkv, 3 * d, EPI_STORE, qkv,
                  3 * d, {VFM_Q, VFM_K, VFM_V}, d));
  fin_rope = FinRope{};
  gemm_rope = GemmRope{};
  // a5: rotary embedding of q and k
  // (with a KV cache the same pass writes each row's rotated k and its v)
  if (!win && c.rope_theta > 0.f && !rope_in_finalize && !rope_in_gemm)
    VFM_TIMED(VFM_PROF_OTHER, launch_rope(c.dtype, pl, qkv, d, c.n_heads, c.head_dim, c.rope_theta,
                                          rope_writes_kv ? k_cache : nullptr, rope_writes_kv ? v_cache : nullptr,
                                          kv_slots, kp, s));
  // a6: attention per request (and the KV-cache write)
  // (timed per kernel inside the launcher)
  if (win) {
    // Rotation in place and cache write in one pass: a sequence that keeps a window of its past goes on to
    // positions at which an angle in fp32 is off (position 700: by up to 4e-5, position 10^6: by 0.06).
    void* const q_out = c.rope_theta > 0.f ? qkv : nullptr;
    if (exps) {
      const Pool8 pool = {(uint8_t*)k_cache, (uint8_t*)v_cache, exps, kv_slots};
      VFM_TIMED(VFM_PROF_OTHER, launch_append8(c.dtype, pl, c.n_heads, c.n_heads, c.head_dim, c.rope_theta, qkv,
                                               3 * (int64_t)d, q_out, 3 * (int64_t)d, pool, kp, s));
    } else {
      VFM_TIMED(VFM_PROF_OTHER, launch_kv_append(c.dtype, pl, c.n_heads, c.n_heads, c.head_dim, c.rope_theta, qkv,
                                                 3 * (int64_t)d, q_out, 3 * (int64_t)d, k_cache, v_cache, kv_slots, kp, s));
    }
    VFM_HIP(run_attention(*win, pl, ap, qkv, 3 * (int64_t)d, k_cache, v_cache, exps, kv_slots, kp, attn, d,
                          base + ws.aws, s));
  }
  bool chunked = false;                      // a prompt chunk after cached tokens
  if (!win && c.attn == VFM_ATTN_MIXED) {
    const PlanOffsets po = plan_offsets(pl.n_req, pl.n_tasks, pl.T);
    const int32_t* ctx = host_arr(batch, po.ctx);
    const int32_t* cu = host_arr(batch, po.cu_seqlens);
    for (int p = 0; p < pl.n_req && !chunked; ++p) chunked = ctx[p] > 0 && cu[p + 1] - cu[p] > 1;
  }
  if (!win) VFM_HIP(launch_attention(c.dtype, pl, c, qkv, attn, k_cache, v_cache, kv_slots, kp, rope_writes_kv, chunked,
                           base + ws.aws, ws.z - ws.aws, max_keys, s));
  // a7: output projection + LoRA_o + residual
  VFM_TRY(project(VFM_PROF_GEMM_O, attn, d, w->w_o, nullptr, w->b_o, d, EPI_RESID, x, d, {VFM_O}, d,
                  w->norm2_w, w->norm2_b, h));
  // a8: pre-norm 2 (already done with the residual finalize on small batches)
  if (!fused_norm)
    VFM_TIMED(VFM_PROF_NORM, launch_norm(c.dtype, x, T, d, w->norm2_w, w->norm2_b, c.norm, c.norm_eps, h, s));
  // a9: MLP up (+ gate) with LoRA and the activation fused
  if (c.mlp == VFM_MLP_SWIGLU)
    VFM_TRY(project(VFM_PROF_GEMM_UP, h, d, w->w_gate, w->w_up, nullptr, f, EPI_SWIGLU, act, f,
                    {VFM_GATE, VFM_UP}, f));
  else
    VFM_TRY(project(VFM_PROF_GEMM_UP, h, d, w->w_up, nullptr, w->b_up, f, EPI_GELU, act, f,
                    {VFM_UP}, f));
  // a10: down projection + LoRA_down + residual
  VFM_TRY(project(VFM_PROF_GEMM_DOWN, act, f, w->w_down, nullptr, w->b_down, d, EPI_RESID, x, d,
                  {VFM_DOWN}, d));
  return VFM_OK;
}

}  // namespace

extern "C" int vfm_lora_apply(int32_t dtype, int32_t proj, int32_t d_in, int32_t d_out,
                              const vfm_lora_table* lora, const vfm_batch* batch, const void* x,
                              float* y, void* workspace, size_t ws_bytes, void* stream) {
  if (dtype != VFM_F32 && dtype != VFM_BF16) return VFM_ERR_ARG;
  if (proj < 0 || proj >= VFM_NPROJ) return VFM_ERR_ARG;
  if (!lora || !x || !y) return VFM_ERR_ARG;
  Plan pl;
  VFM_TRY(check_batch(batch, &pl));
  VFM_TRY(check_lora(lora, pl));
  if (!lora->A[proj]) return VFM_ERR_ARG;
  if (d_in < 64 || d_in % 64 || d_out < 4 || d_out % 4) return VFM_ERR_SHAPE;
  const int rpad = rpad_of(lora);
  if (rpad == 0) return VFM_OK;
  const size_t need = align_up((size_t)pl.T * rpad * elem_size(dtype));
  if (!workspace || ws_bytes < need || ((uintptr_t)workspace % ALIGN)) return VFM_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  ShrinkArgs a = {};
  a.X = x; a.ldx = d_in; a.K = d_in; a.U = workspace; a.ldu = rpad; a.rpad = rpad;
  a.rank = lora->rank; a.scale = lora->scale;
  a.nsub = std::min(std::max(1, (lora->max_rank + 15) / 16), rpad / 16);
  a.A[0] = lora->A[proj]; a.ucol[0] = 0; a.n_proj = 1;
  VFM_HIP(launch_lora_shrink(dtype, pl, a, s));
  ExpandArgs e = {};
  e.U = workspace; e.ldu = rpad; e.ucol = 0; e.B = lora->B[proj]; e.N = d_out;
  e.Y = y; e.ldy = d_out; e.rank = lora->rank; e.max_rank = lora->max_rank;
  VFM_HIP(launch_lora_expand(dtype, pl, e, s));
  return VFM_OK;
}

extern "C" int vfm_head_forward(const vfm_cfg* cfg, const void* final_norm_w,
                                const void* final_norm_b, const vfm_head_table* heads,
                                const vfm_batch* batch, const float* x, float* out,
                                void* workspace, size_t ws_bytes, void* stream) {
  VFM_TRY(check_cfg(cfg));
  Plan pl;
  VFM_TRY(check_batch(batch, &pl));
  if (!final_norm_w || !x || !out) return VFM_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  const vfm_cfg& c = *cfg;
  if (!heads) {
    return hip_status(launch_norm_pool(c.dtype, pl, x, c.d_model, final_norm_w, final_norm_b,
                                       c.norm, c.norm_eps, -1, nullptr, out, s));
  }
  if (heads->n_tasks != pl.n_tasks || !heads->n_out || !heads->W) return VFM_ERR_ARG;
  if (heads->pool < VFM_POOL_MEAN || heads->pool > VFM_POOL_LAST) return VFM_ERR_ARG;
  if (heads->max_out < 0) return VFM_ERR_SHAPE;
  if (heads->W1) {
    if (heads->hidden < 64 || heads->hidden % 64 || heads->hidden > c.d_model) return VFM_ERR_SHAPE;
    if (heads->act != VFM_ACT_GELU && heads->act != VFM_ACT_RELU) return VFM_ERR_ARG;
  }
  if ((size_t)c.d_model * elem_size(c.dtype) > 64 * 1024) return VFM_ERR_UNSUPPORTED;
  const size_t need = head_ws(c, pl);
  if (!workspace || ws_bytes < need || ((uintptr_t)workspace % ALIGN)) return VFM_ERR_WORKSPACE;
  VFM_HIP(launch_norm_pool(c.dtype, pl, x, c.d_model, final_norm_w, final_norm_b, c.norm,
                           c.norm_eps, heads->pool, workspace, nullptr, s));
  VFM_HIP(launch_heads(c.dtype, pl, workspace, c.d_model, *heads, out, s));
  return VFM_OK;
}

extern "C" int vfm_greedy_tokens(const vfm_batch* batch, const float* out, int32_t* ids, void* stream) {
  Plan pl;
  VFM_TRY(check_batch(batch, &pl));
  if (!out || !ids) return VFM_ERR_ARG;
  return hip_status(launch_greedy(pl, out, ids, (hipStream_t)stream));
}

// ---- decoding over a bounded cache (vfm_decode.h) ----------------------------

namespace {

int workspace_windowed(const vfm_cfg* cfg, const vfm_batch* batch, const vfm_lora_table* lora, int32_t window,
                       int32_t n_sink, bool kv8, size_t* bytes) {
  if (!bytes) return VFM_ERR_ARG;
  VFM_TRY(check_cfg(cfg));
  const vfm_attn a = attn_of_layer(*cfg, window, n_sink);
  VFM_TRY(check_attn(&a));
  Plan pl;
  VFM_TRY(check_batch(batch, &pl));
  VFM_TRY(check_lora(lora, pl));
  AttnPlan ap;
  VFM_TRY(plan_attention(a, batch, pl, kv8, &ap));
  *bytes = std::max(layer_ws(*cfg, pl, lora, 0, ap.bytes).total, head_ws(*cfg, pl));
  return VFM_OK;
}

int workspace_attention(const vfm_attn* attn, const vfm_batch* batch, bool kv8, size_t* bytes) {
  if (!bytes) return VFM_ERR_ARG;
  VFM_TRY(check_attn(attn));
  Plan pl;
  VFM_TRY(check_batch(batch, &pl));
  AttnPlan ap;
  VFM_TRY(plan_attention(*attn, batch, pl, kv8, &ap));
  *bytes = (size_t)ap.bytes;
  return VFM_OK;
}

}  // namespace

extern "C" int vfm_workspace_size_windowed(const vfm_cfg* cfg, const vfm_batch* batch, const vfm_lora_table* lora,
                                           int32_t window, int32_t n_sink, size_t* bytes) {
  return workspace_windowed(cfg, batch, lora, window, n_sink, false, bytes);
}

namespace {

// A launch holds the append's blocks.
int check_append8(const Plan& pl) {
  return pl.n_req > APPEND8_MAX_BLOCKS - ((int64_t)pl.T + 15) / 16 ? VFM_ERR_UNSUPPORTED : VFM_OK;
}

// A layer over a paged cache, in 8 bits where exps is given.
int layer_windowed(const vfm_cfg* cfg, const vfm_layer_weights* w, const vfm_lora_table* lora, const vfm_batch* batch,
                   float* x, const vfm_kv_pages* kv, uint8_t* exps, int32_t window, int32_t n_sink, void* workspace,
                   size_t ws_bytes, void* stream) {
  VFM_TRY(check_pool(kv));
  Plan pl;
  VFM_TRY(check_layer(cfg, w, lora, batch, x, true, &pl, true));
  if (cfg->attn == VFM_ATTN_BIDIR) return VFM_ERR_UNSUPPORTED;
  const vfm_attn a = attn_of_layer(*cfg, window, n_sink);
  VFM_TRY(check_attn(&a));
  if ((int64_t)pl.T * APPEND_THREADS > kMaxThreads) return VFM_ERR_UNSUPPORTED;
  VFM_TRY(check_pages(a, batch, pl, kv, true));
  if (exps) VFM_TRY(check_append8(pl));
  VFM_TRY(check_stream(stream));
  return layer_impl(*cfg, w, lora, batch, pl, x, kv->k, kv->v, kv->n_pages * kv->page_size, pages_of(kv), workspace,
                    ws_bytes, stream, &a, exps);
}

// vfm_attention_paged and its form over 8 bits.
int attend_paged(const vfm_attn* attn, const vfm_batch* batch, const void* q, int64_t ldq, const vfm_kv_pages* kv,
                 const uint8_t* exps, void* out, int64_t ldo, void* workspace, size_t ws_bytes, void* stream) {
  VFM_TRY(check_attn(attn));
  VFM_TRY(check_pool(kv));
  Plan pl;
  VFM_TRY(check_batch(batch, &pl));
  if (!q || !out || !aligned16(q) || !aligned16(out)) return VFM_ERR_ARG;
  const int64_t cols = (int64_t)attn->n_heads * attn->head_dim;
  if (ldq % 8 || ldo % 8 || ldq < cols || ldo < cols) return VFM_ERR_SHAPE;
  VFM_TRY(check_pages(*attn, batch, pl, kv, true));
  AttnPlan ap;
  VFM_TRY(plan_attention(*attn, batch, pl, exps != nullptr, &ap));
  if (ap.bytes > 0 && (!workspace || ws_bytes < (size_t)ap.bytes || ((uintptr_t)workspace % ALIGN)))
    return VFM_ERR_WORKSPACE;
  VFM_TRY(check_stream(stream));
  VFM_HIP(run_attention(*attn, pl, ap, q, ldq, kv->k, kv->v, exps, kv->n_pages * kv->page_size, pages_of(kv), out, ldo,
                        (char*)workspace, (hipStream_t)stream));
  return VFM_OK;
}

// What the two appends check; the plan of the batch.
int check_append(const vfm_attn* attn, const vfm_batch* batch, const void* qkv, int64_t ld, const void* q_out,
                 const vfm_kv_pages* kv, void* stream, Plan* pl) {
  VFM_TRY(check_attn(attn));
  VFM_TRY(check_pool(kv));
  VFM_TRY(check_batch(batch, pl));
  if (!qkv || !q_out || !aligned16(qkv) || !aligned16(q_out)) return VFM_ERR_ARG;
  if (ld % 8 || ld < (int64_t)(attn->n_heads + 2 * attn->n_kv_heads) * attn->head_dim) return VFM_ERR_SHAPE;
  if ((int64_t)pl->T * APPEND_THREADS > kMaxThreads) return VFM_ERR_UNSUPPORTED;
  VFM_TRY(check_pages(*attn, batch, *pl, kv, false));
  return check_stream(stream);
}

int check_exps(const vfm_kv_pages_q8* kv) { return kv && kv->exps && aligned16(kv->exps) ? VFM_OK : VFM_ERR_ARG; }

}  // namespace

extern "C" int vfm_layer_forward_windowed(const vfm_cfg* cfg, const vfm_layer_weights* w, const vfm_lora_table* lora,
                                          const vfm_batch* batch, float* x, const vfm_kv_pages* kv, int32_t window,
                                          int32_t n_sink, void* workspace, size_t ws_bytes, void* stream) {
  return layer_windowed(cfg, w, lora, batch, x, kv, nullptr, window, n_sink, workspace, ws_bytes, stream);
}

extern "C" int vfm_kv_append(const vfm_attn* attn, const vfm_batch* batch, const void* qkv, int64_t ld, void* q_out,
                             const vfm_kv_pages* kv, void* stream) {
  Plan pl;
  VFM_TRY(check_append(attn, batch, qkv, ld, q_out, kv, stream, &pl));
  hipStream_t s = (hipStream_t)stream;
  VFM_TIMED(VFM_PROF_OTHER, launch_kv_append(attn->dtype, pl, attn->n_heads, attn->n_kv_heads, attn->head_dim,
                                             attn->rope_theta, qkv, ld, q_out,
                                             (int64_t)attn->n_heads * attn->head_dim, kv->k, kv->v,
                                             kv->n_pages * kv->page_size, pages_of(kv), s));
  return VFM_OK;
}

extern "C" int vfm_attention_workspace(const vfm_attn* attn, const vfm_batch* batch, size_t* bytes) {
  return workspace_attention(attn, batch, false, bytes);
}

extern "C" int vfm_attention_paged(const vfm_attn* attn, const vfm_batch* batch, const void* q, int64_t ldq,
                                   const vfm_kv_pages* kv, void* out, int64_t ldo, void* workspace, size_t ws_bytes,
                                   void* stream) {
  return attend_paged(attn, batch, q, ldq, kv, nullptr, out, ldo, workspace, ws_bytes, stream);
}

extern "C" int vfm_sample_tokens(const vfm_batch* batch, const float* out, const vfm_sampling* sampling, const float* u,
                                 int32_t* ids, float* logprob, void* stream) {
  Plan pl;
  VFM_TRY(check_batch(batch, &pl));
  if (!out || !sampling || !u || !ids) return VFM_ERR_ARG;
  const PlanOffsets po = plan_offsets(pl.n_req, pl.n_tasks, pl.T);
  const int32_t* off = host_arr(batch, po.out_off);
  int most = 0;
  for (int i = 0; i < pl.n_req; ++i) most = std::max(most, off[i + 1] - off[i]);
  if (most > 1 << 30) return VFM_ERR_SHAPE;
  if ((int64_t)pl.n_req * sample_threads(most) > kMaxThreads) return VFM_ERR_UNSUPPORTED;
  VFM_TRY(check_stream(stream));
  return hip_status(launch_sample(pl, out, *sampling, u, ids, logprob, most, (hipStream_t)stream));
}

extern "C" int vfm_adjust_outputs(const vfm_batch* batch, const float* out, const vfm_adjust* adjust, float* adjusted,
                                  void* stream) {
  Plan pl;
  VFM_TRY(check_batch(batch, &pl));
  if (!out || !adjust || !adjusted || !aligned16(out) || !aligned16(adjusted)) return VFM_ERR_ARG;
  const vfm_adjust& a = *adjust;
  if (a.hist && (!a.hist_begin || !a.hist_len)) return VFM_ERR_ARG;
  if (a.bias && (!a.bias_id || !a.bias_begin || !a.bias_len)) return VFM_ERR_ARG;
  if (a.mask && !a.mask_row) return VFM_ERR_ARG;
  if (a.n_hist < 0 || a.n_bias < 0 || (a.mask && (a.n_masks < 0 || a.mask_words < 1))) return VFM_ERR_SHAPE;
  const PlanOffsets po = plan_offsets(pl.n_req, pl.n_tasks, pl.T);
  const int32_t* off = host_arr(batch, po.out_off);
  int most = 0;
  for (int i = 0; i < pl.n_req; ++i) most = std::max(most, off[i + 1] - off[i]);
  if (pl.n_req > 1 << 23 || adjust_blocks(pl.n_req, most) > kMaxThreads / adjust_threads(adjust_slice(pl.n_req, most))) return VFM_ERR_UNSUPPORTED;
  VFM_TRY(check_stream(stream));
  if (most == 0) return VFM_OK;
  hipStream_t s = (hipStream_t)stream;
  VFM_TIMED(VFM_PROF_OTHER, launch_adjust(pl, out, adjusted, a, most, s));
  return VFM_OK;
}

// ---- decoding over a cache held in 8 bits (vfm_kv8.h) --------------------------

extern "C" int vfm_kv_append_q8(const vfm_attn* attn, const vfm_batch* batch, const void* qkv, int64_t ld, void* q_out,
                                const vfm_kv_pages_q8* kv, void* stream) {
  VFM_TRY(check_exps(kv));
  const vfm_kv_pages& pages = kv->pages;
  Plan pl;
  VFM_TRY(check_append(attn, batch, qkv, ld, q_out, &pages, stream, &pl));
  VFM_TRY(check_append8(pl));
  hipStream_t s = (hipStream_t)stream;
  const Pool8 pool{(uint8_t*)pages.k, (uint8_t*)pages.v, (uint8_t*)kv->exps, pages.n_pages * pages.page_size};
  VFM_TIMED(VFM_PROF_OTHER, launch_append8(attn->dtype, pl, attn->n_heads, attn->n_kv_heads, attn->head_dim,
                                           attn->rope_theta, qkv, ld, q_out, (int64_t)attn->n_heads * attn->head_dim,
                                           pool, pages_of(&pages), s));
  return VFM_OK;
}

extern "C" int vfm_attention_workspace_q8(const vfm_attn* attn, const vfm_batch* batch, size_t* bytes) {
  return workspace_attention(attn, batch, true, bytes);
}

extern "C" int vfm_attention_paged_q8(const vfm_attn* attn, const vfm_batch* batch, const void* q, int64_t ldq,
                                      const vfm_kv_pages_q8* kv, void* out, int64_t ldo, void* workspace,
                                      size_t ws_bytes, void* stream) {
  VFM_TRY(check_exps(kv));
  return attend_paged(attn, batch, q, ldq, &kv->pages, (const uint8_t*)kv->exps, out, ldo, workspace, ws_bytes, stream);
}

extern "C" int vfm_workspace_size_q8(const vfm_cfg* cfg, const vfm_batch* batch, const vfm_lora_table* lora,
                                     int32_t window, int32_t n_sink, size_t* bytes) {
  return workspace_windowed(cfg, batch, lora, window, n_sink, true, bytes);
}

extern "C" int vfm_layer_forward_q8(const vfm_cfg* cfg, const vfm_layer_weights* w, const vfm_lora_table* lora,
                                    const vfm_batch* batch, float* x, const vfm_kv_pages_q8* kv, int32_t window,
                                    int32_t n_sink, void* workspace, size_t ws_bytes, void* stream) {
  VFM_TRY(check_exps(kv));
  return layer_windowed(cfg, w, lora, batch, x, &kv->pages, (uint8_t*)kv->exps, window, n_sink, workspace, ws_bytes,
                        stream);
}
