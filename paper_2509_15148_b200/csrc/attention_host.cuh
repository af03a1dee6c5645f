// C-ABI entry points of the attention side (declared in include/atts.h): argument checks and launch geometry.
// Included by atts.cu behind its own helpers.
#pragma once
#include "norm_rope.cuh"
#include "packed_cache.cuh"
#include "packed_rows.cuh"
#include "rope_cache.cuh"
#include "tree_attention.cuh"

namespace atts {

constexpr int64_t kMaxSlots = kMaxSlotsOfSeq;  // slots of one sequence, columns of a weight row

static inline bool finite_pos(float x) { return x > 0.f && x <= 3.402823466e38f; }

// Checks a cache handle's description and fills the kernels' view of it.
static int cache_view(const atts_kv_cache* c, CacheView* out) {
  if (!c) return ATTS_ERR_NULL;
  if (c->dtype != ATTS_BF16 && c->dtype != ATTS_FP16) return ATTS_ERR_ARG;
  if (c->reserved != 0) return ATTS_ERR_ARG;
  if (c->num_seqs < 0 || c->num_seqs > 65535 || c->heads < 1 || c->heads > 1024) return ATTS_ERR_SHAPE;
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 != 0) return ATTS_ERR_SHAPE;
  if (c->page_size < 8 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0) return ATTS_ERR_SHAPE;
  if (c->num_pages < 0 || c->num_pages > 0x7FFFFFFF || c->table_cols < 0 || c->table_cols > 0x7FFFFFFF) return ATTS_ERR_SHAPE;
  if (c->table_stride < c->table_cols && c->num_seqs > 1) return ATTS_ERR_SHAPE;
  if (c->page_stride < 0 || c->slot_stride < 0 || c->head_stride < 0 || c->page_stride % 8 || c->slot_stride % 8 ||
      c->head_stride % 8)
    return ATTS_ERR_SHAPE;
  if ((c->num_pages > 0 && (!c->k || !c->v)) || (c->num_seqs > 0 && c->table_cols > 0 && !c->block_table)) return ATTS_ERR_NULL;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->block_table, 4)) return ATTS_ERR_ALIGN;
  out->k = static_cast<char*>(c->k);
  out->v = static_cast<char*>(c->v);
  out->table = c->block_table;
  out->table_stride = c->table_stride;
  out->page_stride = c->page_stride;
  out->slot_stride = c->slot_stride;
  out->head_stride = c->head_stride;
  out->table_cols = (int32_t)c->table_cols;
  out->num_pages = (int32_t)c->num_pages;
  out->heads = c->heads;
  int lg = 0;
  while ((1ll << lg) < c->page_size) ++lg;
  out->page_log2 = lg;
  return ATTS_OK;
}

// The same for a packed cache: strides in bytes, no slot stride.
static int packed_view(const atts_packed_cache* c, CacheView* out) {
  if (!c) return ATTS_ERR_NULL;
  if (c->num_seqs < 0 || c->num_seqs > 65535 || c->heads < 1 || c->heads > 1024) return ATTS_ERR_SHAPE;
  if (c->head_dim < 64 || c->head_dim > 256 || c->head_dim % 64 != 0) return ATTS_ERR_SHAPE;
  if (c->page_size < 8 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0) return ATTS_ERR_SHAPE;
  if (c->num_pages < 0 || c->num_pages > 0x7FFFFFFF || c->table_cols < 0 || c->table_cols > 0x7FFFFFFF) return ATTS_ERR_SHAPE;
  if (c->table_stride < c->table_cols && c->num_seqs > 1) return ATTS_ERR_SHAPE;
  const int64_t block = c->page_size / 8 * packed_eight(c->head_dim);
  if (c->page_stride < 0 || c->head_stride < 0 || c->page_stride % 16 || c->head_stride % 16 ||
      (c->num_pages > 1 && c->page_stride < block) || (c->heads > 1 && c->head_stride < block))
    return ATTS_ERR_SHAPE;
  if ((c->num_pages > 0 && (!c->k || !c->v)) || (c->num_seqs > 0 && c->table_cols > 0 && !c->block_table)) return ATTS_ERR_NULL;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->block_table, 4)) return ATTS_ERR_ALIGN;
  out->k = static_cast<char*>(c->k);
  out->v = static_cast<char*>(c->v);
  out->table = c->block_table;
  out->table_stride = c->table_stride;
  out->page_stride = c->page_stride;
  out->slot_stride = 0;
  out->head_stride = c->head_stride;
  out->table_cols = (int32_t)c->table_cols;
  out->num_pages = (int32_t)c->num_pages;
  out->heads = c->heads;
  int lg = 0;
  while ((1ll << lg) < c->page_size) ++lg;
  out->page_log2 = lg;
  return ATTS_OK;
}

// Checks shared by the calls that read a cache against queries.
static int check_queries(const void* q, int64_t q_ts, int64_t q_hs, const atts_kv_cache* c, const int32_t* ctx,
                         const int32_t* cu, const int32_t* pre, const int32_t* end, int64_t M, int32_t Hq,
                         int64_t max_tokens, int64_t max_len, float scale) {
  if (c->head_dim != 64 && c->head_dim != 128) return ATTS_ERR_SHAPE;
  if (M < 0 || M > (1ll << 30) || Hq < 1 || Hq % c->heads != 0 || Hq / c->heads > 128) return ATTS_ERR_SHAPE;
  if (max_tokens < 0 || max_len < 0 || max_len > kMaxSlots || max_tokens > max_len) return ATTS_ERR_SHAPE;
  if (q_ts < 0 || q_hs < 0 || q_ts % 8 || q_hs % 8) return ATTS_ERR_SHAPE;
  // rows of their own: a stride of 0 (a broadcast) is refused where there is more than one entry
  if ((M > 1 && q_ts == 0) || (Hq > 1 && q_hs == 0) || c->num_pages < 1 || (c->num_pages > 1 && c->page_stride == 0) ||
      c->slot_stride == 0 || (c->heads > 1 && c->head_stride == 0))
    return ATTS_ERR_SHAPE;
  if (!finite_pos(scale)) return ATTS_ERR_ARG;
  if ((M > 0 && !q) || (c->num_seqs > 0 && (!ctx || !cu)) || ((pre == nullptr) != (end == nullptr))) return ATTS_ERR_NULL;
  if (!aligned(q, 16) || !aligned(ctx, 4) || !aligned(cu, 4) || !aligned(pre, 4) || !aligned(end, 4)) return ATTS_ERR_ALIGN;
  return ATTS_OK;
}

// Tensor maps.  Queries: (channel, head, token) with boxes of 64 channels, the heads of a group and the tokens of a row
// tile.  Cache: (channel, slot of a page, head, page) with boxes of 64 channels and the slots of a page (128 at most).
static int encode_rows(const DeviceInfo* di, CUtensorMap* map, bool bf16, const void* base, int rank, const int64_t* dims,
                       const int64_t* strides_elems, const int* box) {
  cuuint64_t d[4], st[3];
  cuuint32_t b[4], e[4];
  for (int i = 0; i < rank; ++i) {
    d[i] = (cuuint64_t)dims[i];
    b[i] = (cuuint32_t)box[i];
    e[i] = 1;
    // a dimension of one entry has no stride of its own
    if (i > 0) st[i - 1] = dims[i] > 1 ? (cuuint64_t)strides_elems[i - 1] * 2 : (cuuint64_t)dims[0] * 2;
  }
  const CUresult r = di->encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank,
                                const_cast<void*>(base), d, st, b, e, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? ATTS_OK : ATTS_ERR_CUDA;
}
static int encode_queries(const DeviceInfo* di, CUtensorMap* map, const atts_kv_cache* c, const void* q, int64_t q_ts, int64_t q_hs,
                          int64_t M, int32_t Hq, int tokens) {
  const int64_t dims[3] = {c->head_dim, Hq, M}, st[2] = {q_hs, q_ts};
  const int box[3] = {64, Hq / c->heads, tokens};
  return encode_rows(di, map, c->dtype == ATTS_BF16, q, 3, dims, st, box);
}
static int encode_cache(const DeviceInfo* di, CUtensorMap* map, const atts_kv_cache* c, const void* base) {
  const int64_t dims[4] = {c->head_dim, c->page_size, c->heads, c->num_pages}, st[3] = {c->slot_stride, c->head_stride, c->page_stride};
  const int box[4] = {64, (int)(c->page_size < 128 ? c->page_size : 128), 1, 1};
  return encode_rows(di, map, c->dtype == ATTS_BF16, base, 4, dims, st, box);
}

// Tokens of a row tile: as many as fit 128 rows, and no more than a sequence can have (the rest would be loaded in vain).
static int row_tile_tokens(int G, int64_t max_tokens) {
  const int fit = kAttnTile / G;
  return max_tokens < 1 ? 1 : max_tokens < fit ? (int)max_tokens : fit;
}

// How an attention call is cut up.  Row tiles: as many whole tokens as fit 128 rows; two of them to a CTA if the longest
// sequence has more than one.  Chunks: the number that makes the launch shortest by these measured times (us): a CTA's
// start and end 9, a slot tile 1.2 (2.0 for two row tiles), a chunk's sums one per 45 KB of them, the second launch 3.
// One row tile and more CTAs than SMs: kRowsBrief if its 8 + 3.5 a tile, two CTAs an SM, come out below that.
// A window leaves a row tile with the tiles of the sinks, of the window before its tokens, and of the drafts, two of them cut;
// a packed cache's tiles take 1.55 (1.35 for half the rows) and 2.4, and it has no kRowsBrief (its raw tiles leave no room for two CTAs).
struct AttnShape {
  AttnMode mode;
  bool few;          // packed_rows_kernel
  AttnPlan p;
};
constexpr int64_t kEndless = 0x7FFFFFFF;   // a window that leaves nothing out

// Slot tiles of which a row tile may see something.
static int64_t seen_tiles(int64_t max_tokens, int64_t max_len, AttnForm form, int64_t window, int64_t sinks) {
  const int64_t tiles = (max_len + kAttnTile - 1) / kAttnTile;
  if (!(form & 1)) return tiles;
  const int64_t seen = (max_tokens + window + kAttnTile - 1) / kAttnTile + 2 + (sinks + kAttnTile - 1) / kAttnTile;
  return seen < tiles ? seen : tiles;
}

// packed_rows_kernel: all rows of a sequence's key head in one CTA.  The number of chunks that makes the launch shortest by these measured
// times (us): a CTA's start and end 2, a tile 1.0 alone on an SM and 0.66 in company (1.4 and 0.9 beyond 8 rows), the join of
// chunks 4 and 0.05 a chunk.
static AttnShape few_shape(int sms, int64_t num_seqs, int G, int32_t heads, int64_t max_tokens, int64_t max_len, AttnForm form, int64_t window,
                           int64_t sinks) {
  AttnShape r{};
  r.few = true;
  r.p.tpt = max_tokens < 1 ? 1 : (int)max_tokens;
  r.p.nq = 1;
  const int64_t tiles = seen_tiles(max_tokens, max_len, form, window, sinks), base = num_seqs * heads;
  const bool eight = max_tokens * G <= 8;
  double best = 0.0;
  int64_t best_n = 1;
  for (int64_t n = 1; n <= tiles && n <= 256 && (n == 1 || base * n <= 64 * (int64_t)sms); ++n) {
    const int64_t ct = (tiles + n - 1) / n, k = (base * n + sms - 1) / sms;
    if ((tiles + ct - 1) / ct != n) continue;
    const double tile = k <= 1 ? (eight ? 1.0 : 1.4) : eight ? 0.66 : 0.9;
    const double cost = (double)k * (2.0 + tile * (double)ct) + (n > 1 ? 4.0 + 0.05 * (double)n : 0.0);
    if (n == 1 || cost < best) {
      best = cost;
      best_n = n;
    }
  }
  r.p.chunk = (int)(tiles > 0 ? (tiles + best_n - 1) / best_n : 1);
  r.p.chunks = (int)(tiles > 0 ? (tiles + r.p.chunk - 1) / r.p.chunk : 1);
  return r;
}
static AttnShape attn_shape(int sms, int64_t num_seqs, int32_t Hq, int32_t heads, int32_t head_dim, int64_t max_tokens, int64_t max_len,
                            AttnForm form = kFormPlain, int64_t window = kEndless, int64_t sinks = 0) {
  AttnShape r{};
  const int G = Hq / heads;
  if ((form & 2) && max_tokens * G <= kFewMaxRows) return few_shape(sms, num_seqs, G, heads, max_tokens, max_len, form, window, sinks);
  r.p.tpt = row_tile_tokens(G, max_tokens);
  r.mode = max_tokens > r.p.tpt ? kRowsTwo : form != kFormPlain && max_tokens * G <= 64 ? kRowsHalf : kRowsOne;
  const int64_t per = r.p.tpt * (r.mode == kRowsTwo ? 2 : 1);
  r.p.nq = (int)((max_tokens + per - 1) / per);
  const int64_t tiles = seen_tiles(max_tokens, max_len, form, window, sinks);
  const int64_t base = num_seqs * heads * r.p.nq;
  const double tile = (form & 2) ? (r.mode == kRowsTwo ? 2.4 : r.mode == kRowsHalf ? 1.35 : 1.55) : r.mode == kRowsTwo ? 2.0 : 1.2;
  const double part = (double)((max_tokens < per ? max_tokens : per) * G) * head_dim * 8 / (45 * 1024);
  double best = 0.0;
  int64_t best_n = 1;
  for (int64_t n = 1; n <= tiles && n <= 256 && (n == 1 || base * n <= 64 * (int64_t)sms); ++n) {
    const int64_t ct = (tiles + n - 1) / n;
    if ((tiles + ct - 1) / ct != n) continue;   // the same chunk length with fewer chunks was looked at
    const double cost = (double)((base * n + sms - 1) / sms) * (9.0 + tile * (double)ct + (n > 1 ? part : 0.0)) + (n > 1 ? 3.0 : 0.0);
    if (n == 1 || cost < best) {
      best = cost;
      best_n = n;
    }
  }
  if (!(form & 2) && r.mode != kRowsTwo && base > sms && (double)((base + 2 * sms - 1) / (2 * sms)) * (8.0 + 3.5 * (double)tiles) < best) {
    r.mode = kRowsBrief;
    best_n = 1;
  }
  r.p.chunk = (int)(tiles > 0 ? (tiles + best_n - 1) / best_n : 1);
  r.p.chunks = (int)(tiles > 0 ? (tiles + r.p.chunk - 1) / r.p.chunk : 1);
  return r;
}
static size_t attn_workspace(const AttnShape& s, int64_t M, int32_t Hq, int32_t head_dim) {
  if (s.p.chunks <= 1) return 256;
  const size_t rows = (size_t)M * Hq * s.p.chunks;
  return round_up(rows * 4, 256) + round_up(rows * head_dim * 4, 256);
}

template <typename T, int D>
static int launch_parts_join(const AttnArgs& a, const AttnPlan& p, unsigned num_seqs, cudaStream_t stream) {
  const int64_t rows = (int64_t)a.max_tokens * a.Hq;
  if (p.chunks > kJoinFewParts) return launch_pdl(attention_parts_join_kernel<T, D, 4>, dim3((unsigned)((rows + 1) / 2), num_seqs), dim3(kJoinThreads), 0, stream, a, p);
  return launch_pdl(attention_parts_join_kernel<T, D, 1>, dim3((unsigned)((rows + 7) / 8), num_seqs), dim3(kJoinThreads), 0, stream, a, p);
}

template <typename T, int D, AttnMode MODE, AttnForm FORM>
static int launch_attention(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const AttnArgs& a, const AttnPlan& p,
                            dim3 grid, unsigned* status, cudaStream_t stream) {
  using Cfg = AttnCfg<D, MODE, FORM>;
  int st = launch_pdl(tree_attention_kernel<T, D, MODE, FORM>, grid, dim3(Cfg::kThreads), Cfg::kSmemBytes, stream, mq, mk, mv, a, p, status);
  if (st != ATTS_OK || p.chunks <= 1) return st;
  const int64_t rows = (int64_t)a.max_tokens * a.Hq;
  if (FORM & 1) return launch_parts_join<T, D>(a, p, grid.z, stream);
  return launch_pdl(attention_join_kernel<T, D>, dim3((unsigned)((rows + 7) / 8), grid.z), dim3(256), 0, stream, a, p);
}

template <typename T, int D>
static int launch_few(const AttnArgs& a, const AttnPlan& p, dim3 grid, unsigned* status, cudaStream_t stream) {
  const int64_t most = (int64_t)a.max_tokens * a.G;
  const int st = most <= 8 ? launch_pdl(packed_rows_kernel<T, D, 1>, grid, dim3(kFewThreads), FewCfg<D, 1>::kSmemBytes, stream, a, p, status)
                           : launch_pdl(packed_rows_kernel<T, D, 2>, grid, dim3(kFewThreads), FewCfg<D, 2>::kSmemBytes, stream, a, p, status);
  if (st != ATTS_OK || p.chunks <= 1) return st;
  return launch_parts_join<T, D>(a, p, grid.z, stream);
}

// An attention call, its cache and queries checked (a.cache is filled): the remaining checks, the cut of the work, the launches.
// `c` describes the cache for the tensor maps (of a packed one only type and sizes are used).
template <AttnForm FORM>
static int attend(AttnArgs& a, const atts_kv_cache* c, const void* q, int64_t q_ts, int64_t q_hs, const int32_t* ctx, const int32_t* cu,
                  const int32_t* pre, const int32_t* end, const int32_t* depth, int64_t window, int64_t sinks, int64_t M, int32_t Hq,
                  int64_t max_tokens, int64_t max_len, float scale, void* out, int64_t o_ts, int64_t o_hs, float* lse, void* workspace,
                  size_t workspace_bytes, void* cuda_stream) {
  if (o_ts < 0 || o_hs < 0 || o_ts % 8 || o_hs % 8) return ATTS_ERR_SHAPE;
  if ((M > 0 && !out) || !workspace) return ATTS_ERR_NULL;
  if (!aligned(out, 16) || !aligned(lse, 4) || !aligned(workspace, 256)) return ATTS_ERR_ALIGN;
  const DeviceInfo* di;
  const int st = device_info(&di);
  if (st != ATTS_OK) return st;
  AttnShape sh = attn_shape(di->sm_count, c->num_seqs, Hq, c->heads, c->head_dim, max_tokens, max_len, FORM, window, sinks);
  if (workspace_bytes < attn_workspace(sh, M, Hq, c->head_dim)) return ATTS_ERR_WORKSPACE;
  if (M == 0 || c->num_seqs == 0 || max_tokens == 0) return ATTS_OK;
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.q_ts = q_ts; a.q_hs = q_hs; a.o_ts = o_ts; a.o_hs = o_hs;
  a.ctx = ctx; a.cu = cu; a.pre = pre; a.end = end;
  a.depth = depth; a.window = (int)window; a.sinks = (int)sinks;
  a.M = (int)M; a.Hq = Hq; a.G = Hq / c->heads; a.max_tokens = (int)max_tokens; a.max_len = (int)max_len;
  a.scale = scale;
  sh.p.part_lse = static_cast<float*>(workspace);
  sh.p.part_o = sh.p.part_lse + round_up((size_t)M * Hq * sh.p.chunks * 4, 256) / 4;
  sh.p.wait_limit = wait_limit();
  sh.p.withhold_loads = g_withhold_loads.load(std::memory_order_relaxed);
  const int64_t gx = (int64_t)sh.p.nq * sh.p.chunks;
  if (gx > 0x7FFFFFFF || (int64_t)max_tokens * Hq > 0x7FFFFFFF) return ATTS_ERR_SHAPE;
  const dim3 grid((unsigned)gx, (unsigned)c->heads, (unsigned)c->num_seqs);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const bool bf = c->dtype == ATTS_BF16;
  if constexpr ((FORM & 2) != 0)
    if (sh.few) {
      if (c->head_dim == 128) return bf ? launch_few<__nv_bfloat16, 128>(a, sh.p, grid, di->dev_status, stream) : launch_few<__half, 128>(a, sh.p, grid, di->dev_status, stream);
      return bf ? launch_few<__nv_bfloat16, 64>(a, sh.p, grid, di->dev_status, stream) : launch_few<__half, 64>(a, sh.p, grid, di->dev_status, stream);
    }
  CUtensorMap mq, mk, mv;
  if (encode_queries(di, &mq, c, q, q_ts, q_hs, M, Hq, sh.p.tpt) != ATTS_OK) return ATTS_ERR_CUDA;
  if (FORM & 2) mk = mv = mq;   // not used
  else if (encode_cache(di, &mk, c, c->k) != ATTS_OK || encode_cache(di, &mv, c, c->v) != ATTS_OK) return ATTS_ERR_CUDA;
#define ATTS_ATTEND(D, MODE)                                                                                      \
  (bf ? launch_attention<__nv_bfloat16, D, MODE, FORM>(mq, mk, mv, a, sh.p, grid, di->dev_status, stream)         \
      : launch_attention<__half, D, MODE, FORM>(mq, mk, mv, a, sh.p, grid, di->dev_status, stream))
  if (sh.mode == kRowsTwo) return c->head_dim == 128 ? ATTS_ATTEND(128, kRowsTwo) : ATTS_ATTEND(64, kRowsTwo);
  if constexpr (FORM != kFormPlain)
    if (sh.mode == kRowsHalf) return c->head_dim == 128 ? ATTS_ATTEND(128, kRowsHalf) : ATTS_ATTEND(64, kRowsHalf);
  if constexpr (!(FORM & 2))
    if (sh.mode == kRowsBrief) return c->head_dim == 128 ? ATTS_ATTEND(128, kRowsBrief) : ATTS_ATTEND(64, kRowsBrief);
  return c->head_dim == 128 ? ATTS_ATTEND(128, kRowsOne) : ATTS_ATTEND(64, kRowsOne);
#undef ATTS_ATTEND
}

// Arguments of a window: 1 .. 2^30 tokens (or 0, where that means none), 0 .. 2^30 sinks; trees bring their depths.
static int check_window(int64_t window, int64_t sinks, bool may_be_none, const int32_t* pre, const int32_t* depth) {
  if (window < (may_be_none ? 0 : 1) || window > kMaxSlots || sinks < 0 || sinks > kMaxSlots) return ATTS_ERR_ARG;
  if (window > 0 && (pre != nullptr) != (depth != nullptr)) return ATTS_ERR_NULL;
  if (!aligned(depth, 4)) return ATTS_ERR_ALIGN;
  return ATTS_OK;
}

static int attention_workspace(AttnForm form, int64_t num_seqs, int64_t M, int32_t Hq, int32_t heads, int32_t head_dim, int64_t max_tokens,
                               int64_t max_len, int64_t window, int64_t sinks, size_t* bytes) {
  if (!bytes) return ATTS_ERR_NULL;
  if (num_seqs < 0 || num_seqs > 65535 || M < 0 || M > (1ll << 30) || heads < 1 || heads > 1024 || Hq < 1 || Hq % heads != 0 ||
      Hq / heads > 128 || (head_dim != 64 && head_dim != 128) || max_tokens < 0 || max_len < max_tokens || max_len > kMaxSlots)
    return ATTS_ERR_SHAPE;
  const DeviceInfo* di;
  const int st = device_info(&di);
  if (st != ATTS_OK) return st;
  *bytes = attn_workspace(attn_shape(di->sm_count, num_seqs, Hq, heads, head_dim, max_tokens, max_len, form, window, sinks), M, Hq, head_dim);
  return ATTS_OK;
}

// launch_pdl with `cluster` blocks to a cluster; the grid counts clusters.
template <typename... KArgs, typename... Args>
static int launch_pdl_cluster(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid.x * (unsigned)cluster, grid.y, grid.z);
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...) != cudaSuccess) {
    cudaGetLastError();
    return ATTS_ERR_CUDA;
  }
  return ATTS_OK;
}

// Slots of a block of the packed append and of the call that reads back: enough blocks for every SM first.
static int pack_tokens(int sms, int64_t slots) {
  int n = kPackMaxTokens;
  while (n > 1 && slots < 4 * (int64_t)n * sms) n /= 2;
  return n;
}

// Checks and launch shared by the two normed rotations; the caller has filled what is its own.
template <bool ROWS>
static int norm_rope(NormRopeArgs& a, const void* q, int64_t q_ts, int64_t q_hs, const void* k, int64_t k_ts, int64_t k_hs,
                     const int32_t* positions, const double* freqs, int32_t pairs, float mscale, int32_t interleaved, const void* q_gain,
                     const void* k_gain, float eps, int32_t dtype, int64_t M, int32_t Hq, int32_t Hk, int32_t D, void* q_out, int64_t o_ts,
                     int64_t o_hs, bool wide, bool none, int64_t num_seqs, void* cuda_stream) {
  if (M < 0 || M > (1ll << 30) || Hq < 0 || Hq > (1 << 20)) return ATTS_ERR_SHAPE;
  if (pairs < 0 || 2 * (int64_t)pairs > D) return ATTS_ERR_SHAPE;
  if (q_ts < 0 || q_hs < 0 || k_ts < 0 || k_hs < 0 || o_ts < 0 || o_hs < 0) return ATTS_ERR_SHAPE;
  if (interleaved != 0 && interleaved != 1) return ATTS_ERR_ARG;
  if (!(mscale >= -3.402823466e38f && mscale <= 3.402823466e38f) || !(eps >= 0.f && eps <= 3.402823466e38f)) return ATTS_ERR_ARG;
  if (M > 0 && ((Hk > 0 && !k) || (Hq > 0 && (!q || !q_out)) || (pairs > 0 && (!positions || !freqs)))) return ATTS_ERR_NULL;
  if (!aligned(q, 2) || !aligned(k, 2) || !aligned(q_out, 2) || !aligned(q_gain, 2) || !aligned(k_gain, 2) || !aligned(positions, 4) ||
      !aligned(freqs, 8))
    return ATTS_ERR_ALIGN;
  const DeviceInfo* di;
  const int st = device_info(&di);
  if (st != ATTS_OK) return st;
  if (M == 0 || none) return ATTS_OK;
  a.q = static_cast<const char*>(q);
  a.k = static_cast<const char*>(k);
  a.q_gain = static_cast<const char*>(q_gain);
  a.k_gain = static_cast<const char*>(k_gain);
  a.q_out = static_cast<char*>(q_out);
  a.q_ts = q_ts; a.q_hs = q_hs; a.k_ts = k_ts; a.k_hs = k_hs; a.o_ts = o_ts; a.o_hs = o_hs;
  a.positions = positions; a.freqs = freqs;
  a.pairs = pairs; a.D = D; a.Hq = Hq; a.Hk = Hk; a.M = (int)M; a.mscale = mscale; a.eps = eps;
  const int64_t bits = (Hq > 0 ? q_ts | q_hs | o_ts | o_hs : 0) | (Hk > 0 ? k_ts | k_hs : 0);
  wide = wide && bits % 8 == 0 && aligned(q, 16) && aligned(k, 16) && aligned(q_out, 16) && aligned(q_gain, 16) && aligned(k_gain, 16) &&
         pairs % (interleaved ? 4 : 8) == 0;
  a.lanes_log2 = 0;
  while (a.lanes_log2 < 4 && 16 << a.lanes_log2 < D) ++a.lanes_log2;   // two pieces of eight channels a thread
  const int64_t span = ROWS ? M : a.max_tokens;
  a.inv_d = 1.f / (float)D;
  a.tpb = 1;                        // as many tokens as leave two blocks to an SM if sequences fill them: what a block sets up is shared by more rows
  while (a.tpb < kNormRopeMaxTokens && M >= 4 * a.tpb * (int64_t)di->sm_count) a.tpb *= 2;
  const dim3 grid((unsigned)((span + a.tpb - 1) / a.tpb), ROWS ? 1 : (unsigned)num_seqs);
  const size_t smem = sizeof(float2) * a.tpb * (size_t)pairs;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
#define ATTS_NORM(T, I, W) return launch_pdl(norm_rope_kernel<T, I, W, ROWS>, grid, dim3(kRopeThreads), smem, stream, a, di->dev_status)
#define ATTS_NORM_T(T)                                                                        \
  do {                                                                                        \
    if (interleaved) { if (wide) ATTS_NORM(T, true, true); else ATTS_NORM(T, true, false); }  \
    else { if (wide) ATTS_NORM(T, false, true); else ATTS_NORM(T, false, false); }            \
  } while (0)
  if (dtype == ATTS_BF16) ATTS_NORM_T(__nv_bfloat16);
  else ATTS_NORM_T(__half);
#undef ATTS_NORM_T
#undef ATTS_NORM
}

template <typename T, int D, bool MANY>
static int launch_weights(const CUtensorMap& mq, const CUtensorMap& mk, const WeightArgs& a, dim3 clusters, unsigned* status, cudaStream_t stream) {
  return launch_pdl_cluster(cache_weights_kernel<T, D, MANY>, clusters, dim3(kWeightThreads), WeightCfg<D>::kSmemBytes, a.cluster, stream, mq, mk, a,
                            status);
}

}  // namespace atts

using namespace atts;

extern "C" {

int atts_tree_plan(const int32_t* parent, const int32_t* cu_tokens, int64_t num_seqs, int32_t* pre, int32_t* end,
                   int32_t* depth) {
  if (num_seqs < 0 || num_seqs >= (1ll << 31)) return ATTS_ERR_SHAPE;
  if (num_seqs == 0) return ATTS_OK;
  if (!cu_tokens) return ATTS_ERR_NULL;
  if (cu_tokens[0] != 0) return ATTS_ERR_ARG;
  for (int64_t b = 0; b < num_seqs; ++b)
    if (cu_tokens[b + 1] < cu_tokens[b]) return ATTS_ERR_ARG;
  if (cu_tokens[num_seqs] > 0 && (!parent || !pre || !end)) return ATTS_ERR_NULL;
  for (int64_t b = 0; b < num_seqs; ++b) {
    const int32_t n = cu_tokens[b + 1] - cu_tokens[b];
    const int32_t* par = parent + cu_tokens[b];
    int32_t *p = pre + cu_tokens[b], *e = end + cu_tokens[b];
    for (int32_t i = 0; i < n; ++i) {
      if (par[i] < -2 || par[i] >= i || (par[i] >= 0 && par[par[i]] == -2)) return ATTS_ERR_ARG;
      e[i] = 1;
    }
    // sizes of the subtrees (children come after their parents), kept in end
    for (int32_t i = n - 1; i >= 0; --i)
      if (par[i] >= 0) e[par[i]] += e[i];
    // A token's place follows its parent's and the subtrees of the siblings before it.  While a token still has
    // children to come, its subtree's unplaced part ends at pre + size: the first child takes the last piece.
    int32_t top = 0;
    for (int32_t i = 0; i < n; ++i) {
      if (par[i] == -2) {
        p[i] = e[i] = -1;
        continue;
      }
      const int32_t size = e[i];
      if (par[i] == -1) {
        p[i] = top;
        top += size;
      } else {
        e[par[i]] -= size;        // end of the parent's part that is not placed yet
        p[i] = e[par[i]];
      }
      e[i] = p[i] + size;
    }
    // restore the ends: after the pass above end[i] = pre[i] + 1 for every token; the true end is the largest among
    // its descendants'
    for (int32_t i = n - 1; i >= 0; --i)
      if (par[i] >= 0 && e[par[i]] < e[i]) e[par[i]] = e[i];
    if (depth) {
      int32_t* d = depth + cu_tokens[b];
      for (int32_t i = 0; i < n; ++i) d[i] = par[i] >= 0 ? d[par[i]] + 1 : 0;
    }
  }
  return ATTS_OK;
}

int atts_rope_append(const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k, int64_t k_token_stride,
                     int64_t k_head_stride, const void* v, int64_t v_token_stride, int64_t v_head_stride,
                     const int32_t* positions, const double* freqs, int32_t rotary_pairs, float mscale,
                     int32_t interleaved, const atts_kv_cache* cache, const int32_t* ctx_lens, const int32_t* cu_tokens,
                     int64_t M, int32_t Hq, int64_t max_tokens, void* q_out, int64_t out_token_stride,
                     int64_t out_head_stride, void* cuda_stream) {
  RopeArgs a;
  int st = cache_view(cache, &a.cache);
  if (st != ATTS_OK) return st;
  const int D = cache->head_dim;
  if (M < 0 || M > (1ll << 30) || Hq < 0 || Hq > (1 << 20) || max_tokens < 0 || max_tokens > kMaxSlots) return ATTS_ERR_SHAPE;
  if (rotary_pairs < 0 || 2 * (int64_t)rotary_pairs > D) return ATTS_ERR_SHAPE;
  if (q_token_stride < 0 || q_head_stride < 0 || k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 ||
      v_head_stride < 0 || out_token_stride < 0 || out_head_stride < 0)
    return ATTS_ERR_SHAPE;
  if (interleaved != 0 && interleaved != 1) return ATTS_ERR_ARG;
  if (!(mscale >= -3.402823466e38f && mscale <= 3.402823466e38f)) return ATTS_ERR_ARG;
  if (cache->num_seqs > 0 && (!ctx_lens || !cu_tokens)) return ATTS_ERR_NULL;
  if (M > 0 && (!k || !v || (Hq > 0 && (!q || !q_out)) || (rotary_pairs > 0 && (!positions || !freqs)))) return ATTS_ERR_NULL;
  if (!aligned(q, 2) || !aligned(k, 2) || !aligned(v, 2) || !aligned(q_out, 2) || !aligned(positions, 4) || !aligned(freqs, 8) ||
      !aligned(ctx_lens, 4) || !aligned(cu_tokens, 4))
    return ATTS_ERR_ALIGN;
  const DeviceInfo* di;
  st = device_info(&di);
  if (st != ATTS_OK) return st;
  if (M == 0 || cache->num_seqs == 0 || max_tokens == 0) return ATTS_OK;
  a.q = static_cast<const char*>(q);
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.q_out = static_cast<char*>(q_out);
  a.q_ts = q_token_stride; a.q_hs = q_head_stride;
  a.k_ts = k_token_stride; a.k_hs = k_head_stride;
  a.v_ts = v_token_stride; a.v_hs = v_head_stride;
  a.o_ts = out_token_stride; a.o_hs = out_head_stride;
  a.positions = positions; a.ctx = ctx_lens; a.cu = cu_tokens; a.freqs = freqs;
  a.pairs = rotary_pairs; a.D = D; a.Hq = Hq; a.M = (int)M; a.max_tokens = (int)max_tokens; a.mscale = mscale;
  const int64_t bits = (Hq > 0 ? q_token_stride | q_head_stride | out_token_stride | out_head_stride : 0) | k_token_stride |
                       k_head_stride | v_token_stride | v_head_stride;
  const bool wide = bits % 8 == 0 && aligned(q, 16) && aligned(k, 16) && aligned(v, 16) && aligned(q_out, 16) &&
                    rotary_pairs % (interleaved ? 4 : 8) == 0;
  a.lanes_log2 = 0;
  while (a.lanes_log2 < 3 && 16 << a.lanes_log2 < D) ++a.lanes_log2;
  a.tpb = M >= 4 * 8 * (int64_t)di->sm_count ? 4 : 1;
  const int64_t gx = (max_tokens + a.tpb - 1) / a.tpb;
  if (gx > 0x7FFFFFFF) return ATTS_ERR_SHAPE;
  const dim3 grid((unsigned)gx, (unsigned)cache->num_seqs);
  const size_t smem = sizeof(float2) * a.tpb * (size_t)rotary_pairs;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
#define ATTS_ROPE(T, I, W) return launch_pdl(rope_append_kernel<T, I, W>, grid, dim3(kRopeThreads), smem, stream, a, di->dev_status)
#define ATTS_ROPE_T(T)                                                                        \
  do {                                                                                        \
    if (interleaved) { if (wide) ATTS_ROPE(T, true, true); else ATTS_ROPE(T, true, false); }  \
    else { if (wide) ATTS_ROPE(T, false, true); else ATTS_ROPE(T, false, false); }            \
  } while (0)
  if (cache->dtype == ATTS_BF16) ATTS_ROPE_T(__nv_bfloat16);
  else ATTS_ROPE_T(__half);
#undef ATTS_ROPE_T
#undef ATTS_ROPE
}

int atts_tree_attention_workspace_bytes(int64_t num_seqs, int64_t M, int32_t Hq, int32_t heads, int32_t head_dim,
                                        int64_t max_tokens, int64_t max_len, size_t* bytes) {
  return attention_workspace(kFormPlain, num_seqs, M, Hq, heads, head_dim, max_tokens, max_len, kEndless, 0, bytes);
}

int atts_tree_attention(const void* q, int64_t q_token_stride, int64_t q_head_stride, const atts_kv_cache* cache,
                        const int32_t* ctx_lens, const int32_t* cu_tokens, const int32_t* pre, const int32_t* end,
                        int64_t M, int32_t Hq, int64_t max_tokens, int64_t max_len, float scale, void* out,
                        int64_t out_token_stride, int64_t out_head_stride, float* lse, void* workspace,
                        size_t workspace_bytes, void* cuda_stream) {
  AttnArgs a;
  int st = cache_view(cache, &a.cache);
  if (st != ATTS_OK) return st;
  st = check_queries(q, q_token_stride, q_head_stride, cache, ctx_lens, cu_tokens, pre, end, M, Hq, max_tokens, max_len, scale);
  if (st != ATTS_OK) return st;
  return attend<kFormPlain>(a, cache, q, q_token_stride, q_head_stride, ctx_lens, cu_tokens, pre, end, nullptr, kEndless, 0, M, Hq, max_tokens,
                            max_len, scale, out, out_token_stride, out_head_stride, lse, workspace, workspace_bytes, cuda_stream);
}

int atts_window_attention_workspace_bytes(int64_t num_seqs, int64_t M, int32_t Hq, int32_t heads, int32_t head_dim, int64_t max_tokens,
                                          int64_t max_len, int64_t window, int64_t sinks, size_t* bytes) {
  const int st = check_window(window, sinks, false, nullptr, nullptr);
  if (st != ATTS_OK) return st;
  return attention_workspace(kFormWindow, num_seqs, M, Hq, heads, head_dim, max_tokens, max_len, window, sinks, bytes);
}

int atts_window_attention(const void* q, int64_t q_token_stride, int64_t q_head_stride, const atts_kv_cache* cache,
                          const int32_t* ctx_lens, const int32_t* cu_tokens, const int32_t* pre, const int32_t* end,
                          const int32_t* depth, int64_t window, int64_t sinks, int64_t M, int32_t Hq, int64_t max_tokens,
                          int64_t max_len, float scale, void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse,
                          void* workspace, size_t workspace_bytes, void* cuda_stream) {
  AttnArgs a;
  int st = cache_view(cache, &a.cache);
  if (st != ATTS_OK) return st;
  st = check_queries(q, q_token_stride, q_head_stride, cache, ctx_lens, cu_tokens, pre, end, M, Hq, max_tokens, max_len, scale);
  if (st != ATTS_OK) return st;
  if ((st = check_window(window, sinks, false, pre, depth)) != ATTS_OK) return st;
  return attend<kFormWindow>(a, cache, q, q_token_stride, q_head_stride, ctx_lens, cu_tokens, pre, end, depth, window, sinks, M, Hq, max_tokens,
                             max_len, scale, out, out_token_stride, out_head_stride, lse, workspace, workspace_bytes, cuda_stream);
}

int atts_packed_attention_workspace_bytes(int64_t num_seqs, int64_t M, int32_t Hq, int32_t heads, int32_t head_dim, int64_t max_tokens,
                                          int64_t max_len, int64_t window, int64_t sinks, size_t* bytes) {
  const int st = check_window(window, sinks, true, nullptr, nullptr);
  if (st != ATTS_OK) return st;
  return attention_workspace(window ? kFormPackedWindow : kFormPacked, num_seqs, M, Hq, heads, head_dim, max_tokens, max_len, window ? window : kEndless, sinks, bytes);
}

int atts_packed_attention(const void* q, int64_t q_token_stride, int64_t q_head_stride, int32_t dtype, const atts_packed_cache* cache,
                          const int32_t* ctx_lens, const int32_t* cu_tokens, const int32_t* pre, const int32_t* end,
                          const int32_t* depth, int64_t window, int64_t sinks, int64_t M, int32_t Hq, int64_t max_tokens,
                          int64_t max_len, float scale, void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse,
                          void* workspace, size_t workspace_bytes, void* cuda_stream) {
  AttnArgs a;
  int st = packed_view(cache, &a.cache);
  if (st != ATTS_OK) return st;
  if (dtype != ATTS_BF16 && dtype != ATTS_FP16) return ATTS_ERR_ARG;
  const atts_kv_cache c = {cache->k, cache->v, cache->block_table, cache->num_seqs, cache->table_cols, cache->table_stride, cache->num_pages,
                           cache->page_size, cache->page_stride, 1, cache->head_stride, cache->heads, cache->head_dim, dtype, 0};
  st = check_queries(q, q_token_stride, q_head_stride, &c, ctx_lens, cu_tokens, pre, end, M, Hq, max_tokens, max_len, scale);
  if (st != ATTS_OK) return st;
  if ((st = check_window(window, sinks, true, pre, depth)) != ATTS_OK) return st;
  if (window)
    return attend<kFormPackedWindow>(a, &c, q, q_token_stride, q_head_stride, ctx_lens, cu_tokens, pre, end, depth, window, sinks, M, Hq,
                                     max_tokens, max_len, scale, out, out_token_stride, out_head_stride, lse, workspace, workspace_bytes,
                                     cuda_stream);
  return attend<kFormPacked>(a, &c, q, q_token_stride, q_head_stride, ctx_lens, cu_tokens, pre, end, nullptr, kEndless, 0, M, Hq, max_tokens,
                             max_len, scale, out, out_token_stride, out_head_stride, lse, workspace, workspace_bytes, cuda_stream);
}

int atts_packed_append(const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                       int64_t v_head_stride, int32_t dtype, const atts_packed_cache* cache, const int32_t* ctx_lens,
                       const int32_t* cu_tokens, int64_t M, int64_t max_tokens, void* cuda_stream) {
  PackArgs a;
  int st = packed_view(cache, &a.cache);
  if (st != ATTS_OK) return st;
  if (dtype != ATTS_BF16 && dtype != ATTS_FP16) return ATTS_ERR_ARG;
  if (M < 0 || M > (1ll << 30) || max_tokens < 0 || max_tokens > kMaxSlots) return ATTS_ERR_SHAPE;
  if (k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 || v_head_stride < 0) return ATTS_ERR_SHAPE;
  if (cache->num_seqs > 0 && (!ctx_lens || !cu_tokens)) return ATTS_ERR_NULL;
  if (M > 0 && (!k || !v)) return ATTS_ERR_NULL;
  if (!aligned(k, 2) || !aligned(v, 2) || !aligned(ctx_lens, 4) || !aligned(cu_tokens, 4)) return ATTS_ERR_ALIGN;
  const DeviceInfo* di;
  st = device_info(&di);
  if (st != ATTS_OK) return st;
  if (M == 0 || cache->num_seqs == 0 || max_tokens == 0) return ATTS_OK;
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.k_ts = k_token_stride; a.k_hs = k_head_stride; a.v_ts = v_token_stride; a.v_hs = v_head_stride;
  a.ctx = ctx_lens; a.cu = cu_tokens;
  a.D = cache->head_dim; a.M = (int)M; a.max_tokens = (int)max_tokens;
  a.tpb = pack_tokens(di->sm_count, M);
  const bool wide = (k_token_stride | k_head_stride | v_token_stride | v_head_stride) % 8 == 0 && aligned(k, 16) && aligned(v, 16);
  const dim3 grid((unsigned)((max_tokens + a.tpb - 1) / a.tpb), (unsigned)cache->num_seqs);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
#define ATTS_PACK(T, W) return launch_pdl(packed_append_kernel<T, W>, grid, dim3(kPackThreads), 0, stream, a, di->dev_status)
  if (dtype == ATTS_BF16) { if (wide) ATTS_PACK(__nv_bfloat16, true); else ATTS_PACK(__nv_bfloat16, false); }
  if (wide) ATTS_PACK(__half, true);
  ATTS_PACK(__half, false);
#undef ATTS_PACK
}

int atts_packed_read(const atts_packed_cache* src, const int32_t* lens, int64_t max_len, const atts_kv_cache* dst, void* cuda_stream) {
  ReadArgs a;
  int st = packed_view(src, &a.src);
  if (st != ATTS_OK) return st;
  if ((st = cache_view(dst, &a.dst)) != ATTS_OK) return st;
  if (src->heads != dst->heads || src->head_dim != dst->head_dim || src->num_seqs != dst->num_seqs) return ATTS_ERR_SHAPE;
  if (max_len < 0 || max_len > kMaxSlots) return ATTS_ERR_SHAPE;
  if (src->num_seqs > 0 && !lens) return ATTS_ERR_NULL;
  if (!aligned(lens, 4)) return ATTS_ERR_ALIGN;
  const DeviceInfo* di;
  st = device_info(&di);
  if (st != ATTS_OK) return st;
  if (src->num_seqs == 0 || max_len == 0) return ATTS_OK;
  a.lens = lens;
  a.D = src->head_dim; a.max_len = (int)max_len;
  a.tpb = pack_tokens(di->sm_count, src->num_seqs * max_len);
  const dim3 grid((unsigned)((max_len + a.tpb - 1) / a.tpb), (unsigned)src->num_seqs);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (dst->dtype == ATTS_BF16) return launch_pdl(packed_read_kernel<__nv_bfloat16>, grid, dim3(kPackThreads), 0, stream, a, di->dev_status);
  return launch_pdl(packed_read_kernel<__half>, grid, dim3(kPackThreads), 0, stream, a, di->dev_status);
}

int atts_norm_rope_append(const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k, int64_t k_token_stride,
                          int64_t k_head_stride, const void* v, int64_t v_token_stride, int64_t v_head_stride,
                          const int32_t* positions, const double* freqs, int32_t rotary_pairs, float mscale, int32_t interleaved,
                          const void* q_gain, const void* k_gain, float eps, const atts_kv_cache* cache, const int32_t* ctx_lens,
                          const int32_t* cu_tokens, int64_t M, int32_t Hq, int64_t max_tokens, void* q_out, int64_t out_token_stride,
                          int64_t out_head_stride, void* cuda_stream) {
  NormRopeArgs a;
  int st = cache_view(cache, &a.cache);
  if (st != ATTS_OK) return st;
  if (max_tokens < 0 || max_tokens > kMaxSlots || v_token_stride < 0 || v_head_stride < 0) return ATTS_ERR_SHAPE;
  if (cache->num_seqs > 0 && (!ctx_lens || !cu_tokens)) return ATTS_ERR_NULL;
  if (M > 0 && !v) return ATTS_ERR_NULL;
  if (!aligned(v, 2) || !aligned(ctx_lens, 4) || !aligned(cu_tokens, 4)) return ATTS_ERR_ALIGN;
  a.v = static_cast<const char*>(v);
  a.v_ts = v_token_stride; a.v_hs = v_head_stride;
  a.ctx = ctx_lens; a.cu = cu_tokens; a.max_tokens = (int)max_tokens;
  const bool none = cache->num_seqs == 0 || max_tokens == 0;
  const bool wide = (v_token_stride | v_head_stride) % 8 == 0 && aligned(v, 16);
  a.k_out = nullptr;
  a.ko_ts = a.ko_hs = 0;
  return norm_rope<false>(a, q, q_token_stride, q_head_stride, k, k_token_stride, k_head_stride, positions, freqs, rotary_pairs, mscale,
                          interleaved, q_gain, k_gain, eps, cache->dtype, M, Hq, cache->heads, cache->head_dim, q_out, out_token_stride,
                          out_head_stride, wide, none, cache->num_seqs, cuda_stream);
}

int atts_norm_rope(const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k, int64_t k_token_stride,
                   int64_t k_head_stride, const int32_t* positions, const double* freqs, int32_t rotary_pairs, float mscale,
                   int32_t interleaved, const void* q_gain, const void* k_gain, float eps, int32_t dtype, int64_t M, int32_t Hq,
                   int32_t Hk, int32_t head_dim, void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, void* k_out,
                   int64_t k_out_token_stride, int64_t k_out_head_stride, void* cuda_stream) {
  if (dtype != ATTS_BF16 && dtype != ATTS_FP16) return ATTS_ERR_ARG;
  if (head_dim < 8 || head_dim > 256 || head_dim % 8 != 0 || Hk < 0 || Hk > (1 << 20)) return ATTS_ERR_SHAPE;
  if (k_out_token_stride < 0 || k_out_head_stride < 0) return ATTS_ERR_SHAPE;
  if (M > 0 && Hk > 0 && !k_out) return ATTS_ERR_NULL;
  if (!aligned(k_out, 2)) return ATTS_ERR_ALIGN;
  NormRopeArgs a = {};
  a.k_out = static_cast<char*>(k_out);
  a.ko_ts = k_out_token_stride; a.ko_hs = k_out_head_stride;
  const bool wide = Hk == 0 || ((k_out_token_stride | k_out_head_stride) % 8 == 0 && aligned(k_out, 16));
  return norm_rope<true>(a, q, q_token_stride, q_head_stride, k, k_token_stride, k_head_stride, positions, freqs, rotary_pairs, mscale,
                         interleaved, q_gain, k_gain, eps, dtype, M, Hq, Hk, head_dim, q_out, q_out_token_stride, q_out_head_stride, wide,
                         Hq + Hk == 0, 1, cuda_stream);
}

int atts_cache_weights(const void* q, int64_t q_token_stride, int64_t q_head_stride, const atts_kv_cache* cache,
                       const float* lse, const int32_t* ctx_lens, const int32_t* cu_tokens, const int32_t* pre,
                       const int32_t* end, int64_t M, int32_t Hq, int64_t max_tokens, int64_t max_len, float scale,
                       const float* weights_in, float* weights_out, int64_t weights_cols, void* cuda_stream) {
  WeightArgs a;
  int st = cache_view(cache, &a.q.cache);
  if (st != ATTS_OK) return st;
  st = check_queries(q, q_token_stride, q_head_stride, cache, ctx_lens, cu_tokens, pre, end, M, Hq, max_tokens, max_len, scale);
  if (st != ATTS_OK) return st;
  if (weights_cols < max_len || weights_cols > kMaxSlots) return ATTS_ERR_SHAPE;
  if ((M > 0 && !lse) || (cache->num_seqs > 0 && max_len > 0 && !weights_out)) return ATTS_ERR_NULL;
  if (!aligned(lse, 4) || !aligned(weights_in, 4) || !aligned(weights_out, 4)) return ATTS_ERR_ALIGN;
  const DeviceInfo* di;
  st = device_info(&di);
  if (st != ATTS_OK) return st;
  if (cache->num_seqs == 0 || max_len == 0) return ATTS_OK;
  const int G = Hq / cache->heads;
  a.q.q = static_cast<const char*>(q);
  a.q.out = nullptr;
  a.q.lse = nullptr;
  a.q.q_ts = q_token_stride; a.q.q_hs = q_head_stride; a.q.o_ts = 0; a.q.o_hs = 0;
  a.q.ctx = ctx_lens; a.q.cu = cu_tokens; a.q.pre = pre; a.q.end = end;
  a.q.M = (int)M; a.q.Hq = Hq; a.q.G = G; a.q.max_tokens = (int)max_tokens; a.q.max_len = (int)max_len;
  a.q.scale = scale;
  a.lse = lse;
  a.win = weights_in; a.wout = weights_out; a.wcols = weights_cols;
  a.tpt = row_tile_tokens(G, max_tokens);
  a.wait_limit = wait_limit();
  a.withhold_loads = g_withhold_loads.load(std::memory_order_relaxed);
  // One row tile: a CTA goes over as many slot tiles as leave two CTAs an SM something to do, eight at most (8 sequences of
  // 2000 slots, 8 heads: spans of 1, 2, 4 and 8 tiles take 25.0, 16.3, 11.8 and 14.2 us; inputs beyond L2, calls in a
  // graph).  More: cached tiles are dealt to clusters whose CTAs take at least two row tiles each, of at most four (8 drafts
  // of 500: clusters of 1, 2, 4 and 8 take 207, 126, 128 and 136 us).
  const int64_t nq = (max_tokens + a.tpt - 1) / a.tpt, tiles = (max_len + kAttnTile - 1) / kAttnTile;
  const bool many = nq > 1;
  a.cluster = 1;
  a.span = 1;
  if (many) {
    while (a.cluster < kWeightMaxCluster && nq >= 4 * a.cluster) a.cluster *= 2;
  } else {
    while (a.span < 8 && tiles * cache->heads * cache->num_seqs > 2 * a.span * (int64_t)di->sm_count) a.span *= 2;
  }
  const int64_t gx = (many ? tiles : (tiles + a.span - 1) / a.span) * cache->heads;   // clusters
  if (gx * a.cluster > 0x7FFFFFFF) return ATTS_ERR_SHAPE;
  const dim3 grid((unsigned)gx, (unsigned)cache->num_seqs);
  CUtensorMap mq, mk;
  // without queries (M == 0) the kernel only writes; the map then describes the cache's keys and is not used
  if (encode_queries(di, &mq, cache, M > 0 ? q : cache->k, q_token_stride, q_head_stride, M > 0 ? M : 1, M > 0 ? Hq : cache->heads, a.tpt) != ATTS_OK ||
      encode_cache(di, &mk, cache, cache->k) != ATTS_OK)
    return ATTS_ERR_CUDA;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const bool bf = cache->dtype == ATTS_BF16;
#define ATTS_WEIGH(D, MANY)                                                                  \
  (bf ? launch_weights<__nv_bfloat16, D, MANY>(mq, mk, a, grid, di->dev_status, stream)      \
      : launch_weights<__half, D, MANY>(mq, mk, a, grid, di->dev_status, stream))
  if (cache->head_dim == 128) return many ? ATTS_WEIGH(128, true) : ATTS_WEIGH(128, false);
  return many ? ATTS_WEIGH(64, true) : ATTS_WEIGH(64, false);
#undef ATTS_WEIGH
}

int atts_cache_select(const float* weights, int64_t weights_cols, const int32_t* lens, int64_t num_seqs, int32_t heads,
                      int64_t budget, int64_t sinks, int64_t recent, int32_t* kept, int32_t* counts, void* cuda_stream) {
  if (num_seqs < 0 || num_seqs > 65535 || heads < 1 || heads > 1024 || weights_cols < 0 || weights_cols > kMaxSlots)
    return ATTS_ERR_SHAPE;
  if (budget < 1 || budget > kMaxSlots || sinks < 0 || recent < 0 || sinks > budget || recent > budget || sinks + recent > budget)
    return ATTS_ERR_SHAPE;
  if (num_seqs > 0 && (!lens || !kept || !counts || (weights_cols > 0 && !weights))) return ATTS_ERR_NULL;
  if (!aligned(weights, 4) || !aligned(lens, 4) || !aligned(kept, 4) || !aligned(counts, 4)) return ATTS_ERR_ALIGN;
  const DeviceInfo* di;
  int st = device_info(&di);
  if (st != ATTS_OK) return st;
  if (num_seqs == 0) return ATTS_OK;
  const SelectArgs a{weights, weights_cols, lens, heads, (int)budget, (int)sinks, (int)recent, kept, counts};
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const dim3 grid((unsigned)(num_seqs * heads));
  // one block with the smallest number of keys a thread (of 1024, or of fewer for the shortest rows) that covers a row, then
  // clusters, then the form that reads the row again for every digit
  if (weights_cols > kSelectCluster * kSelectMaxItems * kSelectThreads)
    return launch_pdl(cache_select_long_kernel, grid, dim3(kSelectThreads), 0, stream, a, di->dev_status);
  const unsigned threads = weights_cols >= kSelectThreads ? kSelectThreads : (unsigned)round_up((size_t)(weights_cols < 1 ? 1 : weights_cols), 32);
  if (weights_cols <= 1024) return launch_pdl(cache_select_kernel<1, 1>, grid, dim3(threads), 0, stream, a, di->dev_status);
  if (weights_cols <= 4096) return launch_pdl(cache_select_kernel<4, 1>, grid, dim3(threads), 0, stream, a, di->dev_status);
  if (weights_cols <= 16384) return launch_pdl_cluster(cache_select_kernel<8, kSelectCluster>, grid, dim3(threads), 0, kSelectCluster, stream, a, di->dev_status);
  return launch_pdl_cluster(cache_select_kernel<kSelectMaxItems, kSelectCluster>, grid, dim3(threads), 0, kSelectCluster, stream, a, di->dev_status);
}

int atts_cache_gather(const atts_kv_cache* src, const int32_t* kept, int64_t kept_cols, const int32_t* counts,
                      const atts_kv_cache* dst, const float* weights_in, int64_t in_cols, float* weights_out,
                      void* cuda_stream) {
  CacheView s, d;
  int st = cache_view(src, &s);
  if (st != ATTS_OK) return st;
  if ((st = cache_view(dst, &d)) != ATTS_OK) return st;
  if (src->dtype != dst->dtype) return ATTS_ERR_ARG;
  if (src->heads != dst->heads || src->head_dim != dst->head_dim || src->num_seqs != dst->num_seqs) return ATTS_ERR_SHAPE;
  if (kept_cols < 0 || kept_cols > kMaxSlots || in_cols < 0 || in_cols > kMaxSlots) return ATTS_ERR_SHAPE;
  if (src->num_seqs > 0 && ((kept_cols > 0 && !kept) || !counts)) return ATTS_ERR_NULL;
  if ((weights_in == nullptr) != (weights_out == nullptr)) return ATTS_ERR_NULL;
  if (!aligned(kept, 4) || !aligned(counts, 4) || !aligned(weights_in, 4) || !aligned(weights_out, 4)) return ATTS_ERR_ALIGN;
  const DeviceInfo* di;
  st = device_info(&di);
  if (st != ATTS_OK) return st;
  if (src->num_seqs == 0 || kept_cols == 0) return ATTS_OK;
  const int lanes = src->head_dim / 8;
  int span = kGatherSpan;
  while (span > 32 && (kept_cols + span - 1) / span * src->heads * src->num_seqs < 2 * (int64_t)di->sm_count) span /= 2;
  const int64_t gx = (kept_cols + span - 1) / span * src->heads;
  if (gx > 0x7FFFFFFF) return ATTS_ERR_SHAPE;
  const dim3 grid((unsigned)gx, (unsigned)src->num_seqs);
  return launch_pdl(cache_gather_kernel, grid, dim3(kGatherThreads), 0, static_cast<cudaStream_t>(cuda_stream), s, d, lanes, span, kept, kept_cols,
                    counts, weights_in, in_cols, weights_out, di->dev_status);
}

}  // extern "C"
