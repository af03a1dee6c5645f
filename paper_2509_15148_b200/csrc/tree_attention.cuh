// Attention of drafted tokens over a paged cache, and attention weight per cached slot.
#pragma once
#include <math.h>

#include "conformal.cuh"
#include "lmhead_lse.cuh"
#include "packed_cache.cuh"
#include "rope_cache.cuh"

namespace atts {

struct AttnArgs {
  const char* q;
  char* out;
  float* lse;
  int64_t q_ts, q_hs, o_ts, o_hs;  // elements
  const int32_t *ctx, *cu, *pre, *end;
  int M, Hq, G, max_tokens, max_len;
  float scale;
  CacheView cache;          // (a packed cache: strides in bytes, no slot stride)
  // Windowed forms only.  A token's place on its line: a cached slot's number, or ctx + depth among the drafts.
  const int32_t* depth;     // NULL: chains
  int window, sinks;
};

// What a drafted token sees: the cached slots below ctx, and the drafted tokens j with lo(j) <= mine < hi(j).
struct SeqView {
  int first, n, ctx, len;
};
__device__ __forceinline__ bool seq_view(const int32_t* cu, const int32_t* ctx, int seq, int M, int max_tokens, int max_len,
                                         SeqView& s, unsigned* dev_status, bool record) {
  bool ok = seq_rows(cu, seq, M, s.first, s.n);
  s.ctx = ctx[seq];
  ok = ok && s.ctx >= 0 && s.ctx <= kMaxSlotsOfSeq && s.n <= max_tokens;   // (both at most 2^30: their sum fits)
  s.len = ok ? s.ctx + s.n : 0;
  if (record && (!ok || s.len > max_len)) atomicOr(dev_status, kDevSeqRange);
  s.len = min(s.len, max_len);
  return ok;
}

// ------------------------------------------------------------------------------------------------------------------
// PTX wrappers beyond those of lmhead_lse.cuh
// ------------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1, int c2, int c3) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
// Descriptors here are kept as their low word (address and leading offset); the high word is a constant and the step along
// K an immediate, added inside the instruction's block: whole descriptors, one per step and tile, would be kept in more
// registers than the issuing thread has, and every spilled one costs the tensor pipe a trip to L2.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);   // groups of eight rows 1024 bytes apart, 128-byte swizzle
__device__ __forceinline__ uint32_t desc_low(uint32_t smem_addr, uint32_t lbo) { return (smem_addr >> 4) | ((lbo >> 4) << 16); }
// One lane of a converged warp, always the same one.  A whole warp runs the issuing loops and one lane is elected around the
// products themselves: their operands then stay in the warp's uniform registers.  Issued from a loop that one lane runs by itself
// every operand is moved there first: about 110 cycles a product instead of the 64 that it takes the tensor pipe.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0u;
}
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }
// D[tmem] (+)= A[smem] * B[smem]^T, both at `step` 16-byte units from their descriptors.
__device__ __forceinline__ void umma_ss(uint32_t tmem_d, uint32_t a_low, uint32_t b_low, uint32_t step, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b32 x, y;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "add.u32 x, %1, %3;\n\tadd.u32 y, %2, %3;\n\t"
      "mov.b64 da, {x, %6};\n\tmov.b64 db, {y, %6};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}"
      ::"r"(tmem_d), "r"(a_low), "r"(b_low), "r"(step), "r"(idesc), "r"(accumulate), "r"(kDescHigh)
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem], the A operand packed two 16-bit values to a tensor-memory column.
__device__ __forceinline__ void umma_ts(uint32_t tmem_d, uint32_t tmem_a, uint32_t b_low, uint32_t step_a, uint32_t step_b, uint32_t idesc,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b32 x, y;\n\t.reg .b64 db;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "add.u32 x, %1, %3;\n\tadd.u32 y, %2, %4;\n\t"
      "mov.b64 db, {y, %7};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %5, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "r"(b_low), "r"(step_a), "r"(step_b), "r"(idesc), "r"(accumulate), "r"(kDescHigh)
      : "memory");
}
#define ATTS_TMEM_ST_16(taddr, v)                                                                                          \
  asm volatile(                                                                                                            \
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "                                                                      \
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),                              \
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),         \
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])                                                \
      : "memory")
#define ATTS_TMEM_LD_16(taddr, v)                                                                                          \
  asm volatile(                                                                                                            \
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "                                                                            \
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"                                     \
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),         \
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])                            \
      : "r"(taddr)                                                                                                         \
      : "memory")
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ------------------------------------------------------------------------------------------------------------------
// Tree attention.  A CTA takes tiles of 128 rows (the query heads of one key head for 128 / G tokens: grouped heads share
// the keys and values that are read) against the slots of its sequence, 128 at a time:
//   S = Q K^T (tcgen05, fp32 in tensor memory) -> one thread per row: running maximum, p = 2^(c s - c m), sum
//   -> p rounded to the inputs' type, back into tensor memory over S -> O += P V (A operand from tensor memory).
// Two streams of this alternate on the tensor pipe, so that one's products hide the other's exponentials:
//   kRowsTwo: two row tiles against the same slots;  kRowsOne: one row tile, even and odd slot tiles, joined at the end.
// Short sequences in great number take kRowsBrief instead, one stream a CTA and two CTAs an SM: what a CTA costs to start and
// end (about 9 us) is then hidden by the other one (384 CTAs of two tiles: 41 us with kRowsOne, 30 us; 128 CTAs of up to
// 20 tiles: 38 against 50 us, since half the shared memory leaves no room to load ahead).
// Bound: few rows over a long cache (4 x 13 tokens, 32 / 8 heads of 128, 131,071 slots) 332 to 367 us on different GPUs = 4.6 to
// 5.1 TB/s; many rows (chunk of 2048 over 6144, 64 / 8 heads) 881 to 920 us = 921 to 961 TFLOP/s, where a stream's chain of scores,
// exponentials (1,400 of a round's 3,750 cycles) and products keeps the tensor pipe 55 % busy and the power cap sets the clock.
// Probabilities are rounded because the tensor pipe multiplies 16-bit operands: the output's error against 64 bits is 0.0019 of it
// in bf16 and 0.00028 in fp16, where the output's own rounding makes 0.0017 and 0.00021; the sums are of the unrounded ones.
// Registers: ptxas spills 8 to 24 bytes a thread, loaded again 472 to 476 bytes' worth in kRowsOne and 140 to 148 in the others; windowed
// forms 20 in kRowsHalf (loaded again 192 to 196) and none in the others; packed forms 36 to 72 (52 to 80), none in kRowsHalf.
// The running maximum that p refers to only moves when a row exceeds it by 2^8: p <= 256, and
// O is rescaled (a pass over tensor memory) in a few tiles instead of in every one.
// The slots may be cut into chunks of `chunk` tiles over CTAs (few rows, long caches); the parts are then joined by
// attention_join_kernel.
//
// Which of the tiles behind the cached part a CTA needs, and in which groups of 32 slots pairs have to be looked at one by
// one, is listed while the cached tiles are already on their way: the rows' warps look at a tile each, warp 3 makes the
// list; whoever comes to the end of the cached tiles waits for it.
//
// Warps: 0 and 2 load (TMA, one box per page and 64 channels), 1 issues the products, 3 makes the list, lays out the intervals
// of the tiles that need them and clears the values of slots that hold nothing (whatever lies there, 0 * NaN must not reach
// O), 4-7 and 8-11 are the two streams' rows.
// ------------------------------------------------------------------------------------------------------------------
//
// Windowed form: a row sees, of all that the tree lets it see, the places nearer than `window` to its own and the first `sinks`.
// The cached tiles between the sinks and the first place that any of the CTA's rows sees are left out of the count of tiles
// (WindowView), so neither time nor chunks are spent on them; at the window's edge pairs are looked at one by one, as in a tree.
// Packed form: the cache holds 4 bits a channel (packed_cache.cuh).  Warps 0 and 2 bring codes and scales into a ring of raw tiles
// (one bulk copy a page), eight more warps (12-19) expand them into the ring that the products read, with zeros for slots that hold
// nothing; the expanded values are exact, so everything behind is the same arithmetic.  A warp takes about 1,400 cycles to expand 32
// slots of a tile beside the rows' warps (shifts, masks and multiply-adds at half rate): with four of them expanding set the pace
// (16 trees of up to 24 tokens over 1500 to 2500 slots 67 us, 8 drafts of 500 over 1013 256; with eight 39 and 192, in 16 bits 38
// and 165).
// At most 64 rows (windowed and packed forms): kRowsHalf is kRowsOne with every row there twice, in the upper and in the lower half of the
// row tile.  The upper one takes the first 64 slots of each tile and the lower one the others (zeros for the rest in the products with
// V), each with maxima and sums of its own, so that a tile's chain of maximum and exponentials is half as long and all four
// schedulers work on it, where otherwise the warps of the lower half had no rows; the halves are joined with the streams at the end.
// 4 x 13 tokens over 131,071 packed slots: 305 us (kRowsOne 353); one token of 8 samples through a window of 1024: 22.6 (24.2).
enum AttnMode { kRowsTwo, kRowsOne, kRowsBrief, kRowsHalf };
enum AttnForm { kFormPlain = 0, kFormWindow = 1, kFormPacked = 2, kFormPackedWindow = 3 };
constexpr int kAttnTile = 128;          // rows of a tile, slots of a tile
constexpr int kAttnTreeTiles = 1024;    // tiles behind the cached part that are listed; further ones are all looked at
constexpr int kMaskRing = 4;

template <int D, AttnMode MODE, AttnForm FORM = kFormPlain>
struct AttnCfg {
  static constexpr bool kWindow = (FORM & 1) != 0, kPacked = (FORM & 2) != 0;
  static constexpr int kStreams = MODE == kRowsBrief ? 1 : 2;
  static constexpr int kExpand = 8;                                  // warps that expand a packed cache's tiles
  static constexpr int kThreads = 128 + 128 * kStreams + (kPacked ? 32 * kExpand : 0);
  static constexpr int kTmem = 256 * kStreams;                       // columns: scores (over them the probabilities), then O
  static constexpr int kTileBytes = kAttnTile * D * 2;
  static constexpr int kQBytes = (MODE == kRowsTwo ? 2 : 1) * kTileBytes;
  static constexpr int kStages = kPacked ? (D == 128 ? (MODE == kRowsTwo ? 3 : 4) : 6)
                                 : D == 128 ? (MODE == kRowsTwo ? 4 : MODE == kRowsBrief ? 2 : 5) : MODE == kRowsBrief ? 4 : 8;
  static constexpr int kRawStages = !kPacked ? 0 : D == 128 ? (MODE == kRowsTwo ? 4 : 6) : 8;
  static constexpr int kRawBytes = kAttnTile / 8 * packed_eight(D);
  static constexpr int kRing = kQBytes;                              // byte offsets in (aligned) shared memory
  static constexpr int kMask = kRing + kStages * kTileBytes;         // [kMaskRing][128] int2
  static constexpr int kPlaces = kMask + kMaskRing * kAttnTile * 8;  // [kMaskRing][128] int, windowed forms
  static constexpr int kRaw = kPlaces + (kWindow ? kMaskRing * kAttnTile * 4 : 0);   // [kRawStages] raw tiles, packed form
  static constexpr int kList = kRaw + kRawStages * kRawBytes;        // [kAttnTreeTiles] uint32
  static constexpr int kStats = kList + kAttnTreeTiles * 4;          // [128] float2: maximum and sum of the odd stream; kRowsHalf [3][64]
  static constexpr int kBars = kStats + (MODE == kRowsHalf ? 192 : kAttnTile) * 8;
  static constexpr int kSmemBytes = kBars + 512 + 1024;
  static constexpr int kLead = MODE == kRowsOne || MODE == kRowsHalf ? 2 : 1;             // key tiles loaded ahead of the first value tile
  static_assert(kSmemBytes <= 232448, "shared memory of one SM");
  static_assert(MODE != kRowsBrief || 2 * (kSmemBytes + 1024) <= 233472, "two CTAs share an SM");
  static_assert(MODE != kRowsHalf || kStages * kTileBytes >= 192 * (D + 4) * 4, "the other sums of a row are joined through the ring");
  static_assert(MODE != kRowsOne || kStages * kTileBytes >= kAttnTile * (D + 4) * 4, "the odd stream's sums are joined through the ring");
};

// A tile's flags: two bits for each group of 32 slots (0 nobody sees any, 1 pairs differ, 2 everybody sees all), then
enum : uint32_t {
  kTileDead = 1u << 8,      // some slots hold nothing
  kTileMasked = 1u << 9,    // some group is neither empty nor full
  kTileFull = 0xAAu,
  kTileUnknown = 0x55u | kTileDead | kTileMasked
};

struct AttnPlan {
  int chunk;        // slot tiles per CTA
  int nq, chunks;   // row tiles (or pairs of them) and chunks of the longest sequence
  int tpt;          // tokens per row tile
  float* part_o;    // [M * Hq][chunks][D]
  float* part_lse;  // [M * Hq][chunks], base 2
  long long wait_limit;
  int withhold_loads;
};

template <typename T>
struct AttnType;
template <>
struct AttnType<__nv_bfloat16> { static constexpr uint32_t fmt = 1; static constexpr float shift = 0.f; };
// fp16 probabilities are carried 2^6 larger (they stay below 2^14): those under 2^-14 would lose digits otherwise.
template <>
struct AttnType<__half> { static constexpr uint32_t fmt = 0; static constexpr float shift = 6.f; };

// What slots of a tile hold, as the interval of preorder places that see them: mine is in it iff
// (unsigned)(mine - x) < (unsigned)y.
__device__ __forceinline__ int2 slot_interval(const AttnArgs& a, const SeqView& s, int slot) {
  if (slot < s.ctx && slot < s.len) return make_int2(0, 0x7FFFFFFF);
  if (slot >= s.len) return make_int2(0, 0);
  const int j = slot - s.ctx;
  if (!a.pre) return make_int2(j, 0x7FFFFFFF);
  const int lo = a.pre[s.first + j], hi = a.end[s.first + j];
  return (lo < 0 || hi <= lo) ? make_int2(0, 0) : make_int2(lo, hi - lo);
}

// Depth of drafted token j, and the place on its line of what a slot holds (any number where it holds nothing).  A depth that
// no tree can have is cut to what one can, so that places stay below a sequence's length.
__device__ __forceinline__ int draft_depth(const AttnArgs& a, const SeqView& s, int j) {
  return a.depth ? max(0, min(a.depth[s.first + j], s.n - 1)) : j;
}
__device__ __forceinline__ int slot_place(const AttnArgs& a, const SeqView& s, int slot) {
  const int j = slot - s.ctx;
  return j < 0 || j >= s.n ? slot : s.ctx + draft_depth(a, s, j);
}

// What the window leaves of a sequence for rows whose depths span [dmin, dmax]: tiles are numbered without the `skip` ones from number
// `sink_tiles` on, of which no row sees anything.
struct WindowView {
  int near_first, near_all;   // the shallowest row sees places from near_first on, every row those from near_all on
  int sink_tiles, skip;
  int full_from;              // every row sees the whole of cached tiles from this one on
  bool live;                  // some row is not padding
  __device__ __forceinline__ int tile(int number) const { return number < sink_tiles ? number : number + skip; }
};
__device__ __forceinline__ WindowView window_view(const AttnArgs& a, const SeqView& s, int tok0, int ntok, int ntiles, int lane) {
  int dmin = 0x7FFFFFFF, dmax = -1;
  for (int t = tok0 + lane; t < tok0 + ntok; t += 32) {
    if (a.pre && a.pre[s.first + t] < 0) continue;
    const int d = draft_depth(a, s, t);
    dmin = min(dmin, d);
    dmax = max(dmax, d);
  }
  dmin = __reduce_min_sync(0xFFFFFFFFu, dmin);
  dmax = __reduce_max_sync(0xFFFFFFFFu, dmax);
  WindowView w;
  w.live = dmax >= 0;
  if (!w.live) dmin = dmax = 0;
  w.near_first = s.ctx + dmin - a.window + 1;             // (at most 2^30 each: the sum fits)
  w.near_all = s.ctx + dmax - a.window + 1;
  // A drafted token's slot is never below its place, so the first places that rows see bound the slots too; but a token of a low
  // place (a sink) may lie anywhere among the drafts, so where the drafts have sinks none of their tiles is left out.
  int first = max(0, w.near_first) / kAttnTile;
  if (s.ctx < a.sinks) first = min(first, s.ctx / kAttnTile);
  first = min(first, ntiles);
  w.sink_tiles = min((int)(((int64_t)a.sinks + kAttnTile - 1) / kAttnTile), first);
  w.skip = first - w.sink_tiles;
  w.full_from = (max(0, w.near_all) + kAttnTile - 1) / kAttnTile;
  return w;
}

// The same for a whole tile by one warp, slots e * 32 + lane, all loads under way at once.
__device__ __forceinline__ void tile_intervals(const AttnArgs& a, const SeqView& s, int tile, int lane, int2 (&v)[kAttnTile / 32]) {
  constexpr int E = kAttnTile / 32;
  int lo[E], hi[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int j = tile * kAttnTile + e * 32 + lane - s.ctx;
    lo[e] = hi[e] = 0;
    if (a.pre && j >= 0 && j < s.n) {
      lo[e] = a.pre[s.first + j];
      hi[e] = a.end[s.first + j];
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int slot = tile * kAttnTile + e * 32 + lane;
    if (slot >= s.len) v[e] = make_int2(0, 0);
    else if (slot < s.ctx) v[e] = make_int2(0, 0x7FFFFFFF);
    else if (!a.pre) v[e] = make_int2(slot - s.ctx, 0x7FFFFFFF);
    else v[e] = (lo[e] < 0 || hi[e] <= lo[e]) ? make_int2(0, 0) : make_int2(lo[e], hi[e] - lo[e]);
  }
}

// The window's part of a slot's visibility: whether any row sees place x, whether every row does.
__device__ __forceinline__ bool window_any(const AttnArgs& a, const WindowView& w, int x) { return x >= w.near_first || x < a.sinks; }
__device__ __forceinline__ bool window_all(const AttnArgs& a, const WindowView& w, int x) { return x >= w.near_all || x < a.sinks; }

// Flags of a tile of cached slots under a window.
__device__ __forceinline__ uint32_t window_flags(const AttnArgs& a, const WindowView& w, int tile) {
  if (tile >= w.full_from) return kTileFull;              // nearly all of them
  uint32_t f = 0;
#pragma unroll
  for (int e = 0; e < kAttnTile / 32; ++e) {
    const int x = tile * kAttnTile + e * 32, last = x + 31;
    if (x >= w.near_all || last < a.sinks) f |= 2u << (2 * e);
    else if (last >= w.near_first || x < a.sinks) f |= (1u << (2 * e)) | kTileMasked;
  }
  return f;
}

// Flags of one tile for rows whose places span [qmin, qmax] (whole warp); 0: nobody sees anything of it.
template <bool WINDOW = false>
__device__ __forceinline__ uint32_t tile_flags(const AttnArgs& a, const SeqView& s, int tile, int qmin, int qmax, int lane,
                                               const WindowView* w = nullptr) {
  uint32_t f = 0;
  int2 v[kAttnTile / 32];
  tile_intervals(a, s, tile, lane, v);
#pragma unroll
  for (int e = 0; e < kAttnTile / 32; ++e) {
    const unsigned last = (unsigned)v[e].x + (unsigned)v[e].y;    // one past the interval
    const bool none = v[e].y == 0;
    bool in = true, in_all = true;
    if (WINDOW) {
      const int x = slot_place(a, s, tile * kAttnTile + e * 32 + lane);
      in = window_any(a, *w, x);
      in_all = window_all(a, *w, x);
    }
    const bool any = __any_sync(0xFFFFFFFFu, !none && in && v[e].x <= qmax && (unsigned)qmin < last);
    const bool all = __all_sync(0xFFFFFFFFu, !none && in_all && v[e].x <= qmin && (unsigned)qmax < last);
    if (any) f |= all ? 2u << (2 * e) : (1u << (2 * e)) | kTileMasked;
    if (__any_sync(0xFFFFFFFFu, none)) f |= kTileDead;
  }
  return (f & 0xFFu) ? f : 0u;
}

// Loads a tile of slots, a lane per box (one page, 64 channels).  A TMA instruction costs its warp about 117 cycles when one
// lane issues one after the other and 56 when lanes issue side by side, whatever its size, and warps do not disturb one
// another (measured, boxes of 8 to 128 rows): so small pages are issued by many lanes, keys and values by two warps.
template <int D, int kHalves = D / 64>
struct TileBoxes {
  int page_log2, rows, boxes, slot;   // slots of a box, boxes of a tile (<= 32), this lane's first slot in the tile
  __device__ __forceinline__ TileBoxes(int page_log2_, int lane) : page_log2(page_log2_) {
    rows = min(1 << page_log2, kAttnTile);
    boxes = (kAttnTile / rows) * kHalves;
    slot = (lane / kHalves) * rows;
  }
  __device__ __forceinline__ void issue(uint32_t dst, const CUtensorMap* map, uint32_t bar, int tile, int hk, int page, int lane) const {
    if (lane < boxes)
      tma_load_4d(dst + (uint32_t)(lane % kHalves) * (kAttnTile * 128) + (uint32_t)slot * 128u, map, bar, (lane % kHalves) * 64,
                  (tile * kAttnTile + slot) & ((1 << page_log2) - 1), hk, page);
    __syncwarp();
  }
};

// Loads one row tile's 32 columns, scales by the row's factor, stores them back.
template <int D>
__device__ __forceinline__ void rescale_o(uint32_t taddr, float f) {
#pragma unroll 1
  for (int j = 0; j < D / 16; ++j) {   // few columns at a time: the row's scores are in registers meanwhile
    uint32_t v[16];
    ATTS_TMEM_LD_16(taddr + 16u * j, v);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
    ATTS_TMEM_ST_16(taddr + 16u * j, v);
  }
  tmem_st_wait();
}

// One bulk copy of a contiguous piece (addresses and size multiples of 16 bytes).
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar) : "memory");
}

// A part of a raw tile (16 slots) by one warp into the 16-bit tile that the products read: blocks of 64 channels, a row of 128
// bytes a slot, 16-byte pieces swizzled by the row.  A thread takes a group of 32 channels; groups 2 and 3 write their pieces in
// another order than groups 0 and 1, so that eight threads that store together never share a bank.  `dead`: bit per turn, slots that
// hold nothing (zeros, whatever lies there).
template <typename T, int D>
__device__ __forceinline__ void expand_rows(uint32_t raw, uint32_t tile, int first, int lane, uint32_t dead) {
  constexpr int kPer = D / 32, kRows = 32 / kPer, kTurns = 16 / kRows;    // threads a slot, slots a turn
  const int g = lane % kPer, row = first + lane / kPer, r7 = row & 7;   // of the first turn; r7 is every turn's
  const bool swap = g >= 2;
  const uint32_t codes = raw + (uint32_t)((row >> 3) * packed_eight(D) + r7 * (D / 2) + g * 16);
  const uint32_t scales = raw + (uint32_t)((row >> 3) * packed_eight(D) + 4 * D + r7 * (D / 32) + g);
  uint32_t out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = tile + (uint32_t)((g >> 1) * (kAttnTile * 128) + row * 128 + ((((g & 1) * 4 + (swap ? i ^ 2 : i)) ^ r7) * 16));
  uint4 w[kTurns];
  uint32_t byte[kTurns];
#pragma unroll
  for (int it = 0; it < kTurns; ++it) {                   // every load is on its way before the first store
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[it].x), "=r"(w[it].y), "=r"(w[it].z), "=r"(w[it].w)
                 : "r"(codes + it * (kRows / 8) * packed_eight(D)));
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(byte[it]) : "r"(scales + it * (kRows / 8) * packed_eight(D)));
  }
#pragma unroll
  for (int it = 0; it < kTurns; ++it) {
    if ((dead >> it) & 1u) {
      w[it] = make_uint4(0x88888888u, 0x88888888u, 0x88888888u, 0x88888888u);
      byte[it] = 0;
    }
    uint32_t s2, m2;
    const float sc = packed_scale(byte[it]);
    Expand<T>::scale(sc, sc, s2, m2);
    const uint32_t word[4] = {swap ? w[it].z : w[it].x, swap ? w[it].w : w[it].y, swap ? w[it].x : w[it].z, swap ? w[it].y : w[it].w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(out[i] + it * kRows * 128), "r"(expand_pair<T, 0>(word[i], s2, m2)),
                   "r"(expand_pair<T, 1>(word[i], s2, m2)), "r"(expand_pair<T, 2>(word[i], s2, m2)), "r"(expand_pair<T, 3>(word[i], s2, m2)) : "memory");
  }
}

template <typename T, int D, AttnMode MODE, AttnForm FORM>
__global__ void __launch_bounds__(AttnCfg<D, MODE, FORM>::kThreads, MODE == kRowsBrief ? 2 : 1)
tree_attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttnArgs a,
                      const __grid_constant__ AttnPlan plan, unsigned* __restrict__ dev_status) {
  using Cfg = AttnCfg<D, MODE, FORM>;
  constexpr bool WINDOW = Cfg::kWindow, PACKED = Cfg::kPacked;
  constexpr bool HALF = MODE == kRowsHalf, TWO = MODE != kRowsOne && !HALF;   // TWO: a stream's rows are its own, and it takes every tile
  constexpr int kStreams = Cfg::kStreams;
  constexpr uint32_t kO = 128u * kStreams;              // first column of O
  constexpr int kStages = Cfg::kStages;
  constexpr int kLead = Cfg::kLead;
  extern __shared__ uint8_t smem_raw[];
  const int seq = blockIdx.z, hk = blockIdx.y;
  const int qt = plan.nq - 1 - (int)(blockIdx.x % plan.nq), chunk = blockIdx.x / plan.nq;   // late rows see most: first

  pdl_wait();
  // ---- what this CTA works on: nothing at all, or rows [tok0, tok0 + ntok) and slot tiles [tile0, tile1) ----
  SeqView s;
  if (!seq_view(a.cu, a.ctx, seq, a.M, a.max_tokens, a.max_len, s, dev_status, threadIdx.x == 0 && blockIdx.x == 0 && hk == 0)) return;
  const int per = plan.tpt * (MODE == kRowsTwo ? 2 : 1);
  const int tok0 = qt * per;
  if (tok0 >= s.n) return;
  const int ntok = min(per, s.n - tok0);
  int ntiles = (s.len + kAttnTile - 1) / kAttnTile;
  int tree0 = min(s.ctx, s.len) / kAttnTile;          // first tile that is not all cached slots (a cache cut at max_len ends inside one)
  WindowView win;
  if (WINDOW) {                                       // tile numbers from here on leave out what no row sees
    win = window_view(a, s, tok0, ntok, ntiles, threadIdx.x & 31);
    const int first = win.sink_tiles + win.skip;
    tree0 = tree0 >= first ? tree0 - win.skip : min(tree0, win.sink_tiles);
    ntiles -= win.skip;
  }
  const int tile0 = chunk * plan.chunk, tile1 = min(ntiles, tile0 + plan.chunk);
  if (chunk > 0 && tile0 >= ntiles) {
    // the join of a windowed batch does not know how many tiles a row tile had: it asks every chunk
    if (WINDOW)
      for (int i = threadIdx.x; i < ntok * a.G; i += Cfg::kThreads)
        plan.part_lse[((int64_t)(s.first + tok0 + i / a.G) * a.Hq + hk * a.G + i % a.G) * plan.chunks + chunk] = -INFINITY;
    return;
  }
  const bool two = MODE == kRowsTwo && ntok > plan.tpt;

  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  int2* mask = reinterpret_cast<int2*>(smem + Cfg::kMask);
  int* places = reinterpret_cast<int*>(smem + Cfg::kPlaces);
  volatile uint32_t* list = reinterpret_cast<volatile uint32_t*>(smem + Cfg::kList);
  float2* stats = reinterpret_cast<float2*>(smem + Cfg::kStats);
  const uint32_t bar0 = smem_base + Cfg::kBars;
  auto full_bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
  auto empty_bar = [&](int i) { return bar0 + 8u * (uint32_t)(kStages + i); };
  // One for each stage, so that warp 3 cannot be two completions ahead of warp 1 (whose wait by parity would not see the first):
  // a stage is cleaned again only after it was refilled, and refilled only after warp 1's products released it.
  auto clean_bar = [&](int i) { return bar0 + 8u * (uint32_t)(2 * kStages + i); };
  const uint32_t q_bar = bar0 + 8u * (3 * kStages), join_bar = q_bar + 8u, flag_bar = q_bar + 16u, list_bar = q_bar + 24u;
  auto s_bar = [&](int i) { return q_bar + 32u + 8u * (uint32_t)i; };
  auto p_bar = [&](int i) { return q_bar + 48u + 8u * (uint32_t)i; };
  auto o_bar = [&](int i) { return q_bar + 64u + 8u * (uint32_t)i; };
  auto m_full = [&](int i) { return q_bar + 80u + 8u * (uint32_t)i; };
  auto m_empty = [&](int i) { return q_bar + 80u + 8u * (uint32_t)(kMaskRing + i); };
  auto raw_full = [&](int i) { return q_bar + 80u + 8u * (uint32_t)(2 * kMaskRing + i); };
  auto raw_empty = [&](int i) { return q_bar + 80u + 8u * (uint32_t)(2 * kMaskRing + Cfg::kRawStages + i); };
  constexpr int kBarCount = 3 * kStages + 10 + 2 * kMaskRing + 2 * Cfg::kRawStages;
  static_assert(8 * kBarCount + 32 <= 512, "room for the barriers");
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + Cfg::kBars + 8 * kBarCount);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  volatile int* range = reinterpret_cast<volatile int*>(tmem_slot + 2);   // smallest and largest place of the rows
  volatile int* listed = range + 2;                                       // entries of the list

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    prefetch_tmap(&map_q);
    if (!PACKED) {
      prefetch_tmap(&map_k);
      prefetch_tmap(&map_v);
    }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(full_bar(i), PACKED ? Cfg::kExpand : 1);     // the copies, or the warps that expand
      mbar_init(empty_bar(i), PACKED ? 1 : 2);    // the products that read the stage, and warp 3
      mbar_init(clean_bar(i), 1);
    }
    for (int i = 0; i < Cfg::kRawStages; ++i) {
      mbar_init(raw_full(i), 1);
      mbar_init(raw_empty(i), Cfg::kExpand);
    }
    mbar_init(q_bar, 1);
    mbar_init(join_bar, HALF ? 6 : 4);
    mbar_init(flag_bar, 4 * kStreams);
    mbar_init(list_bar, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_bar(i), 1);
      mbar_init(p_bar(i), 4);
      mbar_init(o_bar(i), 1);
    }
    for (int i = 0; i < kMaskRing; ++i) {
      mbar_init(m_full(i), 1);
      mbar_init(m_empty(i), two ? 8 : 4);   // the warps that read it
    }
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"((uint32_t)Cfg::kTmem) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (warp == 2) {
    int lo = 0x7FFFFFFF, hi = -1;
    for (int t = lane; t < ntok; t += 32) {
      const int p = a.pre ? a.pre[s.first + tok0 + t] : tok0 + t;
      if (p >= 0) lo = min(lo, p);
      hi = max(hi, p);
    }
    lo = __reduce_min_sync(0xFFFFFFFFu, lo);
    hi = __reduce_max_sync(0xFFFFFFFFu, hi);
    if (lane == 0) {
      range[0] = lo;
      range[1] = hi;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const long long limit = plan.wait_limit;
  auto wait_one = [&](uint32_t bar, uint32_t parity) { return mbar_wait(bar, parity, abort_flag, limit, 0u); };
  auto wait_warp = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, wait_one(bar, parity)) != 0; };

  // The CTA's visible tiles: number i is tile0 + i among the cached ones (none if every row is padding), then the listed
  // ones of [t0, t0 + kAttnTreeTiles), then all further ones.
  const bool rows_live = range[1] >= 0;
  const int t0 = max(tile0, tree0), t_far = min(tile1, t0 + kAttnTreeTiles);
  const int npre = rows_live ? max(0, min(tile1, tree0) - tile0) : 0;
  int nlist = -1, ntile = npre;           // known once the list has been waited for
  auto has = [&](int i, bool one_thread) -> bool {
    if (i < npre) return true;
    if (nlist < 0) {
      if (!(one_thread ? wait_one(list_bar, 0) : wait_warp(list_bar, 0))) return false;   // gave up: every other wait does too
      nlist = *listed;
      ntile = npre + nlist + (rows_live ? max(0, tile1 - t0 - kAttnTreeTiles) : 0);
    }
    return i < ntile;
  };
  auto tile_at = [&](int number) { return WINDOW ? win.tile(number) : number; };
  auto tile_of = [&](int i, uint32_t& f) -> int {
    f = kTileFull;
    if (i < npre) {
      const int t = tile_at(tile0 + i);
      if (WINDOW) f = window_flags(a, win, t);
      return t;
    }
    if (i - npre < nlist) {
      const uint32_t e = list[i - npre];
      f = e & 0xFFFFu;
      return tile_at(t0 + (int)(e >> 16));
    }
    f = kTileUnknown;
    return tile_at(t0 + kAttnTreeTiles + (i - npre - nlist));
  };
  // Where a tile of keys or values stands in the rings' order: K_0 .. K_{lead-1}, then V_i, K_{i+lead}.  Before V_i come i values
  // and min(lead + i, ntile) keys.
  auto place_of = [&](int i, bool value) {
    return value ? (has(kLead + i - 1, false) ? kLead + 2 * i : ntile + i) : i < kLead ? i : 2 * i - kLead + 1;
  };

  pdl_launch_dependents();

  // A row's 128 scores stay in registers: 224 (200) for the rows' warps and 56 for the others, 384 x 168 (256 x 128) in all as
  // launched; packed form 168, 56 and 40 for those that expand, of 640 x 96.
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 0 || warp == 2) {
      // ---------------- loads: keys (and the queries) by warp 0, values by warp 2.  The ring's order is that of use:
      // K_0 .. K_{lead-1}, then V_i, K_{i+lead} ----------------
      const TileBoxes<D, PACKED ? 1 : D / 64> bx(a.cache.page_log2, lane);
      constexpr int kNoSlot = -2;                               // nothing that anybody sees: no page, filled with zeros
      auto look_up = [&](int i) -> int {                        // the table's entry for this lane's box, not looked at yet
        if (!has(i, false)) return kNoSlot;
        uint32_t f;
        const int slot = tile_of(i, f) * kAttnTile + bx.slot;
        if (lane >= bx.boxes || slot >= s.len) return kNoSlot;
        // a page of which no row sees anything need not be there: what is behind a window may have been freed
        if (WINDOW && slot + bx.rows <= min(s.ctx, win.near_first) && slot >= a.sinks) return kNoSlot;
        const int col = slot >> bx.page_log2;
        return col < a.cache.table_cols ? a.cache.table[(int64_t)seq * a.cache.table_stride + col] : -1;
      };
      auto page_of = [&](int entry) -> int {
        if (entry >= 0 && entry < a.cache.num_pages) return entry;
        if (entry != kNoSlot) atomicOr(dev_status, kDevPageRange);
        return a.cache.num_pages;                               // out of the map: filled with zeros
      };
      if (!plan.withhold_loads) {
        const bool value = warp == 2;
        int e0 = look_up(0);                                    // entries of the next two tiles
        if (!value && lane == 0 && has(0, true)) {              // nothing is loaded that nothing waits for
          mbar_expect_tx(q_bar, (uint32_t)((two || HALF ? 2 : 1) * a.G * plan.tpt * D * 2));
          for (int i = 0; i < (two || HALF ? 2 : 1); ++i)
            for (int c = 0; c < D / 64; ++c)
              tma_load_3d(smem_base + (uint32_t)i * (HALF ? 64 * 128 : Cfg::kTileBytes) + (uint32_t)c * (kAttnTile * 128), &map_q, q_bar, c * 64, hk * a.G,
                          s.first + tok0 + (HALF ? 0 : i * plan.tpt));
        }
        __syncwarp();
        int e1 = look_up(1);
        bool ok = true;
        for (int i = 0; ok && has(i, false); ++i) {
          const int page = page_of(e0);
          e0 = e1;
          e1 = look_up(i + 2);
          const int pos = place_of(i, value);
          if constexpr (PACKED) {
            // Raw tiles: a page's piece of the tile is contiguous.  A missing page reads as zeros, and so does one that nobody sees;
            // slots behind the sequence are left as they are (the warps that expand them look at the lengths).
            const int stage = pos % Cfg::kRawStages;
            ok = wait_warp(raw_empty(stage), ((uint32_t)(pos / Cfg::kRawStages) & 1u) ^ 1u);
            if (!ok) break;
            uint32_t f;
            const int slot = tile_of(i, f) * kAttnTile + bx.slot;
            const uint32_t bytes = (uint32_t)(bx.rows / 8) * packed_eight(D);
            const uint32_t dst = smem_base + Cfg::kRaw + (uint32_t)stage * Cfg::kRawBytes + (uint32_t)(bx.slot / 8) * packed_eight(D);
            const bool copied = page < a.cache.num_pages, missing = !copied && lane < bx.boxes && slot < s.len;
            if (missing) {
              for (uint32_t o = 0; o < bytes; o += 16)
                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(dst + o), "r"(0u) : "memory");
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            const uint32_t copies = __popc(__ballot_sync(0xFFFFFFFFu, copied));
            __syncwarp();
            if (lane == 0) mbar_expect_tx(raw_full(stage), copies * bytes);
            __syncwarp();
            if (copied)
              bulk_load(dst, (value ? a.cache.v : a.cache.k) + (int64_t)page * a.cache.page_stride + (int64_t)hk * a.cache.head_stride +
                                 (int64_t)((slot & ((1 << a.cache.page_log2) - 1)) / 8) * packed_eight(D),
                        bytes, raw_full(stage));
            __syncwarp();
            continue;
          }
          const int stage = pos % kStages;
          ok = wait_warp(empty_bar(stage), ((uint32_t)(pos / kStages) & 1u) ^ 1u);
          if (!ok) break;
          if (lane == 0) mbar_expect_tx(full_bar(stage), Cfg::kTileBytes);
          __syncwarp();
          uint32_t f;
          bx.issue(smem_base + Cfg::kRing + (uint32_t)stage * Cfg::kTileBytes, value ? &map_v : &map_k, full_bar(stage), tile_of(i, f), hk, page, lane);
        }
      }
    } else if (warp == 1) {
      // ---------------- products ----------------
      constexpr uint32_t kFmt = (1u << 4) | (AttnType<T>::fmt << 7) | (AttnType<T>::fmt << 10) | ((uint32_t)(kAttnTile >> 4) << 24);
      constexpr uint32_t kIdescS = kFmt | ((uint32_t)(kAttnTile >> 3) << 17);
      constexpr uint32_t kIdescO = kFmt | (1u << 16) | ((uint32_t)(D >> 3) << 17);   // B with its N dimension contiguous
      int stage = 0;
      uint32_t phase = 0;
      bool ok = has(0, false) && wait_warp(q_bar, 0);
      uint32_t p_phase = 0, clean_phase = 0;   // a bit per stream, a bit per stage
      const int streams = TWO ? (two ? 2 : 1) : 1;   // that use each tile
      const uint32_t tm = uniform(tmem_base), base = uniform(smem_base);
      // S_st = Q (of stream st if TWO) K^T of the tile in stage `at`; `last`: nothing else reads the stage
      auto qk = [&](int st, int at, bool last) {
        const uint32_t u = uniform((uint32_t)st), ring = uniform((uint32_t)at);
        const uint32_t da = desc_low(base + (TWO ? u * Cfg::kTileBytes : 0u), 16);   // K contiguous: the leading offset is unused
        const uint32_t db = desc_low(base + Cfg::kRing + ring * Cfg::kTileBytes, 16);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < D / kUmmaK; ++k)
            umma_ss(tm + u * kAttnTile, da, db, (uint32_t)((k / 4) * (kAttnTile * 128 / 16) + (k % 4) * 2), kIdescS, (uint32_t)(k != 0));
          umma_commit(s_bar(0) + 8u * u);
          if (last) umma_commit(empty_bar(0) + 8u * ring);
        }
        __syncwarp();
      };
      for (int ik = 0; ik < kLead && ok && has(ik, false); ++ik) {
        ok = wait_warp(full_bar(stage), phase);
        if (!ok) break;
        tc_fence_after();
        for (int u = 0; u < streams; ++u) qk(TWO ? u : ik & 1, stage, u + 1 == streams);
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
      for (int i = 0; ok && has(i, false); ++i) {
        uint32_t f;
        tile_of(i, f);
        ok = wait_warp(full_bar(stage), phase);
        if (!PACKED && ok && (f & kTileDead)) {
          ok = wait_warp(clean_bar(stage), (clean_phase >> stage) & 1u);
          clean_phase ^= 1u << stage;
        }
        const bool more = ok && has(i + kLead, false);
        if (!ok) break;
        const int vstage = stage;
        const int kstage = stage + 1 == kStages ? 0 : stage + 1;
        const uint32_t kphase = stage + 1 == kStages ? phase ^ 1u : phase;
        for (int w = 0; w < streams && ok; ++w) {
          const int st = TWO ? w : i & 1;
          ok = wait_warp(p_bar(st), (p_phase >> st) & 1u);
          if (!ok) break;
          p_phase ^= 1u << st;
          tc_fence_after();
          {
            const uint32_t u = uniform((uint32_t)st), ring = uniform((uint32_t)vstage), more_o = uniform((uint32_t)(TWO ? i > 0 : i > 1));
            // channels contiguous: blocks of 64 channels kAttnTile * 128 bytes apart, 16 slots are two groups of eight rows
            const uint32_t db = desc_low(base + Cfg::kRing + ring * Cfg::kTileBytes, kAttnTile * 128);
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < kAttnTile / kUmmaK; ++k)
                umma_ts(tm + kO + u * D, tm + u * kAttnTile, db, 8u * k, (uint32_t)(k * (kUmmaK * 128 / 16)), kIdescO, k == 0 ? more_o : 1u);
              umma_commit(o_bar(0) + 8u * u);
              if (w + 1 == streams) umma_commit(empty_bar(0) + 8u * ring);
            }
            __syncwarp();
          }
          if (more) {
            if (w == 0) {
              ok = wait_warp(full_bar(kstage), kphase);
              if (!ok) break;
              tc_fence_after();
            }
            qk(st, kstage, w + 1 == streams);
          }
        }
        if (!ok) break;
        for (int u = 0; u < (more ? 2 : 1); ++u)
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
    } else {
      // ---------------- the list of visible tiles behind the cached part; then, along the ring, the intervals of tiles that
      // need them, and zeros over the values of slots that hold nothing ----------------
      bool ok = wait_warp(flag_bar, 0);
      int n = 0;
      for (int base = t0; ok && base < t_far; base += 32) {
        const uint32_t f = base + lane < t_far ? list[base - t0 + lane] : 0u;
        const uint32_t some = __ballot_sync(0xFFFFFFFFu, f != 0u);
        __syncwarp();
        if (f) list[n + __popc(some & ((1u << lane) - 1u))] = f | ((uint32_t)(base - t0 + lane) << 16);
        n += __popc(some);
      }
      if (lane == 0) *listed = n;
      __syncwarp();
      if (ok && lane == 0) mbar_arrive(list_bar);
      int stage = 0, masked = 0;
      uint32_t phase = 0;
      auto intervals = [&](int i) {
        uint32_t f;
        const int t = tile_of(i, f);
        if (!(f & kTileMasked)) return;
        const int b = masked % kMaskRing;
        ok = wait_warp(m_empty(b), ((uint32_t)(masked / kMaskRing) & 1u) ^ 1u);
        if (!ok) return;
        int2 v[kAttnTile / 32];
        tile_intervals(a, s, t, lane, v);
#pragma unroll
        for (int e = 0; e < kAttnTile / 32; ++e) {
          mask[b * kAttnTile + e * 32 + lane] = v[e];
          if (WINDOW) places[b * kAttnTile + e * 32 + lane] = slot_place(a, s, t * kAttnTile + e * 32 + lane);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(m_full(b));
        ++masked;
      };
      auto release = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(empty_bar(stage));
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      };
      if constexpr (PACKED) {                        // the ring is other warps' business
        for (int i = 0; ok && has(i, false); ++i) intervals(i);
      } else {
        int ik = 0;
        auto pass_key = [&]() {
          intervals(ik++);
          ok = ok && wait_warp(full_bar(stage), phase);
          if (ok) release();
        };
        while (ik < kLead && ok && has(ik, false)) pass_key();
        for (int i = 0; ok && has(i, false); ++i) {
          ok = wait_warp(full_bar(stage), phase);
          if (!ok) break;
          uint32_t f;
          const int t = tile_of(i, f);
          if (f & kTileDead) {
            uint8_t* v = smem + Cfg::kRing + stage * Cfg::kTileBytes;
            int2 iv[kAttnTile / 32];
            tile_intervals(a, s, t, lane, iv);
#pragma unroll 1
            for (int e = 0; e < kAttnTile / 32; ++e) {
              if (iv[e].y != 0) continue;
              uint8_t* at = v + (e * 32 + lane) * 128;
              for (int c = 0; c < D / 64; ++c)
#pragma unroll
                for (int x = 0; x < 8; ++x) *reinterpret_cast<uint4*>(at + c * (kAttnTile * 128) + x * 16) = make_uint4(0, 0, 0, 0);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(clean_bar(stage));
          }
          release();
          if (has(ik, false)) pass_key();
        }
      }
    }
  } else if (PACKED && warp >= 4 + 4 * kStreams) {
    // ---------------- raw tiles are expanded, in the rings' order ----------------
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if constexpr (PACKED) {
      const int first = 16 * (warp - 4 - 4 * kStreams);     // of this warp's slots in a tile
      int pos = 0;
      bool ok = true;
      auto expand = [&](int i) {
        const int from = pos % Cfg::kRawStages, to = pos % kStages;
        ok = wait_warp(raw_full(from), (uint32_t)(pos / Cfg::kRawStages) & 1u) && wait_warp(empty_bar(to), ((uint32_t)(pos / kStages) & 1u) ^ 1u);
        if (!ok) return;
        uint32_t f, dead = 0;
        const int t = tile_of(i, f);
        if (f & kTileDead) {
          constexpr int kRows = 32 / (D / 32);
          for (int it = 0; it < 16 / kRows; ++it)
            dead |= (slot_interval(a, s, t * kAttnTile + first + it * kRows + lane / (D / 32)).y == 0 ? 1u : 0u) << it;
        }
        expand_rows<T, D>(smem_base + Cfg::kRaw + (uint32_t)(from * Cfg::kRawBytes), smem_base + Cfg::kRing + (uint32_t)(to * Cfg::kTileBytes), first, lane, dead);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(full_bar(to));
          mbar_arrive(raw_empty(from));
        }
        ++pos;
      };
      for (int i = 0; i < kLead && ok && has(i, false); ++i) expand(i);
      for (int i = 0; ok && has(i, false); ++i) {
        expand(i);
        if (ok && has(i + kLead, false)) expand(i + kLead);
      }
    }
  } else {
    // ---------------- rows ----------------
    if (PACKED) asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    else if (MODE == kRowsBrief) asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    {
      const int qmin = range[0], qmax = range[1];    // all rows padding: qmax is -1 and no tile is visible
      for (int t = t0 + warp - 4; t < t_far; t += 4 * kStreams) {
        const uint32_t f = qmax < 0 ? 0u : tile_flags<WINDOW>(a, s, tile_at(t), qmin, qmax, lane, &win);
        if (lane == 0) list[t - t0] = f;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(flag_bar);
    }
    const int st = (warp - 4) >> 2;                    // stream
    const int quarter = warp & 3;
    const int row = quarter * 32 + lane;
    const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
    const uint32_t t_s = tmem_base + lane_base + (uint32_t)st * kAttnTile, t_o = tmem_base + lane_base + kO + (uint32_t)st * D;
    constexpr int kCols = HALF ? 64 : 128;                           // of a tile's slots that this thread takes
    const int own = HALF ? row & 63 : row, col0 = HALF ? row & 64 : 0;
    const int tok = (TWO ? st * plan.tpt : 0) + own / a.G;           // within the CTA's tokens
    const bool in = own < plan.tpt * a.G && tok < ntok;
    const bool warp_in = __any_sync(0xFFFFFFFFu, in);
    const int64_t token = (int64_t)s.first + tok0 + tok;
    const int head = hk * a.G + own % a.G;
    const int mine = !in ? -1 : a.pre ? a.pre[token] : tok0 + tok;
    const int near = WINDOW && in ? s.ctx + draft_depth(a, s, tok0 + tok) - a.window + 1 : 0;   // first place within this row's window
    const float c = a.scale * 1.4426950408889634f;
    float m = -INFINITY, l = 0.f;
    int done = 0;                                      // tiles of this stream so far
    int masked = 0;                                    // tiles with intervals so far, of both streams
    bool ok = true;
    const bool active = TWO ? (st == 0 || two) : true;
    for (int i = 0; ok && active && has(i, false); ++i) {
      uint32_t f;
      tile_of(i, f);
      if (!TWO && (i & 1) != st) {
        masked += (f & kTileMasked) ? 1 : 0;
        continue;
      }
      ok = wait_warp(s_bar(st), (uint32_t)done & 1u);
      if (ok && (f & kTileMasked)) ok = wait_warp(m_full(masked % kMaskRing), (uint32_t)(masked / kMaskRing) & 1u);
      if (!ok) break;
      tc_fence_after();
      if (warp_in) {
        uint32_t v[kCols];
#pragma unroll
        for (int j = 0; j < kCols / 32; ++j) ATTS_TMEM_LD_32(t_s + (uint32_t)col0 + 32u * j, (&v[32 * j]));
        tmem_ld_wait();
        if ((f & 0xFFu) != kTileFull) {
          const int2* mk = mask + (masked % kMaskRing) * kAttnTile + col0;
#pragma unroll
          for (int g = 0; g < kCols / 32; ++g) {
            const uint32_t kind = (f >> (2 * g + col0 / 16)) & 3u;
            if (kind == 0u) {
#pragma unroll
              for (int j = 32 * g; j < 32 * g + 32; ++j) v[j] = 0xFF800000u;
            } else if (kind == 1u) {
#pragma unroll
              for (int j = 32 * g; j < 32 * g + 32; j += 2) {
                const int4 w = *reinterpret_cast<const int4*>(mk + j);
                bool out0 = (unsigned)(mine - w.x) >= (unsigned)w.y, out1 = (unsigned)(mine - w.z) >= (unsigned)w.w;
                if (WINDOW) {
                  const int2 x = *reinterpret_cast<const int2*>(places + (masked % kMaskRing) * kAttnTile + col0 + j);
                  out0 |= x.x < near && x.x >= a.sinks;
                  out1 |= x.y < near && x.y >= a.sinks;
                }
                if (out0) v[j] = 0xFF800000u;
                if (out1) v[j + 1] = 0xFF800000u;
              }
            }
          }
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < kCols; j += 8)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx[e] = max3(mx[e], __uint_as_float(v[j + e]), __uint_as_float(v[j + 4 + e]));
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        // the reference moves when a row's maximum passes it by more than 8 (base 2), and for the first visible slot
        float keep = 1.f;
        if ((top - m) * c > 8.f) {
          keep = ex2_approx((m - top) * c);     // 0 for m = -inf
          m = top;
          l *= keep;
        }
        if (done > 0 && __any_sync(0xFFFFFFFFu, keep != 1.f)) {
          ok = wait_warp(o_bar(st), (uint32_t)(done - 1) & 1u);
          if (!ok) break;
          tc_fence_after();
          rescale_o<D>(t_o, keep);
        }
        const float off = (m == -INFINITY ? 0.f : -m * c) + AttnType<T>::shift;
        const uint64_t c2 = pair2(c, c), off2 = pair2(off, off);
        uint64_t sum2[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < kCols; j += 32) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const uint64_t x = fma2(pair2(__uint_as_float(v[j + e]), __uint_as_float(v[j + e + 1])), c2, off2);
            const float p0 = ex2_approx(low2(x)), p1 = ex2_approx(high2(x));
            sum2[(e >> 1) & 1] = add2(sum2[(e >> 1) & 1], pair2(p0, p1));
            w[e / 2] = Pack<T>::pack(p0, p1);
          }
          ATTS_TMEM_ST_16(t_s + (uint32_t)((col0 + j) / 2), w);
        }
        if (HALF) {                                    // the other half's slots are not this row's
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) w[e] = 0u;
          ATTS_TMEM_ST_16(t_s + (uint32_t)((64 - col0) / 2), w);
          ATTS_TMEM_ST_16(t_s + (uint32_t)((64 - col0) / 2 + 16), w);
        }
        const uint64_t sum = add2(sum2[0], sum2[1]);
        l += low2(sum) + high2(sum);
        tmem_st_wait();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(p_bar(st));
        if (f & kTileMasked) mbar_arrive(m_empty(masked % kMaskRing));
      }
      masked += (f & kTileMasked) ? 1 : 0;
      ++done;
    }
    if (active && ok && done > 0) ok = wait_warp(o_bar(st), (uint32_t)(done - 1) & 1u);
    tc_fence_after();
    // ---- join of the two streams (one row tile): the odd one hands its sums over through the ring, which is free once
    // every product has finished: this stream's last one has; the other's last but one has, and its last is waited for ----
    float2 other = make_float2(-INFINITY, 0.f);
    const bool joined = !TWO && !HALF && ntile > 1;
    float* pass = reinterpret_cast<float*>(smem + Cfg::kRing);
    if (joined && st == 1) {
      if (ok) ok = wait_warp(o_bar(0), (uint32_t)((ntile + 1) / 2 - 1) & 1u);
      if (ok && warp_in) {
        stats[row] = make_float2(m, l);
#pragma unroll 1
        for (int j = 0; j < D; j += 32) {   // run once: short code costs less to fetch than unrolled code saves
          uint32_t v[32];
          ATTS_TMEM_LD_32(t_o + (uint32_t)j, v);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; i += 4) *reinterpret_cast<uint4*>(pass + row * (D + 4) + j + i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(join_bar);
    }
    if (joined && st == 0 && ok) {
      ok = wait_warp(join_bar, 0);
      if (ok && warp_in) other = stats[row];
    }
    // kRowsHalf: three others (1 the lower half of this stream, 2 and 3 the halves of the odd one) hand theirs over, none of which
    // may have seen a tile.
    const int part = HALF ? 2 * st + (col0 >> 6) : 0;
    float2 others[3] = {other, other, other};
    if (HALF && part > 0) {
      const int theirs = st == 0 ? ntile / 2 : (ntile + 1) / 2;      // the other stream's tiles
      if (ok && theirs > 0) ok = wait_warp(o_bar(1 - st), (uint32_t)(theirs - 1) & 1u);
      if (ok && warp_in) {
        stats[(part - 1) * 64 + own] = done > 0 ? make_float2(m, l) : other;
        if (done > 0)
#pragma unroll 1
          for (int j = 0; j < D; j += 32) {
            uint32_t v[32];
            ATTS_TMEM_LD_32(t_o + (uint32_t)j, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              *reinterpret_cast<uint4*>(pass + ((part - 1) * 64 + own) * (D + 4) + j + i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
          }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(join_bar);
    }
    if (HALF && part == 0 && ok) {
      ok = wait_warp(join_bar, 0);
      if (ok && warp_in)
#pragma unroll
        for (int i = 0; i < 3; ++i) others[i] = stats[i * 64 + own];
    }
    if (ok && active && warp_in && (TWO || st == 0) && part == 0) {
      // o = (O_0 f0 + O_1 f1) / (l_0 f0 + l_1 f1), fk = 2^(c (m_k - max))
      float mm = fmaxf(m, other.x);
      if (HALF) mm = fmaxf(m, max3(others[0].x, others[1].x, others[2].x));
      const float f0 = m == -INFINITY ? 0.f : ex2_approx((m - mm) * c), f1 = other.x == -INFINITY ? 0.f : ex2_approx((other.x - mm) * c);
      float sum = l * f0 + other.y * f1, fh[3] = {0.f, 0.f, 0.f};
      if (HALF)
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          fh[i] = others[i].x == -INFINITY ? 0.f : ex2_approx((others[i].x - mm) * c);
          sum += others[i].y * fh[i];
        }
      // A NaN among a row's scores is not empty: it reaches out and lse.  Nor is a score that the scale takes beyond fp32, which makes
      // every exponential 0: out and lse become the NaN that +inf makes of them.
      const bool empty = mine < 0 || (sum == 0.f && mm == -INFINITY);
      const float g0 = empty ? 0.f : f0 / sum, g1 = empty ? 0.f : f1 / sum;
      if (HALF)
#pragma unroll
        for (int i = 0; i < 3; ++i) fh[i] = empty ? 0.f : fh[i] / sum;
      const float lse2 = empty ? -INFINITY : sum == 0.f ? NAN : mm * c - AttnType<T>::shift + log2f(sum);
      const int parts = WINDOW ? plan.chunks : (ntiles + plan.chunk - 1) / plan.chunk;
      const int64_t r = token * a.Hq + head;
      if (in) {
        if (parts > 1) plan.part_lse[r * plan.chunks + chunk] = lse2;
        else if (a.lse) a.lse[r] = lse2 * 0.6931471805599453f;
      }
      // Rows go out through the queries' shared memory, D * 2 bytes of each at a time (whole rows in the outputs' type, halves of
      // the fp32 sums of a chunk), so that a store covers whole rows: written by its own thread, a row's pieces would
      // cost one access to L1 each (4,000 cycles of 74,000 in a tile of 12).
      constexpr int kLanes = D / 8, kRowBytes = D * 2;               // lanes that share a row
      uint8_t* buf = smem + (TWO ? st * Cfg::kTileBytes : 0) + quarter * 32 * kRowBytes;
      char* dst = parts > 1 ? reinterpret_cast<char*>(plan.part_o + (r * plan.chunks + chunk) * D)
                            : a.out + 2 * (token * a.o_ts + (int64_t)head * a.o_hs);
      const uint32_t rows = __ballot_sync(0xFFFFFFFFu, in);
      const int sub = lane % kLanes;
      auto rows_out = [&](int offset) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 32; i += 32 / kLanes) {
          const int from = i + lane / kLanes;
          const uint64_t to = __shfl_sync(0xFFFFFFFFu, reinterpret_cast<uint64_t>(dst), from);
          if ((rows >> from) & 1u)
            *reinterpret_cast<uint4*>(to + offset + sub * 16) = *reinterpret_cast<const uint4*>(buf + from * kRowBytes + ((sub ^ (from & 7)) * 16));
        }
        __syncwarp();
      };
      uint8_t* mine_at = buf + lane * kRowBytes;
#pragma unroll 1
      for (int j = 0; j < D; j += 32) {
        uint32_t v[32];
        if (done > 0) {
          ATTS_TMEM_LD_32(t_o + (uint32_t)j, v);
          tmem_ld_wait();
        }
        float o[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = empty || done == 0 ? 0.f : __uint_as_float(v[e]) * g0;
        if (joined && !empty) {
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const float4 x = *reinterpret_cast<const float4*>(pass + row * (D + 4) + j + e);
            o[e] += x.x * g1; o[e + 1] += x.y * g1; o[e + 2] += x.z * g1; o[e + 3] += x.w * g1;
          }
        }
        if (HALF && !empty) {
#pragma unroll 1
          for (int i = 0; i < 3; ++i) {
            const float g = i == 0 ? fh[0] : i == 1 ? fh[1] : fh[2];
            if (g == 0.f) continue;                    // (nothing was handed over where no tile was seen)
            const float* from = pass + (i * 64 + own) * (D + 4) + j;
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const float4 x = *reinterpret_cast<const float4*>(from + e);
              o[e] += x.x * g; o[e + 1] += x.y * g; o[e + 2] += x.z * g; o[e + 3] += x.w * g;
            }
          }
        }
        if (parts > 1) {
          const int at = j % (D / 2);
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *reinterpret_cast<float4*>(mine_at + ((((at + e) / 4) ^ (lane & 7)) * 16)) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          if (at + 32 == D / 2) rows_out((j / (D / 2)) * kRowBytes);
        } else {
#pragma unroll
          for (int e = 0; e < 32; e += 8)
            *reinterpret_cast<uint4*>(mine_at + ((((j + e) / 8) ^ (lane & 7)) * 16)) =
                make_uint4(Pack<T>::pack(o[e], o[e + 1]), Pack<T>::pack(o[e + 2], o[e + 3]), Pack<T>::pack(o[e + 4], o[e + 5]), Pack<T>::pack(o[e + 6], o[e + 7]));
        }
      }
      if (parts <= 1) rows_out(0);
    }
  }

  // ---------------- teardown ----------------
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // A wait expired.  Record it, give copies and products still in flight time to land, then free tensor memory.
    if (threadIdx.x == 0) atomicOr(dev_status, 2u);
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)Cfg::kTmem) : "memory");
  }
}

// Joins the chunks of a row: o = sum_c o_c 2^(lse_c - max) / sum_c 2^(lse_c - max), one warp per row, chunks in order.
template <typename T, int D>
__global__ void __launch_bounds__(256)
attention_join_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ AttnPlan plan) {
  pdl_wait();
  const int seq = blockIdx.y;
  SeqView s;
  unsigned none;
  if (!seq_view(a.cu, a.ctx, seq, a.M, a.max_tokens, a.max_len, s, &none, false)) return;
  const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (r >= (int64_t)s.n * a.Hq) return;
  const int ntiles = (s.len + kAttnTile - 1) / kAttnTile;
  const int parts = (ntiles + plan.chunk - 1) / plan.chunk;
  if (parts <= 1) return;
  const int64_t row = (int64_t)s.first * a.Hq + r;
  const float* lse = plan.part_lse + row * plan.chunks;
  float top = -INFINITY;
  for (int i = lane; i < parts; i += 32) top = fmaxf(top, lse[i]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  constexpr int E = D / 32;
  float o[E], sum = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int i = 0; i < parts; ++i) {
    const float w = lse[i] == -INFINITY ? 0.f : ex2_approx(lse[i] - top);
    if (w == 0.f) continue;
    sum += w;
    const float* p = plan.part_o + (row * plan.chunks + i) * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += w * p[e];
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;    // (NaN stays NaN)
  const int64_t token = row / a.Hq;
  const int head = (int)(row - token * a.Hq);
  uint32_t* out = reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(a.out) + token * a.o_ts + (int64_t)head * a.o_hs + lane * E);
#pragma unroll
  for (int e = 0; e < E; e += 2) out[e / 2] = Pack<T>::pack(o[e] * inv, o[e + 1] * inv);
  if (a.lse && lane == 0) a.lse[row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

// The same where every chunk of every row has written its part (a part with lse = -inf no sums): windowed and packed forms.  WARPS
// a row, each with its share of the parts and four of them on their way.  Many parts take four: one warp that goes over 33 of them one
// by one takes 11 us.  A few take one: with four, 15,000 rows of two parts are four times the blocks, 25 us instead of 5.
constexpr int kJoinThreads = 256, kJoinFewParts = 8;
template <typename T, int D, int WARPS>
__global__ void __launch_bounds__(kJoinThreads)
attention_parts_join_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ AttnPlan plan) {
  constexpr int kRows = kJoinThreads / 32 / WARPS;
  __shared__ float sums[kRows][WARPS][D];
  pdl_wait();
  SeqView s;
  unsigned none;
  if (!seq_view(a.cu, a.ctx, blockIdx.y, a.M, a.max_tokens, a.max_len, s, &none, false)) return;
  const int which = threadIdx.x / (32 * WARPS), warp = threadIdx.x / 32 % WARPS, lane = threadIdx.x & 31;
  const int64_t r = (int64_t)blockIdx.x * kRows + which, row = (int64_t)s.first * a.Hq + r;
  if (r - which >= (int64_t)s.n * a.Hq) return;                       // none of the block's rows exists
  const bool in = r < (int64_t)s.n * a.Hq;
  constexpr int E = D / 32;
  float o[E] = {}, top = -INFINITY, sum = 0.f;
  if (in) {
    const float* lse = plan.part_lse + row * plan.chunks;
    for (int i = lane; i < plan.chunks; i += 32) top = fmaxf(top, lse[i]);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
    for (int i = lane; i < plan.chunks; i += 32) sum += lse[i] == -INFINITY ? 0.f : ex2_approx(lse[i] - top);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
#pragma unroll 4
    for (int i = warp; i < plan.chunks; i += WARPS) {
      const float w = lse[i] == -INFINITY ? 0.f : ex2_approx(lse[i] - top);
      const float* p = plan.part_o + (row * plan.chunks + i) * D + lane * E;
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = p[e];
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] += w == 0.f ? 0.f : w * v[e];   // (an empty part's sums are not there)
    }
#pragma unroll
    for (int e = 0; e < E; ++e) sums[which][warp][lane * E + e] = o[e];
  }
  __syncthreads();
  if (!in || warp != 0) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;    // (NaN stays NaN)
  const int64_t token = row / a.Hq;
  const int head = (int)(row - token * a.Hq);
  uint32_t* out = reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(a.out) + token * a.o_ts + (int64_t)head * a.o_hs + lane * E);
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    float x = 0.f, y = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      x += sums[which][w][lane * E + e];
      y += sums[which][w][lane * E + e + 1];
    }
    out[e / 2] = Pack<T>::pack(x * inv, y * inv);
  }
  if (a.lse && lane == 0) a.lse[row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

struct WeightArgs {
  AttnArgs q;              // out and lse unused
  const float* lse;
  const float* win;
  float* wout;
  int64_t wcols;
  int tpt;                 // tokens per row tile
  int cluster, span;       // CTAs that share a slot tile's row tiles; slot tiles of a CTA that has one row tile
  long long wait_limit;
  int withhold_loads;
};

// ------------------------------------------------------------------------------------------------------------------
// Attention weight per slot.  The product of one slot tile (128 slots of a key head) and one row tile of queries is
//   S^T = K Q^T (tcgen05, fp32 in tensor memory), a thread per slot, and each thread adds 2^(c s - lse2) over the columns
// of its own row: no sum crosses threads, so the order is fixed and nothing is stored but one number per slot.  Products
// alternate between two groups of four warps with an accumulator each, and two CTAs share an SM: the exponentials (one per
// pair, 16 a clock and SM) are what the time goes to first: 8 drafts of 500 over 1013 slots, 40 / 8 heads, have 2.0e8 visible pairs,
// 43 us at that rate, and take 130 us (0.33).  The rest: 14,096 products of which the last of 296 places ends at 63 where an even
// deal ends at 48, and the products themselves (about 1,900 cycles an SM each, where their exponentials take 1,000).  8 sequences of
// one token over 2000 slots: 8 us of kernel for 29 MB.  The exponential is the hardware's approximation (2 ulp) of an argument
// made by one fp32 multiply-add: a weight is off by 5e-7 of itself where an fp32 exponential makes 1e-7.
//
// One operand stays, the other streams.  MANY = false (one row tile covers every sequence's drafts): the queries stay and a CTA
// goes over `span` slot tiles.  MANY = true: a slot tile stays and the row tiles stream.  Every row sees the cached slots,
// so their tiles are dealt to the CTAs of a cluster, whose first one adds up the sums in order through the cluster's shared
// memory; behind the cached part a tree's tile is seen by its own branch only and a CTA takes it alone (a chain's tiles
// are seen by all later rows and are dealt like cached ones).
// ------------------------------------------------------------------------------------------------------------------
constexpr int kWeightThreads = 320;     // warp 0 loads, warp 1 products, 2-5 and 6-9 slots
constexpr int kWeightItems = 1024;      // products of a CTA whose visibility is looked up ahead; further ones are all made
constexpr int kWeightMaxCluster = 4;     // larger ones leave SMs idle while they wait for room together

template <int D>
struct WeightCfg {
  static constexpr int kTileBytes = kAttnTile * D * 2;
  static constexpr int kRing = kTileBytes;                         // the operand that stays, then two stages
  static constexpr int kCols = kRing + 2 * kTileBytes;             // [2 groups][2][128] -lse2, then places
  static constexpr int kFlags = kCols + 2 * 4 * kAttnTile * 4;     // [items] bytes
  static constexpr int kList = kFlags + kWeightItems;              // [items] uint16
  static constexpr int kSums = kList + 2 * kWeightItems;           // [cluster][128] sums, [128] of the odd group
  static constexpr int kBars = kSums + (kWeightMaxCluster + 1) * kAttnTile * 4;
  // At most two CTAs to an SM, whatever their registers: each holds 256 of its 512 columns of tensor memory until the last barrier
  // of its cluster, so a third one would wait for columns while the CTAs that hold them may wait for it.  (With head_dim 64 the
  // buffers alone would let a third one in.)
  static constexpr int kNeeded = kBars + 128 + 1024;
  static constexpr int kSmemBytes = kNeeded > 77824 ? kNeeded : 77824;
  static_assert(2 * (kSmemBytes + 1024) <= 233472 && 3 * (kSmemBytes + 1024) > 233472, "two CTAs share an SM, three do not");
};

// Sum over 16 columns of an accumulator: 2^(c s - lse2), pairs of columns side by side.  (With 32 at a time the registers of two
// blocks, their columns' numbers and the sums do not fit, and the exponentials wait for shared memory.)
template <bool MASKED>
__device__ __forceinline__ void weight_columns(uint32_t (&v)[16], const float* nlse, const int* place, int2 iv, uint64_t c2, uint64_t (&sum)[2]) {
  if (MASKED) {
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int4 w = *reinterpret_cast<const int4*>(place + e);
      if ((unsigned)(w.x - iv.x) >= (unsigned)iv.y) v[e] = 0xFF800000u;
      if ((unsigned)(w.y - iv.x) >= (unsigned)iv.y) v[e + 1] = 0xFF800000u;
      if ((unsigned)(w.z - iv.x) >= (unsigned)iv.y) v[e + 2] = 0xFF800000u;
      if ((unsigned)(w.w - iv.x) >= (unsigned)iv.y) v[e + 3] = 0xFF800000u;
    }
  }
#pragma unroll
  for (int e = 0; e < 16; e += 4) {
    const float4 w = *reinterpret_cast<const float4*>(nlse + e);
    const uint64_t x = fma2(pair2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), c2, pair2(w.x, w.y));
    const uint64_t y = fma2(pair2(__uint_as_float(v[e + 2]), __uint_as_float(v[e + 3])), c2, pair2(w.z, w.w));
    sum[0] = add2(sum[0], pair2(ex2_approx(low2(x)), ex2_approx(high2(x))));
    sum[1] = add2(sum[1], pair2(ex2_approx(low2(y)), ex2_approx(high2(y))));
  }
}

template <typename T, int D, bool MANY>
__global__ void __launch_bounds__(kWeightThreads, 2)
cache_weights_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ WeightArgs a, unsigned* __restrict__ dev_status) {
  using Cfg = WeightCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  // Heads run side by side (a slot's heads are neighbours in memory), and every head's cached tiles, which all rows see, come
  // before the tiles behind them.
  const int ranks_all = MANY ? a.cluster : 1;
  const int in_cluster = blockIdx.x % ranks_all, group = blockIdx.x / ranks_all;
  const int hk = group % a.q.cache.heads, unit = group / a.q.cache.heads, seq = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  SeqView s;
  pdl_wait();
  const bool ok_seq = seq_view(a.q.cu, a.q.ctx, seq, a.q.M, a.q.max_tokens, a.q.max_len, s, dev_status,
                               threadIdx.x == 0 && blockIdx.x == 0);
  const int tpt = a.tpt, nq = (s.n + tpt - 1) / tpt;
  // this CTA's slot tiles [tile0, tile1), and for MANY its row tiles q0, q0 + step, ...
  int ranks = 1, rank = 0, tile0, tile1, q0 = 0, step = 1;
  if (MANY) {
    const int dealt = !ok_seq ? 0 : a.q.pre ? min((s.ctx + kAttnTile - 1) / kAttnTile, (s.len + kAttnTile - 1) / kAttnTile) : (s.len + kAttnTile - 1) / kAttnTile;
    if (unit < dealt) {      // the same for every CTA of a cluster
      ranks = a.cluster;
      rank = q0 = in_cluster;
      step = a.cluster;
      tile0 = unit;
    } else {
      tile0 = dealt + (unit - dealt) * a.cluster + in_cluster;
    }
    tile1 = tile0 + 1;
  } else {
    tile0 = unit * a.span;
    tile1 = min(tile0 + a.span, (a.q.max_len + kAttnTile - 1) / kAttnTile);
  }
  float* wout = a.wout + ((int64_t)seq * a.q.cache.heads + hk) * a.wcols;
  const float* win = a.win ? a.win + ((int64_t)seq * a.q.cache.heads + hk) * a.wcols : nullptr;
  const int len = ok_seq ? s.len : 0;
  // (a sequence that does not fit is left out: what it gathered before stays)
  auto old_weight = [&](int slot) { return win && (slot < len || !ok_seq) ? win[slot] : 0.f; };
  if ((int64_t)tile0 * kAttnTile >= a.q.max_len) return;       // (a cluster behind the dealt tiles reaches beyond the row)
  if (tile0 * kAttnTile >= len || s.n == 0) {
    for (int slot = tile0 * kAttnTile + threadIdx.x; slot < min(tile1 * kAttnTile, a.q.max_len); slot += kWeightThreads) wout[slot] = old_weight(slot);
    return;
  }
  const int items = MANY ? (nq > q0 ? (nq - q0 + step - 1) / step : 0) : min(tile1, (len + kAttnTile - 1) / kAttnTile) - tile0;
  const int ncols = (tpt * a.q.G + 31) & ~31;
  auto slot_tile = [&](int i) { return MANY ? tile0 : tile0 + i; };
  auto row_tile = [&](int i) { return MANY ? q0 + i * step : 0; };

  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  float* col_lse = reinterpret_cast<float*>(smem + Cfg::kCols);
  int* col_place = reinterpret_cast<int*>(smem + Cfg::kCols + 4 * kAttnTile * 4);
  uint32_t* flags = reinterpret_cast<uint32_t*>(smem + Cfg::kFlags);
  volatile uint16_t* list = reinterpret_cast<volatile uint16_t*>(smem + Cfg::kList);
  float* sums = reinterpret_cast<float*>(smem + Cfg::kSums);
  const uint32_t bar0 = smem_base + Cfg::kBars;
  const uint32_t stay_bar = bar0;
  auto r_full = [&](int i) { return bar0 + 8u + 8u * (uint32_t)i; };
  auto r_empty = [&](int i) { return bar0 + 24u + 8u * (uint32_t)i; };
  auto s_full = [&](int i) { return bar0 + 40u + 8u * (uint32_t)i; };
  auto s_empty = [&](int i) { return bar0 + 56u + 8u * (uint32_t)i; };
  auto c_bar = [&](int i) { return bar0 + 72u + 8u * (uint32_t)i; };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + Cfg::kBars + 88);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  volatile int* listed = reinterpret_cast<volatile int*>(tmem_slot + 2);

  for (int i = threadIdx.x; i < kWeightItems / 4; i += kWeightThreads) flags[i] = 0;
  if (threadIdx.x == 0) {
    prefetch_tmap(&map_q);
    prefetch_tmap(&map_k);
    mbar_init(stay_bar, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(r_full(i), 1);
      mbar_init(r_empty(i), 1);
      mbar_init(s_full(i), 1);
      mbar_init(s_empty(i), 4);
      mbar_init(c_bar(i), 4);
    }
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(256u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // rows of a query tile that no token fills, up to the columns used, are zero (a box never writes them)
  {
    const int used = tpt * a.q.G, rows = ncols - used, tiles = MANY ? 2 : 1;
    uint8_t* q = smem + (MANY ? Cfg::kRing : 0);
    for (int r = warp; r < rows * tiles * (D / 64); r += kWeightThreads / 32) {
      const int blk = r / rows;
      if (lane < 8) *reinterpret_cast<uint4*>(q + blk * (kAttnTile * 128) + (used + r - blk * rows) * 128 + lane * 16) = make_uint4(0, 0, 0, 0);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  // Which products have anything visible: bit 0 of an item's byte, some row may see some slot; bit 1, some pair is not visible.
  // A slot tile's intervals are taken together: nobody outside of [lo, hi) sees anything, everybody in [in_lo, in_hi) sees all.
  const int known = min(items, kWeightItems);
  __syncthreads();
  {
    auto bounds = [&](int tile, int& lo, int& hi, int& in_lo, int& in_hi) {
      int2 v[4];
      tile_intervals(a.q, s, tile, lane, v);
      lo = in_hi = 0x7FFFFFFF;
      hi = in_lo = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int end = (int)min((unsigned)v[e].x + (unsigned)v[e].y, 0x7FFFFFFFu);
        const bool none = v[e].y == 0;
        if (!none) {
          lo = min(lo, v[e].x);
          hi = max(hi, end);
          in_lo = max(in_lo, v[e].x);
          in_hi = min(in_hi, end);
        } else if (tile * kAttnTile + e * 32 + lane < s.len) {
          in_hi = -1;            // padding: nobody sees all
        }
      }
      lo = __reduce_min_sync(0xFFFFFFFFu, lo);
      hi = __reduce_max_sync(0xFFFFFFFFu, hi);
      in_lo = __reduce_max_sync(0xFFFFFFFFu, in_lo);
      in_hi = __reduce_min_sync(0xFFFFFFFFu, in_hi);
    };
    int lo, hi, in_lo, in_hi;
    if (MANY) {
      bounds(tile0, lo, hi, in_lo, in_hi);
      for (int t = threadIdx.x; t < s.n; t += kWeightThreads) {
        const int tile = t / tpt, i = (tile - q0) / step;
        if (tile < q0 || tile != q0 + i * step || i >= known) continue;
        const int p = a.q.pre ? a.q.pre[s.first + t] : t;
        uint32_t f = p >= lo && p < hi ? 1u : 0u;
        if (!(p >= in_lo && p < in_hi) || (tile + 1) * tpt > s.n) f |= 2u;
        if (f) atomicOr(&flags[i >> 2], f << (8 * (i & 3)));
      }
    } else {
      for (int i = warp; i < known; i += kWeightThreads / 32) {
        bounds(tile0 + i, lo, hi, in_lo, in_hi);
        uint32_t f = s.n != tpt ? 2u : 0u;
        for (int t = lane; t < s.n; t += 32) {
          const int p = a.q.pre ? a.q.pre[s.first + t] : t;
          if (p >= lo && p < hi) f |= 1u;
          if (!(p >= in_lo && p < in_hi)) f |= 2u;
        }
        f = __reduce_or_sync(0xFFFFFFFFu, f);
        if (lane == 0) atomicOr(&flags[i >> 2], f << (8 * (i & 3)));
      }
    }
  }
  __syncthreads();
  if (warp == 0) {     // the visible ones in order; bit 15: pairs have to be looked at one by one
    int n = 0;
    for (int base = 0; base < known; base += 32) {
      const int i = base + lane;
      const uint32_t f = i < known ? (flags[i >> 2] >> (8 * (i & 3))) & 3u : 0u;
      const uint32_t some = __ballot_sync(0xFFFFFFFFu, f & 1u);
      if (f & 1u) list[n + __popc(some & ((1u << lane) - 1u))] = (uint16_t)(i | (f & 2u ? 0x8000 : 0));
      n += __popc(some);
    }
    if (lane == 0) *listed = n;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int nlist = *listed, count = nlist + items - known;     // products that are made
  auto item_of = [&](int n, bool& masked) -> int {
    if (n < nlist) {
      const int e = list[n];
      masked = (e & 0x8000) != 0;
      return e & 0x7FFF;
    }
    masked = true;
    return known + n - nlist;
  };
  auto item = [&](int n) -> int {
    bool masked;
    return item_of(n, masked);
  };
  const long long limit = a.wait_limit;
  auto wait_warp = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort_flag, limit, 0u)) != 0; };
  const bool work = count > 0;
  pdl_launch_dependents();
  float total = 0.f;
  // another CTA's shared memory may be written once that CTA runs: awaited below
  if (ranks > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");

  if (warp == 0) {
    if (!a.withhold_loads && work) {
      const TileBoxes<D> bx(a.q.cache.page_log2, lane);
      auto page_of = [&](int tile) {
        const int slot = tile * kAttnTile + bx.slot;
        if (tile >= tile1 || lane >= bx.boxes || slot >= s.len) return a.q.cache.num_pages;   // out of the map: filled with zeros
        const int p = cache_page(a.q.cache, seq, slot, dev_status);
        return p >= 0 ? p : a.q.cache.num_pages;
      };
      auto load_rows = [&](uint32_t dst, uint32_t bar, int tile) {
        if (lane == 0) {
          mbar_expect_tx(bar, (uint32_t)(a.q.G * tpt * D * 2));
          for (int c = 0; c < D / 64; ++c) tma_load_3d(dst + (uint32_t)c * (kAttnTile * 128), &map_q, bar, c * 64, hk * a.q.G, s.first + tile * tpt);
        }
        __syncwarp();
      };
      auto load_slots = [&](uint32_t dst, uint32_t bar, int tile, int page) {
        if (lane == 0) mbar_expect_tx(bar, Cfg::kTileBytes);
        __syncwarp();
        bx.issue(dst, &map_k, bar, tile, hk, page, lane);
      };
      int page = page_of(slot_tile(item(0)));
      if (MANY) load_slots(smem_base, stay_bar, tile0, page);
      else load_rows(smem_base, stay_bar, 0);
      for (int n = 0; n < count; ++n) {
        const int next_page = MANY || n + 1 >= count ? 0 : page_of(slot_tile(item(n + 1)));
        const int stage = n & 1;
        if (!wait_warp(r_empty(stage), ((uint32_t)(n >> 1) & 1u) ^ 1u)) break;
        const uint32_t dst = smem_base + Cfg::kRing + (uint32_t)stage * Cfg::kTileBytes;
        if (MANY) load_rows(dst, r_full(stage), row_tile(item(n)));
        else load_slots(dst, r_full(stage), slot_tile(item(n)), page);
        page = next_page;
      }
    }
  } else if (warp == 1) {
    if (work && wait_warp(stay_bar, 0)) {
      const uint32_t idesc = (1u << 4) | (AttnType<T>::fmt << 7) | (AttnType<T>::fmt << 10) | ((uint32_t)(kAttnTile >> 4) << 24) |
                             (uniform((uint32_t)ncols >> 3) << 17);
      const uint32_t tm = uniform(tmem_base), base = uniform(smem_base), stay = desc_low(base, 16);
      for (int n = 0; n < count; ++n) {
        const int at = n & 1;   // stage, accumulator and group at once
        const uint32_t phase = (uint32_t)(n >> 1) & 1u;
        if (!wait_warp(r_full(at), phase) || !wait_warp(s_empty(at), phase ^ 1u)) break;
        tc_fence_after();
        const uint32_t u = uniform((uint32_t)at), ring = desc_low(base + Cfg::kRing + u * Cfg::kTileBytes, 16);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < D / kUmmaK; ++k)
            umma_ss(tm + u * kAttnTile, MANY ? stay : ring, MANY ? ring : stay, (uint32_t)((k / 4) * (kAttnTile * 128 / 16) + (k % 4) * 2), idesc, (uint32_t)(k != 0));
          umma_commit(r_empty(0) + 8u * u);
          umma_commit(s_full(0) + 8u * u);
        }
        __syncwarp();
      }
    }
  } else {
    const int st = (warp - 2) >> 2, quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t t_s = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)st * kAttnTile;
    int2 iv = slot_interval(a.q, s, tile0 * kAttnTile + row);
    const float c = a.q.scale * 1.4426950408889634f;
    const uint64_t c2 = pair2(c, c);
    // column `row` of a row tile: which token and head it stands for
    const int ct = row / a.q.G, ch = hk * a.q.G + row % a.q.G;
    auto column = [&](int tile, float& nl, int& p) {
      const int t = tile * tpt + ct;
      nl = -INFINITY;      // no row: 2^(x - inf) = 0
      p = -1;
      if (ct < tpt && t < s.n) {
        const int64_t token = s.first + t;
        p = a.q.pre ? a.q.pre[token] : t;
        const float x = a.lse[token * a.q.Hq + ch];
        if (x != -INFINITY) nl = x * -1.4426950408889634f;
      }
    };
    float nl;
    int p;
    bool ok = true;
    if (st < count) column(row_tile(item(st)), nl, p);
    for (int n = st, k = 0; n < count; n += 2, ++k) {
      float* nlse = col_lse + (st * 2 + (MANY ? k & 1 : 0)) * kAttnTile;
      int* place = col_place + (st * 2 + (MANY ? k & 1 : 0)) * kAttnTile;
      bool masked;
      const int i = item_of(n, masked);
      const int slot = slot_tile(i) * kAttnTile + row;
      if (MANY || k == 0) {
        nlse[row] = nl;
        place[row] = p;
        __syncwarp();
        if (lane == 0) mbar_arrive(c_bar(st));
        ok = wait_warp(c_bar(st), (uint32_t)k & 1u);
        if (MANY && n + 2 < count) column(row_tile(item(n + 2)), nl, p);   // the next one's, while this one's products are waited for
      }
      float before = 0.f;
      if (!MANY) {
        iv = slot_interval(a.q, s, slot);
        before = old_weight(slot);
      }
      ok = ok && wait_warp(s_full(st), (uint32_t)k & 1u);
      if (!ok) break;
      tc_fence_after();
      const bool warp_in = slot - lane < s.len;
      uint64_t sum[2] = {0, 0};
      if (warp_in) {
        uint32_t v[16], w[16];
        ATTS_TMEM_LD_16(t_s, v);
#pragma unroll 1
        for (int j = 0; j < ncols; j += 32) {   // 16 columns are read while 16 are worked on
          tmem_ld_wait();
          ATTS_TMEM_LD_16(t_s + (uint32_t)(j + 16), w);
          if (masked) weight_columns<true>(v, nlse + j, place + j, iv, c2, sum);
          else weight_columns<false>(v, nlse + j, place + j, iv, c2, sum);
          tmem_ld_wait();
          if (j + 32 < ncols) ATTS_TMEM_LD_16(t_s + (uint32_t)(j + 32), v);
          if (masked) weight_columns<true>(w, nlse + j + 16, place + j + 16, iv, c2, sum);
          else weight_columns<false>(w, nlse + j + 16, place + j + 16, iv, c2, sum);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(s_empty(st));
      const uint64_t both = add2(sum[0], sum[1]);
      const float x = low2(both) + high2(both);
      if (MANY) total += x;
      else if (slot < a.q.max_len) wout[slot] = slot < s.len ? before + x : 0.f;
    }
    if (MANY) {
      if (st == 1) sums[kWeightMaxCluster * kAttnTile + row] = total;
    } else {
      // tiles of which nothing is visible, and those behind the sequence
      for (int t = tile0 + st; t < tile1; t += 2)
        if (t - tile0 >= items || !((flags[(t - tile0) >> 2] >> (8 * ((t - tile0) & 3))) & 1u)) {   // (a span is at most 8 tiles)
          const int slot = t * kAttnTile + row;
          if (slot < a.q.max_len) wout[slot] = old_weight(slot);
        }
    }
  }

  // ---------------- sums of the two groups, then of the cluster's CTAs in order ----------------
  tc_fence_before();
  __syncthreads();
  if (MANY) {
    if (ranks > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    const int row = (warp & 3) * 32 + lane;
    const bool first = warp >= 2 && warp < 6;
    if (first) {
      total += sums[kWeightMaxCluster * kAttnTile + row];
      if (rank == 0) sums[row] = total;
      else
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(map_to_cta(smem_u32(sums + rank * kAttnTile + row), 0)), "f"(total) : "memory");
    }
    if (ranks > 1) cluster_sync_all();
    if (rank == 0 && first) {
      const int slot = tile0 * kAttnTile + row;
      float w = 0.f;
      for (int i = 0; i < ranks; ++i) w += sums[i * kAttnTile + row];
      if (slot < a.q.max_len) wout[slot] = slot < s.len ? old_weight(slot) + w : 0.f;
    }
  }
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicOr(dev_status, 2u);
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(256u) : "memory");
  }
}

// Opt-in shared memory of the kernels above (once per device).
template <typename T, int D, AttnMode MODE, AttnForm FORM>
static cudaError_t attention_attribute(cudaError_t before) {
  return before != cudaSuccess ? before : cudaFuncSetAttribute(tree_attention_kernel<T, D, MODE, FORM>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                               AttnCfg<D, MODE, FORM>::kSmemBytes);
}
template <typename T, int D>
static cudaError_t attention_attributes_of() {
  cudaError_t e = attention_attribute<T, D, kRowsTwo, kFormPlain>(cudaSuccess);
  e = attention_attribute<T, D, kRowsOne, kFormPlain>(e);
  e = attention_attribute<T, D, kRowsBrief, kFormPlain>(e);
  e = attention_attribute<T, D, kRowsTwo, kFormWindow>(e);
  e = attention_attribute<T, D, kRowsOne, kFormWindow>(e);
  e = attention_attribute<T, D, kRowsBrief, kFormWindow>(e);
  e = attention_attribute<T, D, kRowsHalf, kFormWindow>(e);
  e = attention_attribute<T, D, kRowsHalf, kFormPacked>(e);
  e = attention_attribute<T, D, kRowsHalf, kFormPackedWindow>(e);
  e = attention_attribute<T, D, kRowsTwo, kFormPacked>(e);
  e = attention_attribute<T, D, kRowsOne, kFormPacked>(e);
  e = attention_attribute<T, D, kRowsTwo, kFormPackedWindow>(e);
  e = attention_attribute<T, D, kRowsOne, kFormPackedWindow>(e);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(cache_weights_kernel<T, D, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, WeightCfg<D>::kSmemBytes);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(cache_weights_kernel<T, D, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, WeightCfg<D>::kSmemBytes);
  return e;
}
static cudaError_t attention_attributes() {
  cudaError_t e = attention_attributes_of<__nv_bfloat16, 128>();
  if (e == cudaSuccess) e = attention_attributes_of<__nv_bfloat16, 64>();
  if (e == cudaSuccess) e = attention_attributes_of<__half, 128>();
  if (e == cudaSuccess) e = attention_attributes_of<__half, 64>();
  return e;
}

}  // namespace atts
