// Rotary append and eviction over a paged cache: the memory-bound part of the attention side (atts_rope_append,
// atts_cache_select, atts_cache_gather).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "conformal.cuh"

namespace atts {

constexpr int kMaxSlotsOfSeq = 1 << 30;
constexpr unsigned kDevPageRange = 16u, kDevSeqRange = 32u;  // ATTS_DEV_PAGE_RANGE, ATTS_DEV_SEQ_RANGE

// A paged cache as the kernels see it (atts_kv_cache with the page size as a shift).
struct CacheView {
  char* k;
  char* v;
  const int32_t* table;
  int64_t table_stride;
  int64_t page_stride, slot_stride, head_stride;  // elements
  int32_t table_cols, num_pages, page_log2, heads;
};

// Page of a sequence's slot, or -1 (recorded) where the table has none or names one that does not exist.
__device__ __forceinline__ int cache_page(const CacheView& c, int seq, int slot, unsigned* dev_status) {
  const int col = slot >> c.page_log2;
  int page = -1;
  if (slot >= 0 && col < c.table_cols) page = c.table[(int64_t)seq * c.table_stride + col];
  if (page < 0 || page >= c.num_pages) {
    atomicOr(dev_status, kDevPageRange);
    page = -1;
  }
  return page;
}

// Element offset of (page, slot, head 0) in k and v.
__device__ __forceinline__ int64_t cache_offset(const CacheView& c, int page, int slot) {
  return (int64_t)page * c.page_stride + (int64_t)(slot & ((1 << c.page_log2) - 1)) * c.slot_stride;
}

// Rows [first, first + n) of a sequence's drafted tokens, cut to [0, M).
__device__ __forceinline__ bool seq_rows(const int32_t* cu, int seq, int M, int& first, int& n) {
  const int a = cu[seq], b = cu[seq + 1];
  first = a;
  n = b - a;
  return a >= 0 && b >= a && b <= M;
}

template <typename T>
struct Pack;
template <>
struct Pack<__nv_bfloat16> {
  static __device__ __forceinline__ float2 unpack(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ float get(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ __nv_bfloat16 put(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct Pack<__half> {
  static __device__ __forceinline__ float2 unpack(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __half2 r = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ float get(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half put(float x) { return __float2half_rn(x); }
};

// ------------------------------------------------------------------------------------------------------------------
// Rotary append.  A block takes up to `tpb` consecutive drafted tokens of one sequence; it first computes their cosines
// and sines (shared by all heads), then streams the rows [query heads | key heads | value heads] of those tokens.
// The angle pos * f is formed and reduced to a fraction of a turn in 64 bits (2 multiplications and a rounding per
// (token, pair), shared by all heads), so the fp32 cosine sees an argument in [-pi, pi] at any position.
// Bound: HBM.  16,000 tokens of 40 + 8 + 8 heads of 128: 67.5 us = 5.4 TB/s of reads and writes, 0.82 of a plain copy; one to
// four tokens a block, and one thread for every 32 bytes of a row, keep 8 KB under way per block.  Each thread loads two
// 16-byte pieces before it stores either; with the pieces one after the other, 19 x 295 tokens of 40 + 8 + 8 heads with
// half of 128 rotated took 32.8 us instead of 28.6, and 32 x 400 of 16 + 16 + 16 heads of 64, on eight threads a row, 35.2
// instead of 26.1.  Two or eight tokens a block: 70.7 and 72.1 us at 16,000 tokens, against 67.5 with four.
// ------------------------------------------------------------------------------------------------------------------
constexpr int kRopeThreads = 256;

struct RopeArgs {
  const char *q, *k, *v;
  char* q_out;
  int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs;  // elements
  const int32_t *positions, *ctx, *cu;
  const double* freqs;
  int pairs, D, Hq, M, tpb, max_tokens;
  int lanes_log2;  // threads that share a row: one for every 32 bytes, at most 8
  float mscale;
  CacheView cache;
};

template <typename T, bool INTERLEAVED, bool WIDE>
__global__ void __launch_bounds__(kRopeThreads)
rope_append_kernel(const RopeArgs a, unsigned* __restrict__ dev_status) {
  extern __shared__ float2 rope_cs[];  // [tpb][pairs]
  pdl_wait();
  pdl_launch_dependents();
  const int seq = blockIdx.y;
  int first, n;
  const bool ok = seq_rows(a.cu, seq, a.M, first, n);
  const int ctx = a.ctx[seq];
  if (!ok || ctx < 0 || ctx > kMaxSlotsOfSeq || n > a.max_tokens) {
    if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(dev_status, kDevSeqRange);
    return;
  }
  const int t0 = blockIdx.x * a.tpb;
  if (t0 >= n) return;
  const int nt = min(a.tpb, n - t0);
  for (int e = threadIdx.x; e < nt * a.pairs; e += kRopeThreads) {
    const int t = e / a.pairs, i = e - t * a.pairs;
    double turns = (double)a.positions[first + t0 + t] * (a.freqs[i] * 0.15915494309189533577);  // 1 / (2 pi)
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    rope_cs[e] = make_float2(c * a.mscale, s * a.mscale);
  }
  __syncthreads();

  const int rows = a.Hq + 2 * a.cache.heads;
  const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
  for (int r = threadIdx.x >> a.lanes_log2; r < nt * rows; r += kRopeThreads >> a.lanes_log2) {
    const int t = r / rows, h = r - t * rows;
    const int64_t token = first + t0 + t;
    const T* src;
    T* dst;
    bool turn = true;
    if (h < a.Hq) {
      src = reinterpret_cast<const T*>(a.q) + token * a.q_ts + h * a.q_hs;
      dst = reinterpret_cast<T*>(a.q_out) + token * a.o_ts + h * a.o_hs;
    } else {
      const int slot = ctx + t0 + t;
      const int page = cache_page(a.cache, seq, slot, dev_status);
      if (page < 0) continue;
      const int64_t at = cache_offset(a.cache, page, slot);
      if (h < a.Hq + a.cache.heads) {
        const int hk = h - a.Hq;
        src = reinterpret_cast<const T*>(a.k) + token * a.k_ts + hk * a.k_hs;
        dst = reinterpret_cast<T*>(a.cache.k) + at + hk * a.cache.head_stride;
      } else {
        const int hk = h - a.Hq - a.cache.heads;
        src = reinterpret_cast<const T*>(a.v) + token * a.v_ts + hk * a.v_hs;
        dst = reinterpret_cast<T*>(a.cache.v) + at + hk * a.cache.head_stride;
        turn = false;
      }
    }
    const float2* cs = rope_cs + t * a.pairs;
    if (WIDE) {
      const uint4* s4 = reinterpret_cast<const uint4*>(src);
      uint4* d4 = reinterpret_cast<uint4*>(dst);
      const int turned = turn ? a.pairs / 4 : 0;  // 16-byte pieces that are rotated
      // A thread has two pieces under way at a time: the two halves of eight rotated pairs, or neighbours.
      const int pieces = a.D / 8, half = INTERLEAVED ? 0 : turned / 2, rest = INTERLEAVED ? 0 : turned;
      for (int u = lane; u < half + (pieces - rest + 1) / 2; u += lanes) {
        const bool halves = u < half;
        const int pa = halves ? u : rest + 2 * (u - half), pb = halves ? u + half : pa + 1;
        uint4 x = s4[pa], y = make_uint4(0, 0, 0, 0);
        if (pb < pieces) y = s4[pb];
        uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
        if (INTERLEAVED) {
          auto rotate = [&](uint32_t (&w)[4], int piece) {
            if (piece >= turned) return;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = Pack<T>::unpack(w[e]), g = cs[4 * piece + e];
              w[e] = Pack<T>::pack(f.x * g.x - f.y * g.y, f.y * g.x + f.x * g.y);
            }
          };
          rotate(xw, pa);
          rotate(yw, pb);
        } else if (halves) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 f = Pack<T>::unpack(xw[e]), g = Pack<T>::unpack(yw[e]);
            const float2 c0 = cs[8 * u + 2 * e], c1 = cs[8 * u + 2 * e + 1];
            xw[e] = Pack<T>::pack(f.x * c0.x - g.x * c0.y, f.y * c1.x - g.y * c1.y);
            yw[e] = Pack<T>::pack(g.x * c0.x + f.x * c0.y, g.y * c1.x + f.y * c1.y);
          }
        }
        d4[pa] = make_uint4(xw[0], xw[1], xw[2], xw[3]);
        if (pb < pieces) d4[pb] = make_uint4(yw[0], yw[1], yw[2], yw[3]);
      }
    } else {
      const int turned = turn ? a.pairs : 0;
      for (int i = lane; i < turned; i += lanes) {
        const int i0 = INTERLEAVED ? 2 * i : i, i1 = INTERLEAVED ? 2 * i + 1 : i + a.pairs;
        const float x = Pack<T>::get(src[i0]), y = Pack<T>::get(src[i1]);
        dst[i0] = Pack<T>::put(x * cs[i].x - y * cs[i].y);
        dst[i1] = Pack<T>::put(y * cs[i].x + x * cs[i].y);
      }
      for (int i = 2 * turned + lane; i < a.D; i += lanes) dst[i] = src[i];
    }
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Eviction, selection.  Weights are ordered by a monotone 32-bit key (-0 as +0; NaN below every number); the slots that
// stay in any case get the largest key.  T, the budget-th largest key, is found from its highest bit down: a bit of T is
// set if at least `budget` keys are not below T with it.  Kept are the keys above T and, from the lowest slot on, as many
// of those equal to T as there is room for.  As soon as a count is the budget itself the set is known.
//
// Rows of up to 32,768 slots: keys in registers, of one block or, from 4,097 slots on, of a cluster of two (a warp owns
// consecutive slots, so one scan over the warps places everything).  A pass over all keys costs a comparison and an addition
// each, and one barrier behind which every block has every warp's count, written through the cluster's shared memory; once
// no more keys than threads lie between the bounds of T, a block's share of them goes to its shared memory and the
// remaining bits are found among them, two a pass.  64 rows of 32,000 slots: 25 us (clusters of four, two waves of them: 35;
// of eight: 82); 8 rows: 23 us (22, 25); 64 rows of 16,000: 22 us (33, 79).  So the launch does not look at the number of rows.
// Longer rows read their weights again for every digit, one block a row: 32 rows of 131,071 slots 273 us, 8 rows 261.
// (A histogram of digits needs fewer passes over the keys, but weights share a few exponents and its atomics then meet in a few
// bins: 87 us; one block a row 43 us.)
constexpr int kSelectThreads = 1024;
constexpr int kSelectCluster = 2, kSelectMaxItems = 16;     // keys of a thread: rows of up to 2 * 16 * 1024 slots

__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0u;        // NaN
  if ((u & 0x7FFFFFFFu) == 0u) return 0x80000000u;       // both zeros
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);     // -inf has key 0x007FFFFF, +inf 0xFF800000
}

struct SelectArgs {
  const float* weights;
  int64_t cols;
  const int32_t* lens;
  int heads, budget, sinks, recent;
  int32_t *kept, *counts;
};

// Length of a row, the counts' entry, and rows that keep everything; false: nothing is left to do.
__device__ __forceinline__ bool select_row(const SelectArgs& a, int row, bool first, int& len, unsigned* dev_status) {
  const int seq = row / a.heads;
  const int len0 = a.lens[seq];
  len = (int)max((int64_t)0, min((int64_t)len0, a.cols));
  if (first && threadIdx.x == 0 && row == seq * a.heads) {
    if (len != len0) atomicOr(dev_status, kDevSeqRange);
    a.counts[seq] = min(len, a.budget);
  }
  if (len > a.budget) return true;
  int32_t* out = a.kept + (int64_t)row * a.budget;
  if (first)
    for (int i = threadIdx.x; i < a.budget; i += blockDim.x) out[i] = i < len ? i : -1;
  return false;
}

// ITEMS keys a thread, CL blocks a row.
template <int ITEMS, int CL>
__global__ void __launch_bounds__(kSelectThreads)
cache_select_kernel(const SelectArgs a, unsigned* __restrict__ dev_status) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ uint32_t part[2][3][CL * 32];     // counts of every warp of the cluster
  __shared__ uint32_t window[kSelectThreads];
  __shared__ uint32_t windowed;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  const int row = blockIdx.x / CL, rank = blockIdx.x % CL;
  int len;
  if (!select_row(a, row, rank == 0, len, dev_status)) return;   // the same for a whole cluster
  const float* w = a.weights + (int64_t)row * a.cols;
  const int mine_at = rank * 32 + warp;                   // this warp among the cluster's
  const int first = mine_at * 32 * ITEMS + lane;          // this thread's slots: first + 32 k
  // Writes a warp's count where every block of the cluster reads it; barrier() makes them visible.  The other buffer is
  // written next: nobody can be a whole pass behind.
  auto put = [&](int buffer, int c, uint32_t n) {
    if (CL == 1) {
      if (lane == 0) part[buffer][c][warp] = n;
    } else if (lane < CL) {
      uint32_t at;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(&part[buffer][c][mine_at])), "r"(lane));
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(n) : "memory");
    }
  };
  auto barrier = [&]() {
    __syncwarp();
    if (CL == 1) __syncthreads();
    else asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  };
  if (CL > 1) barrier();                                  // the others' shared memory may be written once they run
  uint32_t key[ITEMS];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int i = first + 32 * k;
    key[k] = i < len ? __float_as_uint(w[i]) : 0u;
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int i = first + 32 * k;
    key[k] = i >= len ? 0u : (i < a.sinks || i >= len - a.recent) ? 0xFFFFFFFFu : weight_key(__uint_as_float(key[k]));
  }
  // Slots behind the row have key 0, like NaNs: never above T, and last in the order among equals.
  const uint32_t budget = (uint32_t)a.budget;
  uint32_t T = 0, at_t = (uint32_t)(CL * ITEMS * blockDim.x), above = 0;   // keys >= T, keys above the bits still open
  bool exact = false;     // as many keys >= T as are kept
  int shift = 31, buf = 0;
  auto total = [&](int c) {
    uint32_t n = 0;
#pragma unroll
    for (int r = 0; r < CL; ++r) n += CL > 1 || lane < warps ? part[buf][c][r * 32 + lane] : 0u;
    return __reduce_add_sync(0xFFFFFFFFu, n);
  };
  if (tid == 0) windowed = 0;
  if (ITEMS > 1) {
    for (; shift >= 0 && !exact && at_t - above > blockDim.x; --shift, buf ^= 1) {
      const uint32_t cand = T | (1u << shift);
      uint32_t n = 0;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) n += key[k] >= cand ? 1u : 0u;
      n = __reduce_add_sync(0xFFFFFFFFu, n);
      put(buf, 0, n);
      barrier();
      n = total(0);
      if (n >= budget) {
        T = cand;
        at_t = n;
        exact = n == budget;
      } else {
        above = n;
      }
    }
  }
  if (shift >= 0 && !exact) {
    uint32_t mine = 0;
    if (ITEMS > 1) {
      const uint32_t span = shift == 31 ? 0xFFFFFFFFu : (2u << shift) - 1u;   // T .. T + span are open
      __syncthreads();
      // (one addition a warp: a thousand that wait for one another took 9 us)
      uint32_t own = 0;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) own += (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, key[k] - T <= span));
      uint32_t at = 0;
      if (lane == 0 && own) at = atomicAdd(&windowed, own);
      at = __shfl_sync(0xFFFFFFFFu, at, 0);
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const bool open = key[k] - T <= span;
        const uint32_t some = __ballot_sync(0xFFFFFFFFu, open);
        if (open) window[at + __popc(some & ((1u << lane) - 1u))] = key[k];
        at += __popc(some);
      }
      __syncthreads();
      if (tid < (int)windowed) mine = window[tid];
    } else {
      mine = key[0];
    }
    while (shift >= 0 && !exact) {
      const int bits = shift >= 1 ? 2 : 1, low = shift + 1 - bits, cands = (1 << bits) - 1;
      for (int c = 0; c < cands; ++c) {
        const uint32_t n = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, mine >= (T | ((uint32_t)(c + 1) << low))));
        put(buf, c, n);
      }
      barrier();
      for (int c = cands - 1; c >= 0; --c) {
        const uint32_t n = above + total(c);
        if (n >= budget) {
          T |= (uint32_t)(c + 1) << low;
          exact = n == budget;
          break;
        }
      }
      // (`above` counts keys beyond the window; those inside it are all counted again)
      shift -= bits;
      buf ^= 1;
    }
  }
  // places: keys above T (or all from T on, if that is exactly the budget), then the first ones equal to it
  uint32_t gt = 0, eq = 0;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    gt += key[k] > T ? 1u : 0u;
    eq += key[k] == T ? 1u : 0u;
  }
  gt = __reduce_add_sync(0xFFFFFFFFu, gt);
  eq = __reduce_add_sync(0xFFFFFFFFu, eq);
  put(buf, 0, gt);
  put(buf, 1, eq);
  barrier();
  uint32_t before_gt = 0, before_eq = 0;
#pragma unroll
  for (int r = 0; r < CL; ++r) {
    const bool in_front = r * 32 + lane < mine_at;
    before_gt += in_front ? part[buf][0][r * 32 + lane] : 0u;
    before_eq += in_front ? part[buf][1][r * 32 + lane] : 0u;
  }
  before_gt = __reduce_add_sync(0xFFFFFFFFu, before_gt);
  before_eq = __reduce_add_sync(0xFFFFFFFFu, before_eq);
  const uint32_t all_gt = total(0);
  const uint32_t need = budget - all_gt;                  // of the keys equal to T
  uint32_t g = before_gt, e = before_eq;
  const uint32_t lower = (1u << lane) - 1u;
  int32_t* out = a.kept + (int64_t)row * a.budget;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const bool is_gt = key[k] > T, is_eq = key[k] == T;
    const uint32_t bg = __ballot_sync(0xFFFFFFFFu, is_gt), be = __ballot_sync(0xFFFFFFFFu, is_eq);
    const uint32_t my_e = e + __popc(be & lower);
    if (is_gt || (is_eq && my_e < need)) out[g + __popc(bg & lower) + min(my_e, need)] = first + 32 * k;
    g += __popc(bg);
    e += __popc(be);
  }
}

// Longer rows: digits of eight bits, a histogram each over the slots that still match.  Lanes that hit the same bin count
// together first.
__global__ void __launch_bounds__(kSelectThreads)
cache_select_long_kernel(const SelectArgs a, unsigned* __restrict__ dev_status) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ uint32_t hist[256];
  __shared__ uint32_t scan[32];
  __shared__ uint32_t sh_prefix, sh_need;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int len;
  if (!select_row(a, blockIdx.x, true, len, dev_status)) return;
  const float* w = a.weights + (int64_t)blockIdx.x * a.cols;
  int32_t* out = a.kept + (int64_t)blockIdx.x * a.budget;
  auto key_of = [&](int i) { return (i < a.sinks || i >= len - a.recent) ? 0xFFFFFFFFu : weight_key(w[i]); };
  uint32_t prefix = 0, need = (uint32_t)a.budget;  // need: rank, among the matching slots, of the last one to keep
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kSelectThreads) hist[i] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
    for (int base = 0; base < len; base += kSelectThreads) {
      const int i = base + tid;
      uint32_t k = 0;
      bool hit = i < len;
      if (hit) {
        k = key_of(i);
        hit = (k & mask) == prefix;
      }
      const uint32_t bin = hit ? (k >> shift) & 255u : 256u;
      const uint32_t same = __match_any_sync(0xFFFFFFFFu, bin);
      if (hit && (same & ((1u << lane) - 1u)) == 0u) atomicAdd(&hist[bin], (uint32_t)__popc(same));
    }
    __syncthreads();
    if (warp == 0) {   // lane 0 has the highest eight bins
      uint32_t own = 0;
      for (int d = 0; d < 8; ++d) own += hist[255 - lane * 8 - d];
      uint32_t upto = own;
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += x;
      }
      const uint32_t has = __ballot_sync(0xFFFFFFFFu, upto >= need);   // some lane's: the matching slots are at least `need`
      if (lane == __ffs(has) - 1) {
        uint32_t above = upto - own;
        int d = 255 - lane * 8;
        while (above + hist[d] < need) above += hist[d--];
        sh_prefix = prefix | ((uint32_t)d << shift);
        sh_need = need - above;
      }
    }
    __syncthreads();
    prefix = sh_prefix;
    need = sh_need;
  }
  // slots above the threshold are kept, of those equal to it the first `need`
  uint32_t done = 0, equal_done = 0;
  for (int base = 0; base < len; base += kSelectThreads) {
    const int i = base + tid;
    const uint32_t k = i < len ? key_of(i) : 0u;
    const bool gt = i < len && k > prefix, eq = i < len && k == prefix;
    const uint32_t bg = __ballot_sync(0xFFFFFFFFu, gt), be = __ballot_sync(0xFFFFFFFFu, eq);
    if (lane == 0) scan[warp] = (uint32_t)__popc(bg) | ((uint32_t)__popc(be) << 16);
    __syncthreads();
    const uint32_t mine = scan[lane];
    const uint32_t before = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? mine : 0u), total = __reduce_add_sync(0xFFFFFFFFu, mine);
    const uint32_t lower = (1u << lane) - 1u;
    const uint32_t g = done + (before & 0xFFFFu) + __popc(bg & lower);
    const uint32_t e = equal_done + (before >> 16) + __popc(be & lower);
    if (gt || (eq && e < need)) out[g + min(e, need)] = i;
    done += total & 0xFFFFu;
    equal_done += total >> 16;
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Eviction, move.  A block takes up to kGatherSpan kept rows of one head: its threads first look up a row each (slot, then the two
// pages), then copy, D / 8 threads to a row with 16 bytes of its key and of its value each.  The look-ups are a chain of
// dependent accesses: done by every copying thread for its own rows they, not the bandwidth, set the time (64 x 8192 rows of
// 2 x 256 bytes: 118 us; 84 us so = 6.4 TB/s, 0.98 of a plain copy).
// ------------------------------------------------------------------------------------------------------------------
constexpr int kGatherThreads = 256, kGatherSpan = 256, kGatherUnroll = 4;   // (a span of 256 rows, fewer where that leaves SMs idle)

__global__ void __launch_bounds__(kGatherThreads)
cache_gather_kernel(const CacheView src, const CacheView dst, int lanes, int span, const int32_t* __restrict__ kept, int64_t kept_cols,
                    const int32_t* __restrict__ counts, const float* __restrict__ win, int64_t in_cols,
                    float* __restrict__ wout, unsigned* __restrict__ dev_status) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ int64_t from[kGatherSpan], to[kGatherSpan];   // byte offsets, -1: nothing to copy
  // blocks of the same slots and other heads run side by side: a slot's heads are neighbours in memory
  const int seq = blockIdx.y, head = blockIdx.x % src.heads;
  const int64_t row = (int64_t)seq * src.heads + head;
  const int64_t c0 = (int64_t)(blockIdx.x / src.heads) * span;
  const int64_t count = counts[seq], live_to = max((int64_t)0, min(count, kept_cols));
  if (live_to != count && threadIdx.x == 0 && blockIdx.x == 0) atomicOr(dev_status, kDevSeqRange);
  {
    const int64_t c = c0 + threadIdx.x;
    int64_t a = -1, b = -1;
    float w = 0.f;
    if (threadIdx.x < span && c < live_to) {
      const int slot = kept[row * kept_cols + c];
      const int to_col = (int)(c >> dst.page_log2), from_col = slot >> src.page_log2;
      const int q = to_col < dst.table_cols ? dst.table[seq * dst.table_stride + to_col] : -1;
      const int p = slot >= 0 && from_col < src.table_cols ? src.table[seq * src.table_stride + from_col] : -1;
      bool ok = p >= 0 && p < src.num_pages && q >= 0 && q < dst.num_pages;
      if (ok) {
        a = 2 * (cache_offset(src, p, slot) + head * src.head_stride);
        b = 2 * (cache_offset(dst, q, (int)c) + head * dst.head_stride);
      }
      if (wout && slot >= 0) {
        if (slot < in_cols) w = win[row * in_cols + slot];
        else ok = false;
      }
      if (!ok) atomicOr(dev_status, kDevPageRange);
    }
    from[threadIdx.x] = a;
    to[threadIdx.x] = b;
    if (wout && threadIdx.x < span && c < kept_cols) wout[row * kept_cols + c] = w;
  }
  __syncthreads();
  const int per = kGatherThreads / lanes;                          // rows of the block at a time
  const int sub = threadIdx.x / lanes, piece = 16 * (threadIdx.x - sub * lanes);
  if (sub >= per) return;
  const int rows = (int)max((int64_t)0, min((int64_t)span, live_to - c0));
  for (int r0 = sub; r0 < rows; r0 += per * kGatherUnroll) {
    uint4 k[kGatherUnroll], v[kGatherUnroll];
#pragma unroll
    for (int u = 0; u < kGatherUnroll; ++u) {
      const int r = r0 + u * per;
      if (r < rows && from[r] >= 0) {
        k[u] = *reinterpret_cast<const uint4*>(src.k + from[r] + piece);
        v[u] = *reinterpret_cast<const uint4*>(src.v + from[r] + piece);
      }
    }
#pragma unroll
    for (int u = 0; u < kGatherUnroll; ++u) {
      const int r = r0 + u * per;
      if (r < rows && from[r] >= 0) {
        *reinterpret_cast<uint4*>(dst.k + to[r] + piece) = k[u];
        *reinterpret_cast<uint4*>(dst.v + to[r] + piece) = v[u];
      }
    }
  }
}

}  // namespace atts
