// Rotary append and eviction over a paged cache: the memory-bound part of the attention side (atts_rope_append,
// atts_cache_select, atts_cache_gather).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace atts {

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
  if (col < c.table_cols) page = c.table[(int64_t)seq * c.table_stride + col];
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
// ------------------------------------------------------------------------------------------------------------------
constexpr int kRopeThreads = 256;
constexpr int kRopeLanes = 8;  // threads that share a row

struct RopeArgs {
  const char *q, *k, *v;
  char* q_out;
  int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs;  // elements
  const int32_t *positions, *ctx, *cu;
  const double* freqs;
  int pairs, D, Hq, M, tpb, max_tokens;
  float mscale;
  CacheView cache;
};

template <typename T, bool INTERLEAVED, bool WIDE>
__global__ void __launch_bounds__(kRopeThreads)
rope_append_kernel(const RopeArgs a, unsigned* __restrict__ dev_status) {
  extern __shared__ float2 rope_cs[];  // [tpb][pairs]
  const int seq = blockIdx.y;
  int first, n;
  const bool ok = seq_rows(a.cu, seq, a.M, first, n);
  const int ctx = a.ctx[seq];
  if (!ok || ctx < 0 || n > a.max_tokens) {
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
  const int lane = threadIdx.x % kRopeLanes;
  for (int r = threadIdx.x / kRopeLanes; r < nt * rows; r += kRopeThreads / kRopeLanes) {
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
      if (INTERLEAVED) {
        for (int c = lane; c < a.D / 8; c += kRopeLanes) {
          uint4 x = s4[c];
          if (c < turned) {
            uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = Pack<T>::unpack(w[e]), g = cs[4 * c + e];
              w[e] = Pack<T>::pack(f.x * g.x - f.y * g.y, f.y * g.x + f.x * g.y);
            }
            x = make_uint4(w[0], w[1], w[2], w[3]);
          }
          d4[c] = x;
        }
      } else {
        const int half = turned / 2;
        for (int c = lane; c < half; c += kRopeLanes) {
          const uint4 x = s4[c], y = s4[c + half];
          const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
          uint32_t ow[4], pw[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 f = Pack<T>::unpack(xw[e]), g = Pack<T>::unpack(yw[e]);
            const float2 c0 = cs[8 * c + 2 * e], c1 = cs[8 * c + 2 * e + 1];
            ow[e] = Pack<T>::pack(f.x * c0.x - g.x * c0.y, f.y * c1.x - g.y * c1.y);
            pw[e] = Pack<T>::pack(g.x * c0.x + f.x * c0.y, g.y * c1.x + f.y * c1.y);
          }
          d4[c] = make_uint4(ow[0], ow[1], ow[2], ow[3]);
          d4[c + half] = make_uint4(pw[0], pw[1], pw[2], pw[3]);
        }
        for (int c = turned + lane; c < a.D / 8; c += kRopeLanes) d4[c] = s4[c];
      }
    } else {
      const int turned = turn ? a.pairs : 0;
      for (int i = lane; i < turned; i += kRopeLanes) {
        const int i0 = INTERLEAVED ? 2 * i : i, i1 = INTERLEAVED ? 2 * i + 1 : i + a.pairs;
        const float x = Pack<T>::get(src[i0]), y = Pack<T>::get(src[i1]);
        dst[i0] = Pack<T>::put(x * cs[i].x - y * cs[i].y);
        dst[i1] = Pack<T>::put(y * cs[i].x + x * cs[i].y);
      }
      for (int i = 2 * turned + lane; i < a.D; i += kRopeLanes) dst[i] = src[i];
    }
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Eviction, selection.  Weights are ordered by a monotone 32-bit key (-0 as +0; NaN below every number); the slots that
// stay in any case get the largest key.  One block per (sequence, head) finds the key of the last slot to keep digit by
// digit (four digits of eight bits, a histogram each over the slots that still match), then writes the slots above it
// and, from the lowest on, as many of the slots equal to it as there is room for.
// ------------------------------------------------------------------------------------------------------------------
constexpr int kSelectThreads = 1024;

__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0u;        // NaN
  if ((u & 0x7FFFFFFFu) == 0u) return 0x80000000u;       // both zeros
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);     // -inf has key 0x007FFFFF, +inf 0xFF800000
}

__global__ void __launch_bounds__(kSelectThreads)
cache_select_kernel(const float* __restrict__ weights, int64_t cols, const int32_t* __restrict__ lens, int heads, int budget,
                    int sinks, int recent, int32_t* __restrict__ kept, int32_t* __restrict__ counts,
                    unsigned* __restrict__ dev_status) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t scan[32];
  __shared__ uint32_t sh_prefix, sh_need;
  const int seq = blockIdx.x / heads, head = blockIdx.x - seq * heads;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int len0 = lens[seq];
  const int len = (int)max((int64_t)0, min((int64_t)len0, cols));
  if (tid == 0 && head == 0) {
    if (len != len0) atomicOr(dev_status, kDevSeqRange);
    counts[seq] = min(len, budget);
  }
  const float* w = weights + (int64_t)blockIdx.x * cols;
  int32_t* out = kept + (int64_t)blockIdx.x * budget;
  if (len <= budget) {
    for (int i = tid; i < budget; i += kSelectThreads) out[i] = i < len ? i : -1;
    return;
  }
  auto key_of = [&](int i) { return (i < sinks || i >= len - recent) ? 0xFFFFFFFFu : weight_key(w[i]); };
  uint32_t prefix = 0, need = (uint32_t)budget;  // need: rank, among the matching slots, of the last one to keep
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kSelectThreads) hist[i] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
    for (int i = tid; i < len; i += kSelectThreads) {
      const uint32_t k = key_of(i);
      if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      uint32_t above = 0;
      int d = 255;
      for (; d > 0; --d) {
        if (above + hist[d] >= need) break;
        above += hist[d];
      }
      sh_prefix = prefix | ((uint32_t)d << shift);
      sh_need = need - above;
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
    uint32_t before = 0, total = 0;
    for (int j = 0; j < 32; ++j) {
      if (j < warp) before += scan[j];
      total += scan[j];
    }
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
// Eviction, move.  One warp-wide copy per kept row: D / 8 threads per (sequence, slot, head).
// ------------------------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256)
cache_gather_kernel(const CacheView src, const CacheView dst, int D, const int32_t* __restrict__ kept, int64_t kept_cols,
                    const int32_t* __restrict__ counts, const float* __restrict__ win, int64_t in_cols,
                    float* __restrict__ wout, unsigned* __restrict__ dev_status) {
  const int seq = blockIdx.z, head = blockIdx.y;
  const int lanes = D / 8;
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) / lanes;
  const int piece = (int)(((int64_t)blockIdx.x * 256 + threadIdx.x) % lanes);
  if (c >= kept_cols) return;
  const int64_t row = (int64_t)seq * src.heads + head;
  const bool live = c < counts[seq];
  int slot = live ? kept[row * kept_cols + c] : -1;
  if (live && slot < 0) {
    atomicOr(dev_status, kDevPageRange);
  } else if (live) {
    const int from = cache_page(src, seq, slot, dev_status), to = cache_page(dst, seq, (int)c, dev_status);
    if (from >= 0 && to >= 0) {
      const int64_t a = cache_offset(src, from, slot) + head * src.head_stride + 8 * piece;
      const int64_t b = cache_offset(dst, to, (int)c) + head * dst.head_stride + 8 * piece;
      *reinterpret_cast<uint4*>(dst.k + 2 * b) = *reinterpret_cast<const uint4*>(src.k + 2 * a);
      *reinterpret_cast<uint4*>(dst.v + 2 * b) = *reinterpret_cast<const uint4*>(src.v + 2 * a);
    }
  }
  if (wout && piece == 0) {
    float x = 0.f;
    if (live && slot >= 0) {
      if (slot < in_cols) x = win[row * in_cols + slot];
      else atomicOr(dev_status, kDevPageRange);
    }
    wout[row * kept_cols + c] = x;
  }
}

}  // namespace atts
