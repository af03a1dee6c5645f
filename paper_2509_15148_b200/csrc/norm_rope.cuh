// Norms of queries and keys for each head with the rotation in the same pass (atts_norm_rope_append, atts_norm_rope).
#pragma once
#include "rope_cache.cuh"

namespace atts {

// ------------------------------------------------------------------------------------------------------------------
// A row of D channels becomes  y = x (mean(x^2) + eps)^(-1/2) gain,  then pairs of y are turned, and is rounded once.
// A block takes `tpb` consecutive tokens: first their cosines and sines (the angle reduced in 64 bits, as in rope_append_kernel) and
// the places of their slots, each looked up once for all heads, then the rows [query heads | key heads | value heads].
// `lanes` neighbouring threads share a row and hold it in registers, two 16-byte pieces each, so that it is read once although
// the sum of its squares (in fp32, by a fixed tree) has to be known before the first channel can be written.  A thread's pieces
// are the same in every row, so the gains of both kinds are loaded once and stay in registers too.
// ROWS: keys go to rows of their own instead of a cache, and there are no values (what a cache in 4 bits is filled from).
// ------------------------------------------------------------------------------------------------------------------
struct NormRopeArgs {
  const char *q, *k, *v, *q_gain, *k_gain;   // a NULL gain: that side is not normed
  char *q_out, *k_out;
  int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs, ko_ts, ko_hs;  // elements
  const int32_t *positions, *ctx, *cu;
  const double* freqs;
  int pairs, D, Hq, Hk, M, tpb, max_tokens;
  int lanes_log2;  // threads that share a row
  float mscale, eps;
  CacheView cache;
};
constexpr int kNormRopeMaxTokens = 8;   // of a block

template <typename T>
__device__ __forceinline__ float square_sum(const uint32_t (&w)[4]) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = Pack<T>::unpack(w[e]);
    s = fmaf(f.x, f.x, s);
    s = fmaf(f.y, f.y, s);
  }
  return s;
}
// Sum over the threads that share a row; every thread of the warp takes part.
__device__ __forceinline__ float row_sum(float s, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  return s;
}

template <typename T, bool INTERLEAVED, bool WIDE, bool ROWS>
__global__ void __launch_bounds__(kRopeThreads)
norm_rope_kernel(const __grid_constant__ NormRopeArgs a, unsigned* __restrict__ dev_status) {
  extern __shared__ float2 rope_cs[];                 // [tpb][pairs]
  __shared__ int64_t slot_at[kNormRopeMaxTokens];     // element offset of a token's slot in the cache, -1: none
  pdl_wait();
  pdl_launch_dependents();
  int first = 0, n = a.M, ctx = 0;
  if (!ROWS) {
    const int seq = blockIdx.y;
    const bool ok = seq_rows(a.cu, seq, a.M, first, n);
    ctx = a.ctx[seq];
    if (!ok || ctx < 0 || ctx > kMaxSlotsOfSeq || n > a.max_tokens) {
      if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(dev_status, kDevSeqRange);
      return;
    }
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
  if (!ROWS && threadIdx.x < nt) {
    const int slot = ctx + t0 + threadIdx.x;
    const int page = cache_page(a.cache, blockIdx.y, slot, dev_status);
    slot_at[threadIdx.x] = page < 0 ? -1 : cache_offset(a.cache, page, slot);
  }

  const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
  const int pieces = a.D / 8, turned = a.pairs / 4;      // 16-byte pieces of a row, and those that are rotated
  const int half = INTERLEAVED ? 0 : turned / 2, rest = INTERLEAVED ? 0 : turned;
  // This thread's pieces of every row: the two halves of eight rotated pairs, or neighbours; -1: none.
  const bool halves = lane < half;
  const int pa = WIDE ? (halves ? lane : rest + 2 * (lane - half)) : 0, pb = halves ? lane + half : pa + 1;
  const bool has_a = WIDE && pa < pieces, has_b = WIDE && pb < pieces;
  uint4 gain[2][2] = {};                                  // of queries, of keys
  if (WIDE) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const uint4* from = reinterpret_cast<const uint4*>(g ? a.k_gain : a.q_gain);
      if (from && has_a) gain[g][0] = from[pa];
      if (from && has_b) gain[g][1] = from[pb];
    }
  }
  __syncthreads();

  const int rows = a.Hq + (ROWS ? 1 : 2) * a.Hk, stride = kRopeThreads >> a.lanes_log2;
  for (int r0 = 0; r0 < nt * rows; r0 += stride) {        // as many turns for every thread: rows are summed by whole warps
    const int r = r0 + (threadIdx.x >> a.lanes_log2);
    bool live = r < nt * rows;
    const int t = live ? r / rows : 0, h = r - t * rows;
    const int64_t token = first + t0 + t;
    const T* src = nullptr;
    T* dst = nullptr;
    int kind = 0;                                         // 0 query, 1 key, 2 value
    if (live) {
      if (h < a.Hq) {
        src = reinterpret_cast<const T*>(a.q) + token * a.q_ts + h * a.q_hs;
        dst = reinterpret_cast<T*>(a.q_out) + token * a.o_ts + h * a.o_hs;
      } else {
        kind = h < a.Hq + a.Hk ? 1 : 2;
        const int hk = h - a.Hq - (kind == 2 ? a.Hk : 0);
        src = kind == 1 ? reinterpret_cast<const T*>(a.k) + token * a.k_ts + hk * a.k_hs : reinterpret_cast<const T*>(a.v) + token * a.v_ts + hk * a.v_hs;
        if (ROWS) {
          dst = reinterpret_cast<T*>(a.k_out) + token * a.ko_ts + hk * a.ko_hs;
        } else {
          live = slot_at[t] >= 0;
          dst = reinterpret_cast<T*>(kind == 1 ? a.cache.k : a.cache.v) + slot_at[t] + hk * a.cache.head_stride;
        }
      }
    }
    const char* gains = kind == 0 ? a.q_gain : a.k_gain;
    const bool norm = kind < 2 && gains;
    const float2* cs = rope_cs + t * a.pairs;
    if (WIDE) {
      uint4 x = make_uint4(0, 0, 0, 0), y = x;
      if (live && has_a) x = reinterpret_cast<const uint4*>(src)[pa];
      if (live && has_b) y = reinterpret_cast<const uint4*>(src)[pb];
      uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
      const float f = rsqrtf(row_sum(square_sum<T>(xw) + square_sum<T>(yw), lanes) / (float)a.D + a.eps);
      if (live && kind < 2) {
        const uint4 gx = kind ? gain[1][0] : gain[0][0], gy = kind ? gain[1][1] : gain[0][1];
        const uint32_t gxw[4] = {gx.x, gx.y, gx.z, gx.w}, gyw[4] = {gy.x, gy.y, gy.z, gy.w};
        float u[8], v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 p = Pack<T>::unpack(xw[e]), q = Pack<T>::unpack(yw[e]), g = Pack<T>::unpack(gxw[e]), k = Pack<T>::unpack(gyw[e]);
          u[2 * e] = norm ? p.x * f * g.x : p.x;
          u[2 * e + 1] = norm ? p.y * f * g.y : p.y;
          v[2 * e] = norm ? q.x * f * k.x : q.x;
          v[2 * e + 1] = norm ? q.y * f * k.y : q.y;
        }
        if (INTERLEAVED) {
          auto rotate = [&](float (&w)[8], int piece) {
            if (piece >= turned) return;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 g = cs[4 * piece + e];
              const float x0 = w[2 * e];
              w[2 * e] = x0 * g.x - w[2 * e + 1] * g.y;
              w[2 * e + 1] = w[2 * e + 1] * g.x + x0 * g.y;
            }
          };
          rotate(u, pa);
          rotate(v, pb);
        } else if (halves) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 g = cs[8 * lane + e];
            const float x0 = u[e];
            u[e] = x0 * g.x - v[e] * g.y;
            v[e] = v[e] * g.x + x0 * g.y;
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          xw[e] = Pack<T>::pack(u[2 * e], u[2 * e + 1]);
          yw[e] = Pack<T>::pack(v[2 * e], v[2 * e + 1]);
        }
      }
      if (live && has_a) reinterpret_cast<uint4*>(dst)[pa] = make_uint4(xw[0], xw[1], xw[2], xw[3]);
      if (live && has_b) reinterpret_cast<uint4*>(dst)[pb] = make_uint4(yw[0], yw[1], yw[2], yw[3]);
    } else {
      float s = 0.f;
      if (live && norm)
        for (int i = lane; i < a.D; i += lanes) {
          const float x = Pack<T>::get(src[i]);
          s = fmaf(x, x, s);
        }
      const float f = rsqrtf(row_sum(s, lanes) / (float)a.D + a.eps);
      if (!live) continue;                                // (no warp-wide step follows in this turn)
      const T* g = reinterpret_cast<const T*>(gains);
      auto at = [&](int i) { return norm ? Pack<T>::get(src[i]) * f * Pack<T>::get(g[i]) : Pack<T>::get(src[i]); };
      const int pairs = kind < 2 ? a.pairs : 0;
      for (int i = lane; i < pairs; i += lanes) {
        const int i0 = INTERLEAVED ? 2 * i : i, i1 = INTERLEAVED ? 2 * i + 1 : i + a.pairs;
        const float x = at(i0), y = at(i1);
        dst[i0] = Pack<T>::put(x * cs[i].x - y * cs[i].y);
        dst[i1] = Pack<T>::put(y * cs[i].x + x * cs[i].y);
      }
      for (int i = 2 * pairs + lane; i < a.D; i += lanes) dst[i] = norm ? Pack<T>::put(at(i)) : src[i];
    }
  }
}

}  // namespace atts
