// Norms of queries and keys for each head with the rotation in the same pass (atts_norm_rope_append, atts_norm_rope).
#pragma once
#include "rope_cache.cuh"

namespace atts {

// ------------------------------------------------------------------------------------------------------------------
// A row of D channels becomes  y = x (mean(x^2) + eps)^(-1/2) gain,  then pairs of y are turned, and is rounded once.
// A block takes `tpb` consecutive tokens: first their cosines and sines (the angle reduced in 64 bits, as in rope_append_kernel) and
// the places of their slots, each looked up once for all heads, then the rows [query heads | key heads | value heads].
// `lanes` neighbouring threads share a row and hold it in registers, two 16-byte pieces each, so that it is read once although
// the sum of its squares (in fp32, by a fixed tree) has to be known before the first channel can be written.  A group of them takes
// one token's heads, first queries, then keys, then values, with the products of its channels' gains and cosines and sines in
// registers: a row then costs two packed multiply-adds a pair and a scaling (with cosines from shared memory and gains by the row
// 12,675 tokens of 40 + 8 + 8 heads of 128 took 96 us, bound by instructions).
// Bound: HBM from some thousand tokens on: 12,675 tokens of 40 + 8 + 8 heads of 128 in 32 sequences 71 us = 5.1 TB/s, 0.78 of a plain copy
// (rope_append_kernel 67.5).  Tokens of a block, as many as leave two blocks to an SM if sequences fill theirs: 16 / 8 / 4 tokens
// 71 / 76 / 95 us there, 16 / 4 / 1 at 1,503 tokens in 23 sequences 16.3 / 11.4 / 23.7.  A block takes tokens of one sequence, and the
// number is chosen by the batch's tokens alone: many short sequences leave most of its threads without a row (sequences of one token,
// 600 / 2,400 / 9,600 of them: 14.7 / 77 / 460 us, where rope_append_kernel, which deals rows to all threads, takes 5.4 / 17.7 / 64).
// Two rows' loads on their way and at most 80 registers (three blocks an SM; the append's wide forms spill 24 bytes a thread, the
// wide one from rows to rows that is not interleaved 8); one row and four blocks 85 us.
// ROWS: keys go to rows of their own instead of a cache, and there are no values (what a cache in 4 bits is filled from): 12,675 tokens of
// 40 + 8 heads 60 us = 5.2 TB/s, 1,503 of 28 + 4 8.6, of 9,600 sequences of one token 52 (it knows no sequences).
// ------------------------------------------------------------------------------------------------------------------
struct NormRopeArgs {
  const char *q, *k, *v, *q_gain, *k_gain;   // a NULL gain: that side is not normed
  char *q_out, *k_out;
  int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs, ko_ts, ko_hs;  // elements
  const int32_t *positions, *ctx, *cu;
  const double* freqs;
  int pairs, D, Hq, Hk, M, tpb, max_tokens;
  int lanes_log2;  // threads that share a row
  float mscale, eps, inv_d;
  CacheView cache;
};
constexpr int kNormRopeMaxTokens = 16;   // of a block

// 16 bytes of a row as four pairs of neighbouring channels in fp32.
template <typename T>
__device__ __forceinline__ void unpack_piece(const uint4& x, uint64_t (&v)[4]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = Pack<T>::unpack(w[e]);
    v[e] = pair2(f.x, f.y);
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack_piece(const uint64_t (&v)[4]) {
  return make_uint4(Pack<T>::pack(low2(v[0]), high2(v[0])), Pack<T>::pack(low2(v[1]), high2(v[1])), Pack<T>::pack(low2(v[2]), high2(v[2])),
                    Pack<T>::pack(low2(v[3]), high2(v[3])));
}
// Sum over the threads that share a row; every thread of the warp takes part.
__device__ __forceinline__ float row_sum(float s, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  return s;
}

template <typename T, bool INTERLEAVED, bool WIDE, bool ROWS>
__global__ void __launch_bounds__(kRopeThreads, WIDE ? 3 : 1)
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
  __syncthreads();

  // `lanes` threads are a group; group g takes heads g / tpb, g / tpb + subs, .. of token g % tpb.
  const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.lanes_log2;
  const int t = group % a.tpb, sub = group / a.tpb, subs = (kRopeThreads >> a.lanes_log2) / a.tpb;
  const bool token_in = t < nt;
  const int64_t token = first + t0 + t, at = !ROWS && token_in ? slot_at[t] : -1;
  const float2* cs = rope_cs + (token_in ? t * a.pairs : 0);
  if (WIDE) {
    const int pieces = a.D / 8, turned = a.pairs / 4;    // 16-byte pieces of a row, and those that are rotated
    const int half = INTERLEAVED ? 0 : turned / 2, rest = INTERLEAVED ? 0 : turned;
    // This thread's pieces of every row: the two halves of eight rotated pairs, or neighbours.
    const bool halves = lane < half;
    const int pa = halves ? lane : rest + 2 * (lane - half), pb = halves ? lane + half : pa + 1;
    const bool has_a = pa < pieces, has_b = pb < pieces;
#pragma unroll 1
    for (int kind = 0; kind < (ROWS ? 2 : 3); ++kind) {  // queries, keys, values
      const int heads = kind == 0 ? a.Hq : a.Hk;
      const T* src = reinterpret_cast<const T*>(kind == 0 ? a.q : kind == 1 ? a.k : a.v) + token * (kind == 0 ? a.q_ts : kind == 1 ? a.k_ts : a.v_ts);
      const int64_t src_hs = kind == 0 ? a.q_hs : kind == 1 ? a.k_hs : a.v_hs, dst_hs = kind == 0 ? a.o_hs : ROWS ? a.ko_hs : a.cache.head_stride;
      T* dst = kind == 0 ? reinterpret_cast<T*>(a.q_out) + token * a.o_ts
               : ROWS    ? reinterpret_cast<T*>(a.k_out) + token * a.ko_ts
                         : reinterpret_cast<T*>(kind == 1 ? a.cache.k : a.cache.v) + at;
      const bool token_live = token_in && (kind == 0 || ROWS || at >= 0);
      const char* gains = kind == 0 ? a.q_gain : kind == 1 ? a.k_gain : nullptr;
      // (x, y) of a pair becomes f (x cx + y sx, y cy + x sy): cosines and sines with the channels' gains in them, for this
      // token and kind of row.  Pieces that are not rotated have their gains in cx and cy.
      uint64_t cx[4], cy[4], sx[4], sy[4];
      bool turn_a = false, turn_b = false;
      if (kind < 2) {
        uint64_t ga[4], gb[4];
        const uint64_t ones = pair2(1.f, 1.f);
#pragma unroll
        for (int e = 0; e < 4; ++e) ga[e] = gb[e] = ones;
        if (gains && has_a) unpack_piece<T>(reinterpret_cast<const uint4*>(gains)[pa], ga);
        if (gains && has_b) unpack_piece<T>(reinterpret_cast<const uint4*>(gains)[pb], gb);
        turn_a = INTERLEAVED ? pa < turned : halves;
        turn_b = INTERLEAVED ? pb < turned : halves;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          cx[e] = ga[e];
          cy[e] = gb[e];
          sx[e] = sy[e] = 0;
          if (INTERLEAVED) {                             // both pieces hold pairs of their own: (c g0, c g1) and (-s g1, s g0)
            if (turn_a) {
              const float2 r = cs[4 * pa + e];
              cx[e] = mul2(pair2(r.x, r.x), ga[e]);
              sx[e] = mul2(pair2(-r.y, r.y), pair2(high2(ga[e]), low2(ga[e])));
            }
            if (turn_b) {
              const float2 r = cs[4 * pb + e];
              cy[e] = mul2(pair2(r.x, r.x), gb[e]);
              sy[e] = mul2(pair2(-r.y, r.y), pair2(high2(gb[e]), low2(gb[e])));
            }
          } else if (halves) {
            const float2 r0 = cs[8 * lane + 2 * e], r1 = cs[8 * lane + 2 * e + 1];
            const uint64_t c = pair2(r0.x, r1.x);
            cx[e] = mul2(c, ga[e]);
            cy[e] = mul2(c, gb[e]);
            sx[e] = mul2(pair2(-r0.y, -r1.y), gb[e]);
            sy[e] = mul2(pair2(r0.y, r1.y), ga[e]);
          }
        }
      }
      constexpr int kAtOnce = 2;                         // rows of a thread whose loads are on their way together
#pragma unroll 1
      for (int h0 = 0; h0 < heads; h0 += kAtOnce * subs) {   // as many turns for every thread: rows are summed by whole warps
        uint4 x[kAtOnce], y[kAtOnce];
        bool live[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int h = h0 + u * subs + sub;
          live[u] = token_live && h < heads;
          x[u] = y[u] = make_uint4(0, 0, 0, 0);
          const uint4* from = reinterpret_cast<const uint4*>(src + h * src_hs);
          if (live[u] && has_a) x[u] = from[pa];
          if (live[u] && has_b) y[u] = from[pb];
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          if (kind < 2) {
            uint64_t p[4], q[4];
            unpack_piece<T>(x[u], p);
            unpack_piece<T>(y[u], q);
            float f = 1.f;
            if (gains) {
              uint64_t sum = 0;
#pragma unroll
              for (int e = 0; e < 4; ++e) sum = fma2(q[e], q[e], fma2(p[e], p[e], sum));
              f = rsqrtf(row_sum(low2(sum) + high2(sum), lanes) * a.inv_d + a.eps);
            }
            const uint64_t ff = pair2(f, f);
            uint64_t v[4], w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v[e] = mul2(p[e], cx[e]);
              w[e] = mul2(q[e], cy[e]);
              if (turn_a) v[e] = fma2(INTERLEAVED ? pair2(high2(p[e]), low2(p[e])) : q[e], sx[e], v[e]);
              if (turn_b) w[e] = fma2(INTERLEAVED ? pair2(high2(q[e]), low2(q[e])) : p[e], sy[e], w[e]);
              v[e] = mul2(v[e], ff);
              w[e] = mul2(w[e], ff);
            }
            x[u] = pack_piece<T>(v);
            y[u] = pack_piece<T>(w);
          }
          uint4* to = reinterpret_cast<uint4*>(dst + (h0 + u * subs + sub) * dst_hs);
          if (live[u] && has_a) to[pa] = x[u];
          if (live[u] && has_b) to[pb] = y[u];
        }
      }
    }
  } else {
    for (int h0 = 0; h0 < a.Hq + (ROWS ? 1 : 2) * a.Hk; h0 += subs) {
      const int h = h0 + sub, kind = h < a.Hq ? 0 : h < a.Hq + a.Hk ? 1 : 2, hk = h - a.Hq - (kind == 2 ? a.Hk : 0);
      const bool live = token_in && h < a.Hq + (ROWS ? 1 : 2) * a.Hk && (kind == 0 || ROWS || at >= 0);
      const T* src = kind == 0   ? reinterpret_cast<const T*>(a.q) + token * a.q_ts + h * a.q_hs
                     : kind == 1 ? reinterpret_cast<const T*>(a.k) + token * a.k_ts + hk * a.k_hs
                                 : reinterpret_cast<const T*>(a.v) + token * a.v_ts + hk * a.v_hs;
      T* dst = kind == 0 ? reinterpret_cast<T*>(a.q_out) + token * a.o_ts + h * a.o_hs
               : ROWS    ? reinterpret_cast<T*>(a.k_out) + token * a.ko_ts + hk * a.ko_hs
                         : reinterpret_cast<T*>(kind == 1 ? a.cache.k : a.cache.v) + at + hk * a.cache.head_stride;
      const T* g = reinterpret_cast<const T*>(kind == 0 ? a.q_gain : kind == 1 ? a.k_gain : nullptr);
      float s = 0.f;
      if (live && g)
        for (int i = lane; i < a.D; i += lanes) {
          const float x = Pack<T>::get(src[i]);
          s = fmaf(x, x, s);
        }
      const float f = rsqrtf(row_sum(s, lanes) * a.inv_d + a.eps);
      if (!live) continue;                                // (no warp-wide step follows in this turn)
      auto value = [&](int i) { return g ? Pack<T>::get(src[i]) * f * Pack<T>::get(g[i]) : Pack<T>::get(src[i]); };
      const int pairs = kind < 2 ? a.pairs : 0;
      for (int i = lane; i < pairs; i += lanes) {
        const int i0 = INTERLEAVED ? 2 * i : i, i1 = INTERLEAVED ? 2 * i + 1 : i + a.pairs;
        const float x = value(i0), y = value(i1);
        dst[i0] = Pack<T>::put(x * cs[i].x - y * cs[i].y);
        dst[i1] = Pack<T>::put(y * cs[i].x + x * cs[i].y);
      }
      for (int i = 2 * pairs + lane; i < a.D; i += lanes) dst[i] = g ? Pack<T>::put(value(i)) : src[i];
    }
  }
}

}  // namespace atts
