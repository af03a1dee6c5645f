// Attention of drafted tokens over a paged cache, and attention weight per cached slot.
#pragma once
#include <math.h>

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
  CacheView cache;
};

// What a drafted token sees: the cached slots below ctx, and the drafted tokens j with lo(j) <= mine < hi(j).
struct SeqView {
  int first, n, ctx, len;
};
__device__ __forceinline__ bool seq_view(const int32_t* cu, const int32_t* ctx, int seq, int M, int max_tokens, int max_len,
                                         SeqView& s, unsigned* dev_status, bool record) {
  bool ok = seq_rows(cu, seq, M, s.first, s.n);
  s.ctx = ctx[seq];
  ok = ok && s.ctx >= 0 && s.n <= max_tokens;
  s.len = ok ? s.ctx + s.n : 0;
  if (record && (!ok || s.len > max_len)) atomicOr(dev_status, kDevSeqRange);
  s.len = min(s.len, max_len);
  return ok;
}

// One warp per (token, query head); lanes share the channels.
template <typename T, int D>
__global__ void __launch_bounds__(256)
tree_attention_simple_kernel(const AttnArgs a, unsigned* __restrict__ dev_status) {
  const int seq = blockIdx.z;
  SeqView s;
  if (!seq_view(a.cu, a.ctx, seq, a.M, a.max_tokens, a.max_len, s, dev_status, threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0)) return;
  const int t = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31, h = blockIdx.y;
  if (t >= s.n) return;
  const int64_t token = s.first + t;
  const int mine = a.pre ? a.pre[token] : t;
  constexpr int E = D / 32;
  float q[E], o[E], m = -INFINITY, l = 0.f;
  for (int e = 0; e < E; ++e) {
    q[e] = Pack<T>::get(reinterpret_cast<const T*>(a.q)[token * a.q_ts + h * a.q_hs + lane * E + e]);
    o[e] = 0.f;
  }
  for (int slot = 0; slot < s.len && mine >= 0; ++slot) {
    if (slot >= s.ctx) {
      const int j = slot - s.ctx;
      const bool see = a.pre ? (a.pre[s.first + j] >= 0 && a.pre[s.first + j] <= mine && mine < a.end[s.first + j]) : j <= t;
      if (!see) continue;
    }
    const int page = cache_page(a.cache, seq, slot, dev_status);
    float x = 0.f, v[E];
    for (int e = 0; e < E; ++e) v[e] = 0.f;
    if (page >= 0) {
      const int64_t at = cache_offset(a.cache, page, slot) + (h / a.G) * a.cache.head_stride + lane * E;
      for (int e = 0; e < E; ++e) {
        x += q[e] * Pack<T>::get(reinterpret_cast<const T*>(a.cache.k)[at + e]);
        v[e] = Pack<T>::get(reinterpret_cast<const T*>(a.cache.v)[at + e]);
      }
    }
    for (int i = 16; i > 0; i >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, i);
    x *= a.scale;
    const float mn = fmaxf(m, x), keep = expf(m - mn), p = expf(x - mn);
    l = l * keep + p;
    for (int e = 0; e < E; ++e) o[e] = o[e] * keep + p * v[e];
    m = mn;
  }
  for (int e = 0; e < E; ++e)
    reinterpret_cast<T*>(a.out)[token * a.o_ts + h * a.o_hs + lane * E + e] = Pack<T>::put(l > 0.f ? o[e] / l : 0.f);
  if (a.lse && lane == 0) a.lse[token * a.Hq + h] = l > 0.f ? m + logf(l) : -INFINITY;
}

struct WeightArgs {
  const char* q;
  const float* lse;
  int64_t q_ts, q_hs;
  const int32_t *ctx, *cu, *pre, *end;
  int M, Hq, G, max_tokens, max_len;
  float scale;
  const float* win;
  float* wout;
  int64_t wcols;
  CacheView cache;
};

// One warp per (slot, key head).
template <typename T, int D>
__global__ void __launch_bounds__(256)
cache_weights_simple_kernel(const WeightArgs a, unsigned* __restrict__ dev_status) {
  const int seq = blockIdx.z;
  SeqView s;
  const bool ok = seq_view(a.cu, a.ctx, seq, a.M, a.max_tokens, a.max_len, s, dev_status, threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0);
  const int slot = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31, hk = blockIdx.y;
  if (slot >= a.max_len) return;
  const int64_t at_w = ((int64_t)seq * a.cache.heads + hk) * a.wcols + slot;
  if (!ok || slot >= s.len) {
    if (lane == 0) a.wout[at_w] = 0.f;
    return;
  }
  constexpr int E = D / 32;
  const int page = cache_page(a.cache, seq, slot, dev_status);
  float k[E], sum = 0.f;
  for (int e = 0; e < E; ++e) k[e] = 0.f;
  if (page >= 0) {
    const int64_t at = cache_offset(a.cache, page, slot) + hk * a.cache.head_stride + lane * E;
    for (int e = 0; e < E; ++e) k[e] = Pack<T>::get(reinterpret_cast<const T*>(a.cache.k)[at + e]);
  }
  const int j = slot - s.ctx;
  const int lo = j < 0 ? 0 : a.pre ? a.pre[s.first + j] : j, hi = j < 0 ? 0x7FFFFFFF : a.pre ? a.end[s.first + j] : 0x7FFFFFFF;
  for (int t = 0; t < s.n; ++t) {
    const int64_t token = s.first + t;
    const int mine = a.pre ? a.pre[token] : t;
    if (mine < 0 || lo < 0 || mine < lo || mine >= hi) continue;
    for (int g = hk * a.G; g < (hk + 1) * a.G; ++g) {
      float x = 0.f;
      for (int e = 0; e < E; ++e) x += k[e] * Pack<T>::get(reinterpret_cast<const T*>(a.q)[token * a.q_ts + g * a.q_hs + lane * E + e]);
      for (int i = 16; i > 0; i >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, i);
      sum += expf(x * a.scale - a.lse[token * a.Hq + g]);
    }
  }
  if (lane == 0) a.wout[at_w] = (a.win ? a.win[at_w] : 0.f) + sum;
}

}  // namespace atts
