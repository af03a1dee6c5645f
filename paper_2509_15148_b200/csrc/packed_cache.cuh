// A paged cache that holds keys and values in 4 bits: its layout, the append that writes it (atts_packed_append) and the call that
// reads it back (atts_packed_read).
#pragma once
#include "rope_cache.cuh"

namespace atts {

// ------------------------------------------------------------------------------------------------------------------
// 32 neighbouring channels of a slot share a scale s, one byte of five exponent and three fraction bits (the upper bits of an fp16
// number behind its sign: byte << 7 is s in fp16; 0xFF is NaN); a channel is c * s with a whole c of -7 .. 7.  Both have few
// enough bits that c * s is exact in bf16 (4 + 3 significant bits of 8) and in fp16 (down to 2^-17, its scales' smallest), so
// whoever multiplies by it on the tensor cores rounds nothing: s at most 2048 keeps 24 s, which appears on the way, within fp16.
//
// A page of a head is laid out by eights of slots: the codes of eight slots, D / 2 bytes each, then their scales, D / 32 bytes
// each.  Any eights of a page are therefore one contiguous piece (a multiple of 16 bytes) that one bulk copy moves.  A code is
// held as c + 8; eight channels share a 32-bit word, channel 2 i in bits 4 i and channel 2 i + 1 in bits 16 + 4 i: a shift and a
// mask leave neighbours in the two halves of a register, where 16-bit pairs need them.
// ------------------------------------------------------------------------------------------------------------------
constexpr float kPackedMaxScale = 2048.f;
__host__ __device__ constexpr int packed_eight(int D) { return 4 * D + D / 4; }   // bytes of eight slots

// Byte offsets of a slot's codes and scales within its page of a head.
__device__ __forceinline__ int packed_codes(int entry, int D) { return (entry >> 3) * packed_eight(D) + (entry & 7) * (D / 2); }
__device__ __forceinline__ int packed_scales(int entry, int D) { return (entry >> 3) * packed_eight(D) + 4 * D + (entry & 7) * (D / 32); }

// Scale's byte of a group whose largest magnitude has these bits (sign cleared): max / 7 to fp16, then to three fraction bits,
// to nearest even both times.  (The fp32 product by 1 / 7 is off by 2^-23 of itself at most, max / 7, with 11 bits of max, by 2^-15
// from where fp16 would round the other way, unless it is an fp16 number itself: the first rounding is that of the quotient.)
__device__ __forceinline__ uint32_t packed_scale_byte(uint32_t top) {
  if (top >= 0x7F800000u) return 255u;
  const uint32_t h = __half_as_ushort(__float2half_rn(fminf(__uint_as_float(top) * (1.f / 7.f), kPackedMaxScale)));
  return (h + 63u + ((h >> 7) & 1u)) >> 7;
}
__device__ __forceinline__ float packed_scale(uint32_t byte) { return __half2float(__ushort_as_half((unsigned short)(byte << 7))); }

// The word of eight channels under their group's scale (inverse: 1 / s, 0 for no scale).  x / s to the nearest whole number, ties to
// even: x * (1 / s) is off by 2^-20 at most, while x / s, a quotient of 11 and 4 bits, is a tie or 2^-13 away from one, so the
// product goes to a multiple of 2^-18 first, which makes a tie a tie again.
__device__ __forceinline__ uint32_t packed_word(const float (&x)[8], float inverse) {
  uint32_t w = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float c = __fsub_rn(__fadd_rn(x[j] * inverse, 48.f), 48.f);
    c = fminf(fmaxf(c, -7.f), 7.f);
    const uint32_t whole = __float_as_uint(__fadd_rn(c, 12582920.f));   // 1.5 * 2^23 + 8: the low bits are c + 8
    w |= (whole & 15u) << (4 * (j / 2) + 16 * (j % 2));
  }
  return w;
}

// ------------------------------------------------------------------------------------------------------------------
// Append.  A thread takes eight channels of a key and the same of a value, four threads a group; loads of 16 bytes and stores of 4
// are contiguous over a warp.  Bound: HBM (2 D bytes of a row in, D / 2 + D / 32 out).
// ------------------------------------------------------------------------------------------------------------------
constexpr int kPackThreads = 256, kPackMaxTokens = 16;

struct PackArgs {
  const char *k, *v;
  int64_t k_ts, k_hs, v_ts, v_hs;  // elements
  const int32_t *ctx, *cu;
  int D, M, tpb, max_tokens;
  CacheView cache;                 // strides in bytes, no slot stride
};

template <typename T, bool WIDE>
__device__ __forceinline__ void load_eight(const T* src, float (&x)[8]) {
  if (WIDE) {
    const uint4 w = *reinterpret_cast<const uint4*>(src);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = Pack<T>::unpack(u[e]);
      x[2 * e] = f.x;
      x[2 * e + 1] = f.y;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = Pack<T>::get(src[e]);
  }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(kPackThreads)
packed_append_kernel(const __grid_constant__ PackArgs a, unsigned* __restrict__ dev_status) {
  __shared__ int64_t page_at[kPackMaxTokens];    // byte offset of a token's page, -1: none
  __shared__ int entry_at[kPackMaxTokens];
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
  if (threadIdx.x < nt) {
    const int slot = ctx + t0 + threadIdx.x;
    const int page = cache_page(a.cache, seq, slot, dev_status);
    page_at[threadIdx.x] = page < 0 ? -1 : (int64_t)page * a.cache.page_stride;
    entry_at[threadIdx.x] = slot & ((1 << a.cache.page_log2) - 1);
  }
  __syncthreads();
  const int per_row = a.D / 8, per_token = a.cache.heads * per_row;
  const int total = nt * per_token;              // a multiple of 4: a group's four threads are in it or not together
  for (int e0 = 0; e0 < total; e0 += kPackThreads) {
    const int e = e0 + threadIdx.x;
    const bool in = e < total;
    const int t = in ? e / per_token : 0, u = in ? e - t * per_token : 0;
    const int head = u / per_row, c8 = u - head * per_row;
    const int64_t token = first + t0 + t;
    const bool live = in && page_at[t] >= 0;
    float x[2][8] = {};
    if (live) {
      load_eight<T, WIDE>(reinterpret_cast<const T*>(a.k) + token * a.k_ts + head * a.k_hs + 8 * c8, x[0]);
      load_eight<T, WIDE>(reinterpret_cast<const T*>(a.v) + token * a.v_ts + head * a.v_hs + 8 * c8, x[1]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t top = 0;                          // magnitudes compare as their bits do, NaN above all
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[i][j]) & 0x7FFFFFFFu);
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      if (!live) continue;
      const uint32_t byte = packed_scale_byte(top);
      const float s = packed_scale(byte);
      uint32_t word = 0x88888888u;
      if (byte != 255u) word = packed_word(x[i], s > 0.f ? 1.f / s : 0.f);
      char* base = (i ? a.cache.v : a.cache.k) + page_at[t] + head * a.cache.head_stride;
      *reinterpret_cast<uint32_t*>(base + packed_codes(entry_at[t], a.D) + 4 * c8) = word;
      if ((c8 & 3) == 0) base[packed_scales(entry_at[t], a.D) + c8 / 4] = (char)byte;
    }
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Reading back: slots [0, lens[b]) of every sequence into a cache in 16 bits.  The same shape as the append, the other way round.
// ------------------------------------------------------------------------------------------------------------------
struct ReadArgs {
  const int32_t* lens;
  int D, tpb, max_len;
  CacheView src, dst;              // src: strides in bytes, no slot stride
};

template <typename T>
__device__ __forceinline__ uint4 packed_values(uint32_t word, float s) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = Pack<T>::pack((float)((int)((word >> (4 * i)) & 15u) - 8) * s, (float)((int)((word >> (16 + 4 * i)) & 15u) - 8) * s);
  return make_uint4(r[0], r[1], r[2], r[3]);
}

template <typename T>
__global__ void __launch_bounds__(kPackThreads)
packed_read_kernel(const __grid_constant__ ReadArgs a, unsigned* __restrict__ dev_status) {
  __shared__ int64_t from[kPackMaxTokens], to[kPackMaxTokens];   // byte offset of a slot's page in src, element offset in dst; -1: none
  pdl_wait();
  pdl_launch_dependents();
  const int seq = blockIdx.y;
  const int len0 = a.lens[seq], len = max(0, min(len0, a.max_len));
  if (len != len0 && threadIdx.x == 0 && blockIdx.x == 0) atomicOr(dev_status, kDevSeqRange);
  const int s0 = blockIdx.x * a.tpb;
  if (s0 >= len) return;
  const int n = min(a.tpb, len - s0);
  if (threadIdx.x < n) {
    const int slot = s0 + threadIdx.x;
    const int p = cache_page(a.src, seq, slot, dev_status), q = cache_page(a.dst, seq, slot, dev_status);
    from[threadIdx.x] = p < 0 || q < 0 ? -1 : (int64_t)p * a.src.page_stride;
    to[threadIdx.x] = q < 0 ? -1 : cache_offset(a.dst, q, slot);
  }
  __syncthreads();
  const int per_row = a.D / 8, per_token = a.src.heads * per_row;
  for (int e = threadIdx.x; e < n * per_token; e += kPackThreads) {
    const int t = e / per_token, u = e - t * per_token;
    const int head = u / per_row, c8 = u - head * per_row;
    if (from[t] < 0) continue;
    const int entry = (s0 + t) & ((1 << a.src.page_log2) - 1);
    const int codes = packed_codes(entry, a.D) + 4 * c8, scales = packed_scales(entry, a.D) + c8 / 4;
    const char* k = a.src.k + from[t] + head * a.src.head_stride;
    const char* v = a.src.v + from[t] + head * a.src.head_stride;
    const uint32_t kw = *reinterpret_cast<const uint32_t*>(k + codes), vw = *reinterpret_cast<const uint32_t*>(v + codes);
    const uint32_t kb = (uint8_t)k[scales], vb = (uint8_t)v[scales];
    const int64_t at = to[t] + head * a.dst.head_stride + 8 * c8;
    *reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.dst.k) + at) = packed_values<T>(kw, packed_scale(kb));
    *reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.dst.v) + at) = packed_values<T>(vw, packed_scale(vb));
  }
}

}  // namespace atts
