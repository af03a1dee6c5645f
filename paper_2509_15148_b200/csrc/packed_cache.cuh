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

// Scale's byte of a group whose largest magnitude is `top`: max / 7 to fp16, then to three fraction bits, to nearest even both
// times.  (The fp32 product by 1 / 7 is off by 2^-23 of itself at most, max / 7, with 11 bits of max, by 2^-15 from where fp16 would
// round the other way, unless it is an fp16 number itself: the first rounding is that of the quotient.)
__device__ __forceinline__ uint32_t packed_scale_byte(float top) {
  if (!(top < INFINITY)) return 255u;
  const uint32_t h = __half_as_ushort(__float2half_rn(fminf(top * (1.f / 7.f), kPackedMaxScale)));
  return (h + 63u + ((h >> 7) & 1u)) >> 7;
}
__device__ __forceinline__ float packed_scale(uint32_t byte) { return __half2float(__ushort_as_half((unsigned short)(byte << 7))); }

// The word of eight channels under their group's scale (inverse: 1 / s, 0 for no scale); |x / s| at most 15.  x / s to the nearest whole
// number, ties to even: x * (1 / s) is off by 2^-20 at most, while x / s, a quotient of 11 and 4 bits, is a tie or 2^-13 away from one,
// so 48 + x / s goes to a multiple of 2^-18 first, which makes a tie a tie again, and then to 1.5 * 2^23 + 8 + c, whose low bits are
// c + 8.  The upper bits of the eight, shifted alike, are a constant that the last step takes off.
__device__ __forceinline__ uint32_t packed_word(const float (&x)[8], float inverse) {
  uint32_t w = 0;
  constexpr uint32_t kUpper = 0x4B400000u;
  constexpr uint32_t kTaken = kUpper * (0x1111u + 0x11110000u);
#pragma unroll
  for (int j = 0; j < 8; ++j) w += __float_as_uint(__fadd_rn(fmaf(x[j], inverse, 48.f), 12582920.f - 48.f)) << (4 * (j / 2) + 16 * (j % 2));
  return w - kTaken;
}

// (x * s) in two 16-bit halves, exact: v = 16 + n in the top four fraction bits of each half, n = c + 8, and v s - 24 s = c s.
template <typename T>
struct Expand;
template <>
struct Expand<__nv_bfloat16> {
  static constexpr uint32_t kMask = 0x00780078u, kSixteen = 0x41804180u;
  static constexpr int kShift = 3;      // nibble 0 to the top of the fraction
  static __device__ __forceinline__ void scale(float a, float b, uint32_t& s2, uint32_t& m2) {   // of the low and the high half
    s2 = Pack<__nv_bfloat16>::pack(a, b);
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(m2) : "r"(s2), "r"(0xC1C0C1C0u));
  }
  static __device__ __forceinline__ uint32_t fma2(uint32_t v, uint32_t s, uint32_t m) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(v), "r"(s), "r"(m));
    return r;
  }
};
template <>
struct Expand<__half> {
  static constexpr uint32_t kMask = 0x03C003C0u, kSixteen = 0x4C004C00u;
  static constexpr int kShift = 6;
  static __device__ __forceinline__ void scale(float a, float b, uint32_t& s2, uint32_t& m2) {   // of the low and the high half
    s2 = Pack<__half>::pack(a, b);
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(m2) : "r"(s2), "r"(0xCE00CE00u));
  }
  static __device__ __forceinline__ uint32_t fma2(uint32_t v, uint32_t s, uint32_t m) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(v), "r"(s), "r"(m));
    return r;
  }
};
template <typename T, int I>
__device__ __forceinline__ uint32_t expand_pair(uint32_t word, uint32_t s2, uint32_t m2) {
  constexpr int by = Expand<T>::kShift - 4 * I;           // channel pair I sits in bits 4 I and 16 + 4 I
  const uint32_t v = by >= 0 ? word << (by >= 0 ? by : 0) : word >> (by < 0 ? -by : 0);
  uint32_t x;   // (v & mask) | sixteen in one instruction: from C it becomes two, each with a constant of its own (60.6 against 54.8 us)
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(x) : "r"(v), "r"(Expand<T>::kMask), "r"(Expand<T>::kSixteen));
  return Expand<T>::fma2(x, s2, m2);
}

// ------------------------------------------------------------------------------------------------------------------
// Append.  A thread takes eight channels of a key and the same of a value, four threads a group; loads of 16 bytes and stores of 4
// are contiguous over a warp; it keeps its head and channels and goes over tokens, two of them on their way.  Bound: the arithmetic
// of the codes before HBM (2 D bytes of a row in, D / 2 + D / 32 out): 12,675 tokens of 8 heads of 128 22.7 us = 2.9 TB/s, 0.44 of a plain
// copy, with issue slots 60 % and DRAM 26 % busy.  (The first form, a division of indexes, a clamp and a comparison for every channel,
// took 50 us with the read-back, this one 36.)
// ------------------------------------------------------------------------------------------------------------------
constexpr int kPackThreads = 256, kPackMaxTokens = 32;

struct PackArgs {
  const char *k, *v;
  int64_t k_ts, k_hs, v_ts, v_hs;  // elements
  const int32_t *ctx, *cu;
  int D, M, tpb, max_tokens;
  CacheView cache;                 // strides in bytes, no slot stride
};

template <typename T, bool WIDE>
__device__ __forceinline__ void load_eight(const T* src, uint32_t (&w)[4]) {
  if (WIDE) {
    const uint4 u = *reinterpret_cast<const uint4*>(src);
    w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
  } else {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(src);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (uint32_t)p[2 * e] | ((uint32_t)p[2 * e + 1] << 16);
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
  // A thread keeps its head and channels (u) and goes over tokens; a group's four threads go together.
  const int per_row = a.D / 8, per_token = a.cache.heads * per_row;
  const int side = min(per_token, kPackThreads), tokens = kPackThreads / side, t_first = threadIdx.x / side;
  if (t_first >= tokens) return;
  const unsigned quad = 0xFu << (threadIdx.x & 28);
  for (int u = threadIdx.x - t_first * side; u < per_token; u += side) {
    const int head = u / per_row, c8 = u - head * per_row;
    const T* k = reinterpret_cast<const T*>(a.k) + (int64_t)(first + t0) * a.k_ts + head * a.k_hs + 8 * c8;
    const T* v = reinterpret_cast<const T*>(a.v) + (int64_t)(first + t0) * a.v_ts + head * a.v_hs + 8 * c8;
    for (int t = t_first; t < nt; t += 2 * tokens) {     // two tokens' loads on their way together
      uint32_t x[2][2][4];
#pragma unroll
      for (int w = 0; w < 2; ++w)
        if (t + w * tokens < nt) {
          load_eight<T, WIDE>(k + (t + w * tokens) * a.k_ts, x[w][0]);
          load_eight<T, WIDE>(v + (t + w * tokens) * a.v_ts, x[w][1]);
        }
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const int tt = t + w * tokens;
        if (tt >= nt || page_at[tt] < 0) continue;       // (all four threads of a group)
        const int codes = packed_codes(entry_at[tt], a.D) + 4 * c8, scales = packed_scales(entry_at[tt], a.D) + c8 / 4;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t tops = 0;                             // magnitudes compare as their bits do, NaN above all: two at a time
#pragma unroll
          for (int e = 0; e < 4; ++e) tops = __vmaxu2(tops, x[w][i][e] & 0x7FFF7FFFu);
          tops = __vmaxu2(tops, __shfl_xor_sync(quad, tops, 1));
          tops = __vmaxu2(tops, __shfl_xor_sync(quad, tops, 2));
          const uint32_t byte = packed_scale_byte(Pack<T>::unpack(max(tops & 0xFFFFu, tops >> 16)).x);
          const float s = packed_scale(byte);
          uint32_t word = 0x88888888u;
          if (byte != 255u) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = Pack<T>::unpack(x[w][i][e]);
              y[2 * e] = f.x;
              y[2 * e + 1] = f.y;
            }
            // A scale is max / 7 to 1 / 16 of itself, so no quotient passes 7.5, unless the scale is the largest or below 2^-14.
            if (byte < 8u || s == kPackedMaxScale)
#pragma unroll
              for (int e = 0; e < 8; ++e) y[e] = fminf(fmaxf(y[e], -7.f * s), 7.f * s);
            word = packed_word(y, s > 0.f ? 1.f / s : 0.f);
          }
          char* base = (i ? a.cache.v : a.cache.k) + page_at[tt] + head * a.cache.head_stride;
          *reinterpret_cast<uint32_t*>(base + codes) = word;
          if ((c8 & 3) == 0) base[scales] = (char)byte;
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Reading back: slots [0, lens[b]) of every sequence into a cache in 16 bits.  The same shape as the append, the other way round; codes
// expand as for the products.  Bound: latency and instructions of small accesses (a thread loads 4 bytes of codes and one of a scale at a
// time; issue slots 52 %, ALU 43 %): 12,694 slots of 8 heads of 128 14.6 us = 4.5 TB/s, 0.69 of a plain copy.
// ------------------------------------------------------------------------------------------------------------------
struct ReadArgs {
  const int32_t* lens;
  int D, tpb, max_len;
  CacheView src, dst;              // src: strides in bytes, no slot stride
};

template <typename T>
__device__ __forceinline__ uint4 packed_values(uint32_t word, float s) {
  uint32_t s2, m2;
  Expand<T>::scale(s, s, s2, m2);
  return make_uint4(expand_pair<T, 0>(word, s2, m2), expand_pair<T, 1>(word, s2, m2), expand_pair<T, 2>(word, s2, m2), expand_pair<T, 3>(word, s2, m2));
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
  const int side = min(per_token, kPackThreads), slots = kPackThreads / side, t_first = threadIdx.x / side;
  if (t_first >= slots) return;
  for (int u = threadIdx.x - t_first * side; u < per_token; u += side) {
    const int head = u / per_row, c8 = u - head * per_row;
    const int64_t src_head = head * a.src.head_stride, dst_at = head * a.dst.head_stride + 8 * c8;
    for (int t = t_first; t < n; t += 2 * slots) {       // two slots' loads on their way together
      uint32_t word[2][2], byte[2][2];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const int tt = t + w * slots;
        if (tt >= n || from[tt] < 0) continue;
        const int entry = (s0 + tt) & ((1 << a.src.page_log2) - 1);
        const int64_t at = from[tt] + src_head;
        const int codes = packed_codes(entry, a.D) + 4 * c8, scales = packed_scales(entry, a.D) + c8 / 4;
        word[w][0] = *reinterpret_cast<const uint32_t*>(a.src.k + at + codes);
        word[w][1] = *reinterpret_cast<const uint32_t*>(a.src.v + at + codes);
        byte[w][0] = *reinterpret_cast<const uint8_t*>(a.src.k + at + scales);
        byte[w][1] = *reinterpret_cast<const uint8_t*>(a.src.v + at + scales);
      }
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const int tt = t + w * slots;
        if (tt >= n || from[tt] < 0) continue;
        *reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.dst.k) + to[tt] + dst_at) = packed_values<T>(word[w][0], packed_scale(byte[w][0]));
        *reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.dst.v) + to[tt] + dst_at) = packed_values<T>(word[w][1], packed_scale(byte[w][1]));
      }
    }
  }
}

}  // namespace atts
