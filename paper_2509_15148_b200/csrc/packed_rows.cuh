// Attention of few rows over a packed cache: the single tokens and small trees of a serving step.
#pragma once
#include "tree_attention.cuh"

namespace atts {

// ------------------------------------------------------------------------------------------------------------------
// At most 16 rows: the products are small, and what costs is bringing the codes in and expanding them.  tree_attention_kernel expands
// through shared memory, because its products read both operands there, and computes 128 rows whatever their number.  Here a thread
// expands the codes in registers, in just the order in which the warp-level product (16 x 8 x 16) takes its first operand, and
// nothing is written back:
//   S^T = K Q^T   16 slots x 8 rows a product: a thread's 8 bytes (D = 64) or 16 bytes of a slot's codes are the channels of its K operands;
//                 which channels a step of the product takes is free as long as Q's operand is laid out alike (once, in shared memory).
//   O^T += V^T P^T  pairs of neighbouring slots of one channel: the halves of two slots' words change places (two byte permutations a
//                 pair of words), then they expand as K's do, each half under its own slot's scale.  P^T comes out of S^T's registers, two
//                 8 x 8 transposes for 16 slots and 8 rows.
// The warps take turns at loading: warp t % 8 brings tile t, two tiles after the one that had its place was used up, so that it hardly
// ever waits for the others.  Every warp goes over its own slots of each tile (32 with up to 8 rows, where two sets of warps then take
// turns at tiles, 56 against 59.5 us; 16 beyond, whose sums need the registers) with its own maxima and sums; they are joined at the
// end through shared memory, and over CTAs by attention_parts_join_kernel.  The running maximum is a warp's and moves when a row
// passes it by 2^8, as in tree_attention_kernel; so do the rounding of probabilities and everything that masks.
// Bound: instructions.  16 slots of 128 channels are 402, of which 64 channel pairs of a shift (16 lanes a clock and scheduler), a mask
// (16) and a multiply-add (16), and 16 products (8.2 cycles of the tensor pipe each): 804 issue slots a scheduler and tile, where
// an SM with two CTAs takes about 1,200 cycles.  4 sequences of 20,000 to 32,768 slots, 8 key heads of 128 (17 us at HBM's rate): 8 rows
// 47 us, 16 rows 63 (tree_attention_kernel 114 and 118, and from 24 rows on 88 to 98, where a form for 32 rows here took 105).
// Loads placed a step ahead of their products: 60 against 49 us (more instructions, and latency is covered by the four warps of a
// scheduler as it is); constants of the mask out of shared memory, products that the compiler may move: no difference.
// ------------------------------------------------------------------------------------------------------------------
constexpr int kFewWarps = 8, kFewThreads = 32 * kFewWarps, kFewMaxRows = 16;

template <int D, int NT>      // NT tiles of 8 rows
struct FewCfg {
  static constexpr int kUnits = NT == 1 ? 2 : 1;                               // 16 slots each, of a warp in a tile
  static constexpr int kSets = kUnits, kSetWarps = kFewWarps / kSets;          // warps that share a tile; sets take turns
  static constexpr int kRaw = kAttnTile / 8 * packed_eight(D);                 // keys or values of a tile
  static constexpr int kStages = D == 128 ? 6 : 12;
  static constexpr int kAhead = kStages - 2;                                   // tiles loaded ahead of the one in use
  static constexpr int kQ = kStages * 2 * kRaw;                                // [NT][D / 16][32] uint2
  static constexpr int kStats = kQ + 8 * NT * D * 2;                           // [warps][8 NT] float2
  static constexpr int kBars = kStats + kFewWarps * 8 * NT * 8;
  static constexpr int kSmemBytes = kBars + 16 * kStages + 16;
  static_assert(kStages * 2 * kRaw >= kFewWarps * 8 * NT * D * 4, "the warps' sums are joined through the ring");
  static_assert(kAhead % kSets == 0 && 2 * (kSmemBytes + 1024) <= 233472, "a set loads for itself; two CTAs an SM");
};

template <typename T>
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma_16816<__nv_bfloat16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma_16816<__half>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
// Slot of row k of a product's 16: the two of every odd pair exchanged, so that a keys' load hits every bank once and a values' load,
// whose four slots are two rows of 64 bytes apart, each bank twice instead of four times.
__device__ __forceinline__ int few_slot(int k) { return k ^ ((k >> 1) & 1); }

template <int WORDS>
__device__ __forceinline__ void load_words(uint32_t (&w)[WORDS], uint32_t at) {
  if constexpr (WORDS == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
  else if constexpr (WORDS == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
  else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at));
}
__device__ __forceinline__ uint32_t load_byte(uint32_t at) {
  uint32_t r;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(r) : "r"(at));
  return r;
}
template <typename T>
__device__ __forceinline__ uint32_t expand_any(uint32_t word, int i, uint32_t s2, uint32_t m2) {   // i a constant once unrolled
  return i == 0 ? expand_pair<T, 0>(word, s2, m2) : i == 1 ? expand_pair<T, 1>(word, s2, m2) : i == 2 ? expand_pair<T, 2>(word, s2, m2) : expand_pair<T, 3>(word, s2, m2);
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kFewThreads, 2)
packed_rows_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ AttnPlan plan, unsigned* __restrict__ dev_status) {
  using Cfg = FewCfg<D, NT>;
  constexpr int kSteps = D / 16, kStages = Cfg::kStages, kUnits = Cfg::kUnits, kSets = Cfg::kSets, kSetWarps = Cfg::kSetWarps;
  extern __shared__ __align__(128) uint8_t few_smem[];
  const int seq = blockIdx.z, hk = blockIdx.y, chunk = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  SeqView s;
  if (!seq_view(a.cu, a.ctx, seq, a.M, a.max_tokens, a.max_len, s, dev_status, threadIdx.x == 0 && chunk == 0 && hk == 0)) return;
  if (s.n == 0) return;
  const int rows = s.n * a.G;                              // <= 8 NT: max_tokens bounds them
  int ntiles = (s.len + kAttnTile - 1) / kAttnTile;
  const WindowView win = window_view(a, s, 0, s.n, ntiles, lane);
  const int tree0 = min(s.ctx, s.len) / kAttnTile;         // first tile that is not all cached slots
  ntiles = win.live ? ntiles - win.skip : 0;               // padding alone sees nothing: no page is looked up
  const int tile0 = chunk * plan.chunk, tile1 = min(ntiles, tile0 + plan.chunk);
  const int64_t row0 = (int64_t)s.first * a.Hq + hk * a.G;
  auto row_of = [&](int r) { return row0 + (int64_t)(r / a.G) * a.Hq + r % a.G; };
  if (chunk > 0 && tile0 >= ntiles) {
    for (int r = threadIdx.x; r < rows; r += kFewThreads) plan.part_lse[row_of(r) * plan.chunks + chunk] = -INFINITY;
    return;
  }
  const int ntile = tile1 - tile0;
  const uint32_t base = smem_u32(few_smem);
  float2* stats = reinterpret_cast<float2*>(few_smem + Cfg::kStats);
  auto full_bar = [&](int i) { return base + Cfg::kBars + 16u * (uint32_t)i; };
  auto empty_bar = [&](int i) { return base + Cfg::kBars + 16u * (uint32_t)i + 8u; };
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(few_smem + Cfg::kBars + 16 * kStages);
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(full_bar(i), 1);
      mbar_init(empty_bar(i), kSetWarps);
    }
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // Q in the order of the products' second operand: step t, thread (row lane / 4, quarter lane % 4) has channels D / 4 * quarter + 4 t ..
  uint2* qf = reinterpret_cast<uint2*>(few_smem + Cfg::kQ);
  for (int e = threadIdx.x; e < NT * kSteps * 32; e += kFewThreads) {
    const int l = e & 31, t = (e >> 5) % kSteps, r = (e >> 5) / kSteps * 8 + l / 4;
    uint2 w = make_uint2(0, 0);
    if (r < rows)
      w = *reinterpret_cast<const uint2*>(a.q + 2 * ((int64_t)(s.first + r / a.G) * a.q_ts + (int64_t)(hk * a.G + r % a.G) * a.q_hs + D / 4 * (l & 3) + 4 * t));
    qf[e] = w;
  }
  __syncthreads();
  pdl_launch_dependents();
  const long long limit = plan.wait_limit;
  auto wait_warp = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort_flag, limit, 0u)) != 0; };

  float o[D / 16][NT][4];                                  // channel tile, row tile
  float m[NT][2], l[NT][2];                                // of this thread's rows (lane % 4) * 2, + 1; l of its own slots
  float off[NT][2], bound[NT][2];                          // what p's exponent adds to c x; scores above the bound move the maximum
  const float c = a.scale * 1.4426950408889634f;
  const int n = lane >> 2, j = lane & 3;
  const int set = warp % kSets, member = warp / kSets;     // this warp's tiles are set, set + kSets, ..
  {
    // ---------------- loads: lanes 0-15 keys, 16-31 values, a page's piece of the tile each ----------------
    const TileBoxes<D, 1> bx(a.cache.page_log2, lane & 15);
    const bool value = lane >= 16, mine = (lane & 15) < bx.boxes;
    const uint32_t bytes = (uint32_t)(bx.rows / 8) * packed_eight(D);
    const char* from = (value ? a.cache.v : a.cache.k) + (int64_t)hk * a.cache.head_stride;
    constexpr int kNoSlot = -2;
    auto look_up = [&](int i) -> int {
      if (i >= ntile || !mine) return kNoSlot;
      const int slot = win.tile(tile0 + i) * kAttnTile + bx.slot;
      if (slot >= s.len || (slot + bx.rows <= min(s.ctx, win.near_first) && slot >= a.sinks)) return kNoSlot;
      const int col = slot >> bx.page_log2;
      return col < a.cache.table_cols ? a.cache.table[(int64_t)seq * a.cache.table_stride + col] : -1;
    };
    int next = warp, entry = look_up(warp);                // the tile that this warp loads next, and the table's entry for it
    auto load_next = [&]() -> bool {
      const int i = next, stage = i % kStages, page = entry >= 0 && entry < a.cache.num_pages ? entry : -1;
      if (page < 0 && entry != kNoSlot) atomicOr(dev_status, kDevPageRange);
      next += kFewWarps;
      entry = look_up(next);
      if (plan.withhold_loads) return true;
      if (!wait_warp(empty_bar(stage), ((uint32_t)(i / kStages) & 1u) ^ 1u)) return false;
      const int slot = win.tile(tile0 + i) * kAttnTile + bx.slot;
      const uint32_t dst = base + (uint32_t)(2 * stage + (value ? 1 : 0)) * Cfg::kRaw + (uint32_t)(bx.slot / 8) * packed_eight(D);
      if (mine && page < 0 && slot < s.len) {              // reads as zeros
        for (uint32_t x = 0; x < bytes; x += 16) asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(dst + x), "r"(0u) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      }
      const uint32_t copies = __popc(__ballot_sync(0xFFFFFFFFu, page >= 0));
      __syncwarp();
      if (lane == 0) mbar_expect_tx(full_bar(stage), copies * bytes);
      __syncwarp();
      if (page >= 0)
        bulk_load(dst, from + (int64_t)page * a.cache.page_stride + (int64_t)((slot & ((1 << bx.page_log2) - 1)) / 8) * packed_eight(D), bytes, full_bar(stage));
      __syncwarp();
      return true;
    };
    bool ok = true;
    while (next < min(ntile, Cfg::kAhead)) load_next();    // (places that nobody has used yet)

    // ---------------- slots ----------------
    constexpr int kKeyWords = D / 32, kValueWords = D / 64;
    const uint2* q_at = qf + lane;
    uint2 q_kept[kSteps];                                  // one row tile's operands stay in registers
    if (NT == 1)
#pragma unroll
      for (int t = 0; t < kSteps; ++t) q_kept[t] = q_at[t * 32];
#pragma unroll
    for (int r = 0; r < NT; ++r) {
      m[r][0] = m[r][1] = bound[r][0] = bound[r][1] = -INFINITY;
      l[r][0] = l[r][1] = 0.f;
      off[r][0] = off[r][1] = AttnType<T>::shift;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) o[i][r][0] = o[i][r][1] = o[i][r][2] = o[i][r][3] = 0.f;
    }
    const int first = 16 * kUnits * member;                // of this warp's slots in a tile
    const uint32_t key_at = (uint32_t)(first / 8 * packed_eight(D) + few_slot(n) * (D / 2) + j * (D / 8));
    const uint32_t key_scale_at = (uint32_t)(first / 8 * packed_eight(D) + 4 * D + few_slot(n) * (D / 32) + j * D / 128);
    for (int i = set; ok && i < ntile; i += kSets) {
      if (next == i + Cfg::kAhead && next < ntile) ok = load_next();
      const int stage = i % kStages;
      ok = ok && wait_warp(full_bar(stage), (uint32_t)(i / kStages) & 1u);
      if (!ok) break;
      const int tile = win.tile(tile0 + i);
      const bool masked = tile >= tree0 || (tile < win.full_from && (tile + 1) * kAttnTile > a.sinks);
      const uint32_t keys = base + (uint32_t)(2 * stage) * Cfg::kRaw, values = keys + Cfg::kRaw;
      const int slot0 = tile * kAttnTile + first;
      if (!(masked && slot0 >= s.len)) {
        float x[kUnits][NT][4];
        {
          uint32_t w0[kUnits][kKeyWords], w1[kUnits][kKeyWords], s0[kUnits], m0[kUnits], s1[kUnits], m1[kUnits];
#pragma unroll
          for (int u = 0; u < kUnits; ++u) {
#pragma unroll
            for (int r = 0; r < NT; ++r) x[u][r][0] = x[u][r][1] = x[u][r][2] = x[u][r][3] = 0.f;
            const uint32_t off = (uint32_t)(2 * u * packed_eight(D));
            load_words(w0[u], keys + key_at + off);
            load_words(w1[u], keys + key_at + off + packed_eight(D));
            const float f0 = packed_scale(load_byte(keys + key_scale_at + off));
            Expand<T>::scale(f0, f0, s0[u], m0[u]);
            const float f1 = packed_scale(load_byte(keys + key_scale_at + off + packed_eight(D)));
            Expand<T>::scale(f1, f1, s1[u], m1[u]);
          }
#pragma unroll
          for (int t = 0; t < kSteps; ++t) {
            const int p = 2 * (t & 1);
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
              const uint32_t a0 = expand_any<T>(w0[u][t / 2], p, s0[u], m0[u]), a2 = expand_any<T>(w0[u][t / 2], p + 1, s0[u], m0[u]);
              const uint32_t a1 = expand_any<T>(w1[u][t / 2], p, s1[u], m1[u]), a3 = expand_any<T>(w1[u][t / 2], p + 1, s1[u], m1[u]);
#pragma unroll
              for (int r = 0; r < NT; ++r) {
                const uint2 b = NT == 1 ? q_kept[t] : q_at[(r * kSteps + t) * 32];
                mma_16816<T>(x[u][r], a0, a1, a2, a3, b.x, b.y);
              }
            }
          }
        }
        uint32_t dead = 0;                                   // of this thread's four slots a unit, as values
        if (masked) {
#pragma unroll
          for (int u = 0; u < kUnits; ++u) {
            const int sa = slot0 + 16 * u + few_slot(n), sb = sa + 8;
            const int2 va = slot_interval(a, s, sa), vb = slot_interval(a, s, sb);
            const int pa = slot_place(a, s, sa), pb = slot_place(a, s, sb);
#pragma unroll
            for (int r = 0; r < NT; ++r)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int row = r * 8 + 2 * j + e, tok = row / a.G;
                const int place = row >= rows ? -1 : a.pre ? a.pre[s.first + tok] : tok;
                const int near = row >= rows ? 0 : s.ctx + draft_depth(a, s, tok) - a.window + 1;
                if ((unsigned)(place - va.x) >= (unsigned)va.y || (pa < near && pa >= a.sinks)) x[u][r][e] = -INFINITY;
                if ((unsigned)(place - vb.x) >= (unsigned)vb.y || (pb < near && pb >= a.sinks)) x[u][r][2 + e] = -INFINITY;
              }
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (slot_interval(a, s, slot0 + 16 * u + few_slot(2 * j + (e & 1)) + 8 * (e >> 1)).y == 0) dead |= 1u << (4 * u + e);
          }
        }
        float top[NT][2];
        bool over = false;
#pragma unroll
        for (int r = 0; r < NT; ++r)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            top[r][e] = fmaxf(x[0][r][e], x[0][r][2 + e]);
            if (kUnits == 2) top[r][e] = fmaxf(top[r][e], fmaxf(x[kUnits - 1][r][e], x[kUnits - 1][r][2 + e]));
            over |= top[r][e] > bound[r][e];
          }
        if (__any_sync(0xFFFFFFFFu, over)) {                 // rare once the first tiles are through
#pragma unroll
          for (int r = 0; r < NT; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float t = fmaxf(m[r][e], top[r][e]);
              t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 4));
              t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 8));
              t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 16));
              const float keep = t == m[r][e] ? 1.f : ex2_approx((m[r][e] - t) * c);      // 0 for m = -inf
              m[r][e] = t;
              off[r][e] = (t == -INFINITY ? 0.f : -t * c) + AttnType<T>::shift;
              bound[r][e] = t == -INFINITY ? t : t + 8.f / c;                              // (8 / c is inf for the smallest scales)
              l[r][e] *= keep;
#pragma unroll
              for (int i2 = 0; i2 < D / 16; ++i2) {
                o[i2][r][e] *= keep;
                o[i2][r][2 + e] *= keep;
              }
            }
        }
        uint32_t p[kUnits][NT][2];
#pragma unroll
        for (int r = 0; r < NT; ++r) {
#pragma unroll
          for (int u = 0; u < kUnits; ++u) {
            const float e0 = ex2_approx(fmaf(x[u][r][0], c, off[r][0])), e1 = ex2_approx(fmaf(x[u][r][1], c, off[r][1]));
            const float e2 = ex2_approx(fmaf(x[u][r][2], c, off[r][0])), e3 = ex2_approx(fmaf(x[u][r][3], c, off[r][1]));
            l[r][0] += e0 + e2;
            l[r][1] += e1 + e3;
            p[u][r][0] = transpose_8x8(Pack<T>::pack(e0, e1));
            p[u][r][1] = transpose_8x8(Pack<T>::pack(e2, e3));
          }
        }
        // this thread's channels of four slots a unit: D / 8 of them from D / 8 * n on, in words of eight
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          uint32_t w[4][kValueWords], s2[2], m2[2];
          float sc[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t at = values + (uint32_t)((first / 8 + 2 * u + (e >> 1)) * packed_eight(D)), k = (uint32_t)few_slot(2 * j + (e & 1));
            load_words(w[e], at + k * (D / 2) + (uint32_t)n * (D / 16));
            sc[e] = packed_scale(load_byte(at + 4 * D + k * (D / 32) + (uint32_t)n * (D / 64) / 4));
          }
          if (dead) {                                        // slots that hold nothing: zeros, whatever lies there
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if ((dead >> (4 * u + e)) & 1u) {
                sc[e] = 0.f;
#pragma unroll
                for (int g = 0; g < kValueWords; ++g) w[e][g] = 0x88888888u;
              }
          }
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            Expand<T>::scale(sc[2 * g], sc[2 * g + 1], s2[g], m2[g]);
          }
#pragma unroll
          for (int g = 0; g < kValueWords; ++g) {
            const uint32_t lo0 = __byte_perm(w[0][g], w[1][g], 0x5410), hi0 = __byte_perm(w[0][g], w[1][g], 0x7632);
            const uint32_t lo1 = __byte_perm(w[2][g], w[3][g], 0x5410), hi1 = __byte_perm(w[2][g], w[3][g], 0x7632);
#pragma unroll
            for (int i2 = 0; i2 < 4; ++i2) {
              const uint32_t a0 = expand_any<T>(lo0, i2, s2[0], m2[0]), a1 = expand_any<T>(hi0, i2, s2[0], m2[0]);
              const uint32_t a2 = expand_any<T>(lo1, i2, s2[1], m2[1]), a3 = expand_any<T>(hi1, i2, s2[1], m2[1]);
#pragma unroll
              for (int r = 0; r < NT; ++r) mma_16816<T>(o[4 * g + i2][r], a0, a1, a2, a3, p[u][r][0], p[u][r][1]);
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(stage));
    }
#pragma unroll
    for (int r = 0; r < NT; ++r)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float sum = l[r][e];
        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 4);
        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 8);
        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 16);
        if (n == 0) stats[warp * 8 * NT + r * 8 + 2 * j + e] = make_float2(m[r][e], sum);
      }
  }

  // ---------------- join of the warps ----------------
  __syncthreads();                                           // every tile was consumed: the ring is free
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicOr(dev_status, 2u);
    for (int i = 0; i < 200; ++i) __nanosleep(1000);         // copies still in flight land
    return;
  }
  float* sums = reinterpret_cast<float*>(few_smem);          // [warp][8 NT][D]
#pragma unroll
  for (int r = 0; r < NT; ++r)
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const int channel = n * (D / 8) + 8 * (i / 4) + 2 * (i % 4);
#pragma unroll
      for (int e = 0; e < 2; ++e)
        *reinterpret_cast<float2*>(sums + ((warp * 8 * NT + r * 8 + 2 * j + e) * D + channel)) = make_float2(o[i][r][e], o[i][r][2 + e]);
    }
  __syncthreads();
  constexpr int kLanes = D / 4;                              // threads a row
  for (int e = threadIdx.x; e < rows * kLanes; e += kFewThreads) {
    const int r = e / kLanes, ch = 4 * (e % kLanes);
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) top = fmaxf(top, stats[w * 8 * NT + r].x);
    float sum = 0.f;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      const float2 st = stats[w * 8 * NT + r];
      const float f = st.x == -INFINITY ? 0.f : ex2_approx((st.x - top) * c);
      const float4 v = *reinterpret_cast<const float4*>(sums + ((w * 8 * NT + r) * D + ch));
      sum += st.y * f;
      y.x += v.x * f; y.y += v.y * f; y.z += v.z * f; y.w += v.w * f;
    }
    const int tok = r / a.G;
    const bool empty = (a.pre && a.pre[s.first + tok] < 0) || (sum == 0.f && top == -INFINITY);   // (NaN and scores beyond fp32 are not)
    const float g = empty ? 0.f : 1.f / sum;
    y = empty ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(y.x * g, y.y * g, y.z * g, y.w * g);
    const float lse2 = empty ? -INFINITY : sum == 0.f ? NAN : top * c - AttnType<T>::shift + log2f(sum);
    const int64_t row = row_of(r);
    if (plan.chunks > 1) {
      *reinterpret_cast<float4*>(plan.part_o + (row * plan.chunks + chunk) * D + ch) = y;
      if (ch == 0) plan.part_lse[row * plan.chunks + chunk] = lse2;
    } else {
      char* to = a.out + 2 * ((int64_t)(s.first + tok) * a.o_ts + (int64_t)(hk * a.G + r % a.G) * a.o_hs + ch);
      *reinterpret_cast<uint2*>(to) = make_uint2(Pack<T>::pack(y.x, y.y), Pack<T>::pack(y.z, y.w));
      if (a.lse && ch == 0) a.lse[row] = lse2 * 0.6931471805599453f;
    }
  }
}

template <typename T, int D, int NT>
static cudaError_t few_attribute(cudaError_t before) {
  return before != cudaSuccess ? before : cudaFuncSetAttribute(packed_rows_kernel<T, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<D, NT>::kSmemBytes);
}
static cudaError_t few_attributes() {
  cudaError_t e = few_attribute<__nv_bfloat16, 128, 1>(cudaSuccess);
  e = few_attribute<__nv_bfloat16, 128, 2>(e);
  e = few_attribute<__nv_bfloat16, 64, 1>(e);
  e = few_attribute<__nv_bfloat16, 64, 2>(e);
  e = few_attribute<__half, 128, 1>(e);
  e = few_attribute<__half, 128, 2>(e);
  e = few_attribute<__half, 64, 1>(e);
  return few_attribute<__half, 64, 2>(e);
}

}  // namespace atts
