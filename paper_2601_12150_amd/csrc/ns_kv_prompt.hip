// Attention over the 8-bit key/value cache for many query rows per key/value head (prompts, drafts of large groups): bound by the
// products and the exponentials.
//
// The products are those of ns_kv_attn.hip with tiles of 32 x 32: S^T = K Q^T, O^T = V^T P^T, so that a lane of S^T holds one row's
// logits of 32 keys in groups of four, which are P^T's operand as they stand.  A workgroup's waves have 32 rows each and share tiles of
// 64 keys, whose codes are turned into fp16 once, on the way into LDS: K as [key][channel], V as [channel][key] with the keys in the
// order that P^T has them.  Both have their 16-byte pieces exchanged by the row's number, so that reads and writes meet all banks.
// While a tile is worked on, the next one's codes are written to the other half of the LDS and those after it are loaded.
//
// Rows are numbered r = token * group + head, so that a causal row tile ends after few more keys than it begins with.
//
// Measured: two sequences' 6627 prompt tokens, 32 query heads of 128 channels on 8, bf16 and int8: 240 us, 790 TFLOP/s (512 queries behind
// 32768 tokens 890 to 930; fp32 590), which is what call after call settles at, the first 50 or so after a pause taking 270 to 305; 512 queries
// of 16 heads of 64 channels across 16385 tokens 61 us, 280 TFLOP/s.  A tile of 64 keys
// by 32 rows of 128 channels is 1024 cycles of products, 512 of exponentials, about 1000 of other vector instructions and 256 of LDS reads of
// the CU's 2048 for its eight waves: no one of them alone is the bound.
#include "ns_kv.h"
#include <algorithm>
#include <type_traits>

namespace ns {

namespace {

constexpr int kKeys = 64;
// 16-byte pieces of a row of K (D / 8 of them) and of V^T (8) in LDS.  V^T's rows are written four channels apart and read one
// apart: the exchange of its pieces is one to one in bits 0..2 of the channel as well as in bits 2..4.  Exchanges are exclusive ors, so
// that of another piece of the row the address is another exclusive or.
template <int D> __device__ __forceinline__ uint32_t k_at(int key, int piece) {
  return (uint32_t)(key * D * 2 + ((piece ^ (key & (D == 64 ? 7 : 15))) * 16));
}
__device__ __forceinline__ uint32_t v_at(int channel, int piece) {
  return (uint32_t)(channel * kKeys * 2 + ((piece ^ ((channel & 7) ^ ((channel >> 3) & 3))) * 16));
}
// 2^x exactly, 2^-10 <= s <= 2^5: what V's codes are multiplied with in fp16 without a rounding (e4m3's least code is 2^-9; 1152 + 127
// times it is below 65504)
__device__ __forceinline__ bool plain_ratio(float s) {
  const uint32_t u = __float_as_uint(s);
  return (u & 0x7fffffu) == 0 && u >= (117u << 23) && u <= (132u << 23);
}

// What a launch leaves for the joins and for the weights' pass: records [split][head][row], and the rows' operands.
struct PromptArgs {
  float *part_o, *part_ml;         // splits > 1: [splits][B Hkv][R] D floats / (reference, sum)
  float *lse2;                     // nullable [B Hkv][R]: log2 of the sum, +inf for a row that sees nothing
  int splits;
  int items;                       // row tiles x splits x heads (x halves)
  int *tickets;                    // items > workgroups: a counter, 0 before the launch
};

// Item x: a tile of rows of a head, or its part of the keys.
// DV: channels of V, and of out, that a workgroup takes: all, or half of them (fp32, D = 256: registers; the logits are computed twice)
// FACTOR: as Lift has it
template <typename T, int CODE, int D, int DV, int WAVES, bool FACTOR>
__device__ __forceinline__ void kv_prompt_item(const ns_kv_cache &c, const ns_kv_attn_desc &d, const T *q, const int32_t *lengths, const int32_t *counts,
                                               T *out, float *lse, const PromptArgs &a, int x) {
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1, KS = D / 16, MT = DV / 32, ROWS = WAVES * 32, THREADS = WAVES * 64;
  constexpr uint32_t kV = kKeys * D * 2, kHalf = kV + kKeys * DV * 2;   // bytes of a tile's K, and with its V^T
  // Registers for both parts of the queries, and LDS for two tiles?  fp32 with D = 256 has the second part in LDS, and one tile.
  constexpr bool EARLY = PARTS * D < 512;
  using L = Lift<FACTOR>;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n32 = lane & 31, hh = lane >> 5;
  const int G = d.heads / c.heads_kv, R = G * d.tokens;
  const int tiles = (R + ROWS - 1) / ROWS;
  // the last rows of all heads see most and go first, so that the launch ends with small items; neighbouring ones have different heads
  const uint32_t heads = (uint32_t)c.batch * c.heads_kv, item = (uint32_t)x / heads, head = (uint32_t)x % heads;
  const int part = (int)(item % (D / DV)), split = (int)(item / (D / DV) % a.splits), tile = tiles - 1 - (int)(item / (D / DV) / a.splits);
  const int h = (int)(head % c.heads_kv), b = (int)(head / c.heads_kv);
  const int length = kv_length(lengths, b, c.capacity), count = kv_count(counts, b, d.tokens);
  const int64_t row = (int64_t)b * c.heads_kv + h;

  const int r = tile * ROWS + wave * 32 + n32;
  const bool real = r < R;
  const int t = real ? r / G : 0, hq = h * G + (real ? r - t * G : 0);
  const int limit = real ? kv_seen(d, t, length, count) : 0;
  // the keys of this workgroup: those that some row sees, or its part of them
  const int last_t = min(min(tile * ROWS + ROWS, R) - 1, R - 1) / G;
  int seen = d.causal ? kv_seen(d, min(last_t, count - 1), length, count) : length;
  if (tile * ROWS / G >= count) seen = 0;
  int n_lo = 0, n_hi = seen;
  if (a.splits > 1) {
    const int share = ((seen + a.splits - 1) / a.splits + kKeys - 1) / kKeys * kKeys;
    n_lo = min(split * share, seen);
    n_hi = min(n_lo + share, seen);
  }
  // of the wave: the keys that all its rows see, and those that any of them sees
  int every = real ? limit : 0x7fffffff, any = limit;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    every = min(every, __shfl_xor(every, o));
    any = max(any, __shfl_xor(any, o));
  }
  every = __builtin_amdgcn_readfirstlane(every);
  any = __builtin_amdgcn_readfirstlane(any);

  // ---- codes on their way into LDS
  const uint8_t *kb = static_cast<const uint8_t *>(c.k) + b * c.stride_b + h * c.stride_h;
  const uint8_t *vb = static_cast<const uint8_t *>(c.v) + b * c.stride_b + h * c.stride_h + part * DV;
  const float *ks = c.k_scale + row * (c.capacity / c.block), *vs = c.v_scale + row * (c.capacity / c.block);
  const int lblock = 31 - __clz(c.block);
  constexpr int KP = kKeys * D / 16 / THREADS, VP = kKeys / 4 * (DV / 4) / THREADS;      // pieces a thread has of K (16 codes) and V (4 x 4)
  constexpr int KR = THREADS / (D / 16), VR = THREADS / (DV / 4) * 4;                    // keys between two of its pieces
  static_assert((KP == 1 || (KR <= 32 && 32 % KR == 0)) && (VP == 1 || (VR <= 32 && 32 % VR == 0)), "key 32 begins a piece of all threads");
  const int k_key = tid / (D / 16), v_key = tid / (DV / 4) * 4;
  const uint32_t stride = (uint32_t)c.stride_t, k_off = (uint32_t)k_key * stride + tid % (D / 16) * 16, v_off = (uint32_t)v_key * stride + tid % (DV / 4) * 4;
  u32x4 kraw[KP];
  uint32_t vraw[VP][4];
  float next_ks[2], next_vs[2], staged_ks[2] = {0.f, 0.f};    // scales of the fetched tile, and K's of the staged one
  auto fetch = [&](int n0) {
    const int n1 = min(n0 + 32, c.capacity - 32);   // (behind the capacity: masked, any scale will do)
    next_ks[0] = ks[n0 >> lblock];
    next_ks[1] = ks[n1 >> lblock];
    next_vs[0] = vs[n0 >> lblock];
    next_vs[1] = vs[n1 >> lblock];
    const uint8_t *kp = kb + (int64_t)n0 * c.stride_t, *vp = vb + (int64_t)n0 * c.stride_t;
    // (the last tile of blocks of 32 may reach 32 keys beyond the capacity: their places take the 32 before once more.  Where a thread has
    // several pieces the first ones of all threads are before key 32, and whole pieces lie behind it)
    const uint32_t back = n0 + kKeys > c.capacity ? 32 * stride : 0u;
    const uint8_t *k_far = KP > 1 ? kp - back : kp, *v_far = VP > 1 ? vp - back : vp;
#pragma unroll
    for (int i = 0; i < KP; i++)
      kraw[i] = *reinterpret_cast<const u32x4 *>((i * KR >= 32 ? k_far : kp) + (int64_t)i * KR * c.stride_t + (k_off - (KP == 1 && k_key >= 32 ? back : 0u)));
#pragma unroll
    for (int i = 0; i < VP; i++)
#pragma unroll
      for (int j = 0; j < 4; j++)
        vraw[i][j] = *reinterpret_cast<const uint32_t *>((i * VR >= 32 ? v_far : vp) + (int64_t)(i * VR + j) * c.stride_t +
                                                         (v_off - (VP == 1 && v_key >= 32 ? back : 0u)));
  };
  if (n_lo < n_hi) fetch(n_lo);

  // ---- queries
  Frag qf[PARTS][KS];
  float factor;
  {
    const T *p = q + b * d.q_stride_b + (int64_t)hq * d.q_stride_h + (int64_t)t * d.q_stride_t + 8 * hh;
    uint32_t most = 0;
#pragma unroll
    for (int s = 0; s < KS; s++)
#pragma unroll
      for (int i = 0; i < 2; i++) {
        const f32x4 x = load4(p + 16 * s + 4 * i);
#pragma unroll
        for (int j = 0; j < 4; j++) most = max(most, __float_as_uint(x[j]) & 0x7fffffffu);
      }
    most = max(most, (uint32_t)__shfl_xor((int)most, 32));
    const int shift = kv_row_shift(most);
    factor = real ? ldexpf(d.scale, -shift) * kLog2e : 0.f;
#pragma unroll
    for (int s = 0; s < KS; s++)
#pragma unroll
      for (int i = 0; i < 2; i++) {
        const f32x4 x = load4(p + 16 * s + 4 * i);
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const float x0 = real ? ldexpf(x[j], shift) : 0.f, x1 = real ? ldexpf(x[j + 1], shift) : 0.f;
          const uint32_t hi = pack_f16(x0, x1);
          qf[0][s].w[2 * i + j / 2] = hi;
          if (PARTS == 2) {
            const f16x2 w = __builtin_bit_cast(f16x2, hi);
            qf[PARTS - 1][s].w[2 * i + j / 2] = pack_f16(x0 - (float)w[0], x1 - (float)w[1]);
          }
        }
      }
  }

  uint8_t *q_lds = lds + kHalf + (wave * KS * 64 + lane) * 16;
  if constexpr (!EARLY) {
#pragma unroll
    for (int s = 0; s < KS; s++) *reinterpret_cast<f16x8 *>(q_lds + s * 1024) = qf[PARTS - 1][s].v;
  }

  // V's scales: o is in units of `unit`, a tile's V in LDS in units of `next`, which is the same but where a much larger scale
  // comes along.  Where both halves' scales are next times a plain ratio, V is multiplied by that on its way (slow = false); else (a NaN, far
  // smaller ones, the caller's own that are no powers of two) LDS has the bare codes, and the products are multiplied.
  float unit = 0.f, next = 0.f, inv_next = 0.f, rel0 = 0.f, rel1 = 0.f;
  bool slow = true;
  // (branches, both here and for the last tile: 262 -> 244 us for the prompts of 2 x 4096 tokens)
  uint32_t last_bits0 = 0, last_bits1 = 0;          // the scales that these go by; 0 for none, which have what scales of 0 would make of them
  By<CODE> v_by[VP];
#pragma unroll
  for (int i = 0; i < VP; i++) v_by[i] = kv_by<CODE>(1.f);
  auto stage = [&](int n0, uint32_t at) {
    staged_ks[0] = next_ks[0];
    staged_ks[1] = next_ks[1];
    const float s0 = next_vs[0], s1 = n0 + 32 < length ? next_vs[1] : s0;
    if (__float_as_uint(s0) != last_bits0 || __float_as_uint(s1) != last_bits1) {
      asm volatile("; other scales");
      last_bits0 = __float_as_uint(s0);
      last_bits1 = __float_as_uint(s1);
      const float big = fmaxf(s0, s1);
      if (!(big <= next * 0x1p5f) && big > 0.f && big < INFINITY) {              // (the first tile's too)
        next = big;
        inv_next = 1.f / big;
      }
      rel0 = s0 * inv_next;
      rel1 = s1 * inv_next;
      slow = !EARLY || !(plain_ratio(rel0) && plain_ratio(rel1));
#pragma unroll
      for (int i = 0; i < VP; i++) v_by[i] = kv_by<CODE>(slow ? 1.f : v_key + i * VR >= 32 ? rel1 : rel0);
    }
    // (opaque: else the compiler keeps every address in a register of its own)
    const uint32_t k_to = (uint32_t)opaque((int)(at + k_at<D>(k_key, tid % (D / 16) * 2)));
    const int quad0 = v_key / 4;
    const uint32_t v_to = (uint32_t)opaque((int)(at + kV + v_at(tid % (DV / 4) * 4, (quad0 >> 2) * 2 + (quad0 & 1)) + ((quad0 >> 1) & 1) * 8));
#pragma unroll
    for (int i = 0; i < KP; i++) {
      const uint32_t to = k_to + i * KR * D * 2;
      static_assert(KR % 16 == 0 || KP == 1, "the exchange is the same for all of a thread's pieces");
      *reinterpret_cast<f16x8 *>(lds + to) = kv_frag<CODE>(kraw[i][0], kraw[i][1]).v;
      *reinterpret_cast<f16x8 *>(lds + (to ^ 16)) = kv_frag<CODE>(kraw[i][2], kraw[i][3]).v;
    }
    const bool tail = n0 + kKeys > length;         // what lies behind may be NaN
#pragma unroll
    for (int i = 0; i < VP; i++) {
      const int key = v_key + i * VR;
      static_assert(VP == 1 || VR == 16 || VR == 32, "a thread's keys are 16 or 32 apart: two or four pieces further on");
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; j++) w[j] = kv_raw<CODE>(vraw[i][j]);
      if (tail) {
        asm volatile("; tail");
#pragma unroll
        for (int j = 0; j < 4; j++) w[j] = n0 + key + j >= length ? kv_raw<CODE>(0u) : w[j];
      }
      const uint32_t lo0 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), lo1 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
      const uint32_t hi0 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), hi1 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
      // keys 4 quad .. + 3 are the first or second half of the piece that lanes of half (quad & 1) read for the step quad / 4
      const uint32_t to = v_to ^ (uint32_t)(VR * 2 * i);
      *reinterpret_cast<u32x2 *>(lds + to) = u32x2{kv_f16x2_by<CODE, 0>(lo0, v_by[i]), kv_f16x2_by<CODE, 0>(lo1, v_by[i])};
      *reinterpret_cast<u32x2 *>(lds + (to ^ 16) + kKeys * 2) = u32x2{kv_f16x2_by<CODE, 1>(lo0, v_by[i]), kv_f16x2_by<CODE, 1>(lo1, v_by[i])};
      *reinterpret_cast<u32x2 *>(lds + (to ^ 32) + kKeys * 4) = u32x2{kv_f16x2_by<CODE, 0>(hi0, v_by[i]), kv_f16x2_by<CODE, 0>(hi1, v_by[i])};
      *reinterpret_cast<u32x2 *>(lds + (to ^ 48) + kKeys * 6) = u32x2{kv_f16x2_by<CODE, 1>(hi0, v_by[i]), kv_f16x2_by<CODE, 1>(hi1, v_by[i])};
    }
  };

  f32x16 o[MT];
#pragma unroll
  for (int i = 0; i < MT; i++)
#pragma unroll
    for (int e = 0; e < 16; e++) o[i][e] = 0.f;
  float m = -INFINITY, l = 0.f;

  uint32_t at = 0;
  const uint32_t k_lane = k_at<D>(n32, hh), v_lane = kV + v_at(n32, hh);
  int n0 = n_lo;
  // LDS operands that are read before the products of the ones before them: K's 32 keys and V's 32 channels at a time (277 -> 244 us for
  // the prompts of 2 x 4096 tokens).  Channels of 64 have a third wave for that, which the registers would cost; fp32 and those of 256 have
  // no registers left.
  constexpr bool AHEAD = PARTS == 1 && D == 128;
  // The two waves of a SIMD: one stages the next tile before its own products, the other between them and the values', so that one has
  // matrix instructions for most of what the other has of others (243 -> 239 us; 316 -> 295 us for 512 queries behind 32768 tokens;
  // fp32, whose products are twice as many: 463 against 476 us without and with it)
  constexpr bool LATE = PARTS == 1 && WAVES == 8;
  f16x8 kf[2][AHEAD ? KS : 1];
  auto read_k = [&](int x, uint32_t kl) {
#pragma unroll
    for (int k = 0; k < KS; k++) kf[x][AHEAD ? k : 0] = *reinterpret_cast<const f16x8 *>(lds + (kl ^ (32u * k)) + x * 32 * D * 2);
    __builtin_amdgcn_sched_barrier(0);
  };
  // one tile: its logits, weights and values.  SLOW: its V holds bare codes
  auto tile_of_keys = [&](auto is_slow, auto between, float f_v0, float f_v1, float tile_unit, float sk0, float sk1) {
    constexpr bool SLOW = decltype(is_slow)::value;
    const bool edge = n0 + kKeys > every;
    const uint32_t kl = (uint32_t)opaque((int)(k_lane + at)), vl = (uint32_t)opaque((int)(v_lane + at));
    f32x16 s[2];
#pragma unroll
    for (int x = 0; x < 2; x++) {
#pragma unroll
      for (int e = 0; e < 16; e++) s[x][e] = 0.f;
      if (AHEAD && x == 0) read_k(1, kl);
#pragma unroll
      for (int k = 0; k < KS; k++) {
        const f16x8 kv = AHEAD ? kf[x][AHEAD ? k : 0] : *reinterpret_cast<const f16x8 *>(lds + (kl ^ (32u * k)) + x * 32 * D * 2);
#pragma unroll
        for (int pt = PARTS - 1; pt >= 0; pt--) {
          const f16x8 qv = pt == 1 && !EARLY ? *reinterpret_cast<const f16x8 *>(q_lds + k * 1024) : qf[pt][k].v;
          s[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kv, qv, s[x], 0, 0, 0);
        }
        if (!EARLY && k % 4 == 3) __builtin_amdgcn_sched_barrier(0);      // (not all operands at once)
      }
    }
    f16x8 vf[2][4];
    if constexpr (AHEAD && !SLOW) {
#pragma unroll
      for (int k = 0; k < 4; k++) vf[0][k] = *reinterpret_cast<const f16x8 *>(lds + (vl ^ (32u * k)));
      __builtin_amdgcn_sched_barrier(0);
    }
    const bool fresh = m == -INFINITY;
    const float ref = fresh ? 0.f : m;
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < 2; x++) {
      const float f = factor * (x ? sk1 : sk0);
#pragma unroll
      for (int e = 0; e < 16; e++) s[x][e] = __builtin_fmaf(s[x][e], f, -ref);
    }
    if (edge) {
      asm volatile("; masked");                       // (a branch, not a select for every logit of every tile)
#pragma unroll
      for (int x = 0; x < 2; x++)
#pragma unroll
        for (int e = 0; e < 16; e++) s[x][e] = n0 + x * 32 + (e >> 2) * 8 + hh * 4 + (e & 3) < limit ? s[x][e] : -INFINITY;
    }
#pragma unroll
    for (int x = 0; x < 2; x++)
#pragma unroll
      for (int e = 0; e < 16; e++) top = fmaxf(top, s[x][e]);
    if (__any(top > L::room || (fresh && top > -INFINITY)) || tile_unit != unit) {
      top = half_swap_max(top);
      const bool moved = top > L::room || (fresh && top > -INFINITY);
      const float move = moved ? top - L::exponent : 0.f;
      float fade = __builtin_amdgcn_exp2f(fminf(-move, 0.f));      // (a fresh row's sums are 0, or NaN: not times a factor beyond fp32)
#pragma unroll
      for (int x = 0; x < 2; x++)
#pragma unroll
        for (int e = 0; e < 16; e++) s[x][e] -= move;
      if (moved) m = ref + move;
      l *= fade;
      if (tile_unit != unit) fade *= unit / tile_unit;     // (both are 0 as long as all scales were 0 or NaN)
      unit = tile_unit;
#pragma unroll
      for (int i = 0; i < MT; i++) o[i] *= fade;
    }
    Frag pf[PARTS][4];
    float ls[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 2; x++)
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        float p0 = __builtin_amdgcn_exp2f(s[x][e]), p1 = __builtin_amdgcn_exp2f(s[x][e + 1]);
        ls[e % 4] += p0;
        ls[e % 4 + 1] += p1;
        p0 *= L::factor;
        p1 *= L::factor;
        const uint32_t hi = pack_f16(p0, p1);
        pf[0][x * 2 + e / 8].w[e % 8 / 2] = hi;
        if (PARTS == 2) {
          const f16x2 w = __builtin_bit_cast(f16x2, hi);
          pf[PARTS - 1][x * 2 + e / 8].w[e % 8 / 2] = pack_f16(p0 - (float)w[0], p1 - (float)w[1]);
        }
      }
    l += (ls[0] + ls[1]) + (ls[2] + ls[3]);
    between();
    if constexpr (!SLOW) {
#pragma unroll
      for (int i = 0; i < MT; i++) {
        if (!AHEAD || i + 1 < MT) {
          const int next_i = AHEAD ? i + 1 : i;
#pragma unroll
          for (int k = 0; k < 4; k++) vf[next_i & 1][k] = *reinterpret_cast<const f16x8 *>(lds + (vl ^ (32u * k)) + next_i * 32 * kKeys * 2);
        }
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
          for (int pt = PARTS - 1; pt >= 0; pt--) o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[i & 1][k], pf[pt][k].v, o[i], 0, 0, 0);
      }
    } else {                                          // (a NaN block makes those rows NaN that see it)
      const float f0 = edge && n0 >= limit ? 0.f : f_v0, f1 = edge && n0 + 32 >= limit ? 0.f : f_v1;
#pragma unroll
      for (int i = 0; i < MT; i++)
#pragma unroll
        for (int x = 0; x < 2; x++) {
          f32x16 y;
#pragma unroll
          for (int e = 0; e < 16; e++) y[e] = 0.f;
#pragma unroll
          for (int k = 2 * x; k < 2 * x + 2; k++) {
            const f16x8 vk = *reinterpret_cast<const f16x8 *>(lds + (vl ^ (32u * k)) + i * 32 * kKeys * 2);
#pragma unroll
            for (int pt = PARTS - 1; pt >= 0; pt--) y = __builtin_amdgcn_mfma_f32_32x32x16_f16(vk, pf[pt][k].v, y, 0, 0, 0);
          }
#pragma unroll
          for (int e = 0; e < 16; e++) o[i][e] = __builtin_fmaf(y[e], x ? f1 : f0, o[i][e]);
          __builtin_amdgcn_sched_barrier(0);
        }
    }
  };
  auto ahead = [&] {                                  // the next tile into the other half, the one after it on its way
    if (EARLY && n0 + kKeys < n_hi) {
      stage(n0 + kKeys, at ^ kHalf);
      if (n0 + 2 * kKeys < n_hi) fetch(n0 + 2 * kKeys);
    }
  };
  auto step = [&] {
    __syncthreads();
    if (EARLY) at ^= kHalf;
    n0 += kKeys;
    if (!EARLY && n0 < n_hi) {
      fetch(n0);
      stage(n0, at);
      __syncthreads();
    }
  };
  if (n_lo < n_hi) {
    stage(n_lo, 0);
    unit = next;
    if (EARLY && n_lo + kKeys < n_hi) fetch(n_lo + kKeys);
    __syncthreads();
  }
  const bool late = LATE && wave >= 4;
  // (loops of their own for the two kinds of tiles, and for those that the wave has no part in: o stays in its registers)
  const int n_wave = min(n_hi, any);
  while (n0 < n_wave) {
    if constexpr (EARLY)
      while (n0 < n_wave && !slow) {
        const float u = next, k0 = staged_ks[0], k1 = staged_ks[1];
        if constexpr (AHEAD) read_k(0, (uint32_t)opaque((int)(k_lane + at)));
        if (!late) ahead();
        tile_of_keys(std::false_type{}, [&] { if (late) ahead(); }, 0.f, 0.f, u, k0, k1);
        step();
      }
    while (n0 < n_wave && slow) {
      const float u = next, f0 = rel0, f1 = rel1, k0 = staged_ks[0], k1 = staged_ks[1];
      if constexpr (AHEAD) read_k(0, (uint32_t)opaque((int)(k_lane + at)));
      ahead();
      tile_of_keys(std::true_type{}, [] {}, f0, f1, u, k0, k1);
      step();
    }
  }
  while (n0 < n_hi) {
    ahead();
    step();
  }

  // ---- out: a lane has its row's channels 32 i + 8 (e / 4) + 4 hh + e % 4
  l = half_swap_sum(l);
  if (m == -INFINITY && l != l) m = 0.f;            // a row of NaN is not an empty one
  if (!real) return;
  if (a.splits > 1) {
    const int64_t rec = ((int64_t)split * c.batch * c.heads_kv + row) * R + r;
    const float u = unit * (1.f / L::factor);
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<f32x4 *>(a.part_o + rec * D + part * DV + 32 * i + 2 * e + 4 * hh) = f32x4{o[i][e] * u, o[i][e + 1] * u, o[i][e + 2] * u, o[i][e + 3] * u};
    if (hh == 0 && part == 0) *reinterpret_cast<f32x2 *>(a.part_ml + rec * 2) = f32x2{m, l};
    return;
  }
  const bool some = m != -INFINITY;
  const float by = some ? unit / (l * L::factor) : 0.f;
  T *to = out + b * d.out_stride_b + (int64_t)hq * d.out_stride_h + (int64_t)t * d.out_stride_t + part * DV;
#pragma unroll
  for (int i = 0; i < MT; i++)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      f32x4 y;
#pragma unroll
      for (int j = 0; j < 4; j++) y[j] = some ? o[i][e + j] * by : 0.f;
      T *p = to + 32 * i + 2 * e + 4 * hh;
      store4(p, y);
    }
  if (hh == 0 && part == 0) {
    const float z2 = some ? m + __log2f(l) : -INFINITY;
    if (lse) lse[((int64_t)b * d.heads + hq) * d.tokens + t] = z2 * kLn2;
    if (a.lse2) a.lse2[row * R + r] = some ? z2 : INFINITY;
  }
}

// Workgroups that are through with an item draw the next one.  Dealt out by the hardware, which hands workgroups to the shader engines
// in turn, whether or not another one has room, items of very different lengths (a padded batch, causal rows) kept a third of the CUs
// waiting: 293 us for the prompts of 2 x 4096 tokens that take 262 us drawn (245 us with the operands' reads ahead).
template <typename T, int CODE, int D, int DV, int WAVES, bool FACTOR>
__global__ __launch_bounds__(WAVES * 64, D > 128 ? 1 : D == 64 && sizeof(T) == 2 ? 3 : 2)
void kv_prompt_kernel(ns_kv_cache c, ns_kv_attn_desc d, const T *q, const int32_t *lengths, const int32_t *counts, T *out, float *lse, PromptArgs a) {
  __shared__ int drawn;
  int x = (int)blockIdx.x;
  while (true) {
    if (threadIdx.x == 0 && a.tickets) drawn = (int)gridDim.x + atomicAdd(a.tickets, 1);
    kv_prompt_item<T, CODE, D, DV, WAVES, FACTOR>(c, d, q, lengths, counts, out, lse, a, x);
    if (!a.tickets) return;
    __syncthreads();
    x = drawn;
    if (x >= a.items) return;
    __syncthreads();
  }
}

// (a launch, where the items are more than the workgroups that the chip holds: 4.7 us)
__global__ void kv_no_tickets_kernel(int *tickets) { *tickets = 0; }

// The splits' results together: D / 4 threads per row, four records on their way at a time (12 parts of 8192 rows of 64: 6.9 us).  The workgroups behind those make the operands of the weights' second pass.
template <typename T>
__global__ __launch_bounds__(256) void kv_prompt_join_kernel(ns_kv_cache c, ns_kv_attn_desc d, const T *q, PromptArgs a, T *out, float *lse, Frag *frags,
                                                             float *factors) {
  const int tid = threadIdx.x, D = c.head_dim, quads = D / 4, rows = 256 / quads, G = d.heads / c.heads_kv, R = G * d.tokens;
  const int h = blockIdx.y, b = blockIdx.z, groups = (R + rows - 1) / rows;
  if ((int)blockIdx.x >= groups) {
    const int tile = ((int)blockIdx.x - groups) * 4 + (tid >> 6);
    if (tile < (R + 15) / 16) kv_rows_tile(c, d, q, b, h, tile, tid & 63, frags, factors);
    return;
  }
  const int r = (int)blockIdx.x * rows + tid / quads, dd = tid % quads * 4;
  if (r >= R) return;
  const int64_t heads = (int64_t)c.batch * c.heads_kv, row = (int64_t)b * c.heads_kv + h;
  const float *ml = a.part_ml + (row * R + r) * 2, *o = a.part_o + (row * R + r) * D + dd;
  const int64_t apart = heads * R;                  // records between two splits'
  float M = -INFINITY, L = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.splits; s0 += 4) {        // (four records on their way at a time)
    f32x2 z[4];
    f32x4 v[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int64_t s = min(s0 + i, a.splits - 1);
      z[i] = *reinterpret_cast<const f32x2 *>(ml + s * apart * 2);
      v[i] = *reinterpret_cast<const f32x4 *>(o + s * apart * D);
    }
    float next = M;
#pragma unroll
    for (int i = 0; i < 4; i++) next = fmaxf(next, s0 + i < a.splits ? z[i][0] : -INFINITY);
    const float ref = next == -INFINITY ? 0.f : next, keep = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - ref);
    y *= keep;
    L *= keep;
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (s0 + i < a.splits && z[i][0] != -INFINITY) {
        const float fade = __builtin_amdgcn_exp2f(z[i][0] - ref);
        y += v[i] * fade;
        L += z[i][1] * fade;
      }
    M = next;
  }
  const bool some = M != -INFINITY;
  const int t = r / G, hq = h * G + r - t * G;
  const float inv = some ? 1.f / L : 0.f;
#pragma unroll
  for (int j = 0; j < 4; j++) y[j] = some ? y[j] * inv : 0.f;
  store4(out + b * d.out_stride_b + (int64_t)hq * d.out_stride_h + (int64_t)t * d.out_stride_t + dd, y);
  if (dd == 0) {
    const float z2 = some ? M + __log2f(L) : -INFINITY;
    if (lse) lse[((int64_t)b * d.heads + hq) * d.tokens + t] = z2 * kLn2;
    if (a.lse2) a.lse2[row * R + r] = some ? z2 : INFINITY;
  }
}

// ---- the weights that every position was given: exp(logit - lse) summed over the rows, with K read again.  The rows' operands and
// factors are made once (kv_rows_tile); a wave then has 16 KX keys in registers and takes 16 rows at a time from the L2.  Bound by the
// exponentials and the products (512 rows of 16 heads of 64 channels, 16385 keys: 134 M logits in 40 us), for few rows by the reads of K
// (32 rows, 58990 tokens of 8 heads of 128 channels: 60 MB in 22 us, 2.7 TB/s; through kv_weights_sum_kernel 26).

template <typename T>
__global__ __launch_bounds__(256) void kv_weights_rows_kernel(ns_kv_cache c, ns_kv_attn_desc d, const T *q, Frag *frags, float *factors) {
  const int tile = blockIdx.x * 4 + (threadIdx.x >> 6), R = d.heads / c.heads_kv * d.tokens;
  if (tile < (R + 15) / 16) kv_rows_tile(c, d, q, blockIdx.z, blockIdx.y, tile, threadIdx.x & 63, frags, factors);
}

// Many rows: a wave's keys stay, the rows' operands come from the L2, an operand serves KX tiles of 16 keys.  SHARE: a workgroup's
// waves have the same keys and take the tiles of rows in turn.
template <int PARTS, int CODE, int D, int KX, bool SHARE>
__global__ __launch_bounds__(256, 2) void kv_weights_sum_kernel(ns_kv_cache c, ns_kv_attn_desc d, const int32_t *lengths, const int32_t *counts,
                                                             const Frag *frags, const float *factors, const float *lse2, const float *w_in,
                                                             float *w_out) {
  constexpr int KS = D / 32, kKeysOf = 16 * KX;
  const int lane = threadIdx.x & 63, n16 = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = d.heads / c.heads_kv, R = G * d.tokens, tiles = (R + 15) / 16, lblock = 31 - __clz(c.block);
  const int h = blockIdx.y, b = blockIdx.z, n0 = (SHARE ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave) * kKeysOf;
  constexpr int STEP = SHARE ? 4 : 1;
  __shared__ float sums[4][kKeysOf][17];
  const int length = kv_length(lengths, b, c.capacity), count = kv_count(counts, b, d.tokens);
  const int64_t row = (int64_t)b * c.heads_kv + h;
  if (n0 >= c.capacity) return;
  float sum = 0.f;                                  // of the key n0 + lane
  // causal: the first row that sees key n0 is that of the query at its position
  const int first = d.causal ? (int)min((int64_t)max(0, n0 - (length - count)) * G / 16, (int64_t)tiles) : 0;
  const int last = min(tiles, (count * G + 15) / 16);
  // from here on a tile's rows see all these keys (but for the last tile's, some of which may be no rows)
  const int query = n0 + kKeysOf - 1 - (length - count);              // the one at the last key's position
  const int clear = n0 + kKeysOf > length ? tiles : d.causal ? (int)min(((int64_t)max(0, query) * G + 15) / 16, (int64_t)tiles) : 0;
  if (n0 < length && first < last) {
    const uint8_t *kp = static_cast<const uint8_t *>(c.k) + b * c.stride_b + h * c.stride_h + (int64_t)n0 * c.stride_t;
    const uint32_t off = (uint32_t)n16 * (uint32_t)c.stride_t + 16 * g;
    u32x4 kw[KX][D / 64];
    float sk[KX];
#pragma unroll
    for (int x = 0; x < KX; x++) {
      // (tiles behind the capacity take the last one again; they are masked)
      const int at = min(16 * x, c.capacity - 16 - n0);
#pragma unroll
      for (int i = 0; i < D / 64; i++) kw[x][i] = *reinterpret_cast<const u32x4 *>(kp + (int64_t)at * c.stride_t + 64 * i + off);
      sk[x] = c.k_scale[row * (c.capacity >> lblock) + ((n0 + at) >> lblock)];
    }
    const Frag *qp = frags + (row * tiles * PARTS) * KS * 64 + lane;
    Frag next[PARTS * KS];
    float fr, ref;
    auto load_rows = [&](int tile) {
#pragma unroll
      for (int k = 0; k < PARTS * KS; k++) next[k] = qp[((int64_t)tile * PARTS * KS + k) * 64];
      const int r = tile * 16 + n16;
      fr = factors[row * tiles * 16 + r];
      ref = lse2[row * R + min(r, R - 1)];            // (rows that are none are masked)
    };
    const int from_tile = first + (SHARE ? wave : 0);
    load_rows(min(from_tile, last - 1));
    Frag kf[KX][KS];
#pragma unroll
    for (int x = 0; x < KX; x++)
#pragma unroll
      for (int k = 0; k < KS; k++) kf[x][k] = kv_frag<CODE>(kw[x][k / 2][2 * (k % 2)], kw[x][k / 2][2 * (k % 2) + 1]);
    f32x4 acc[KX];
#pragma unroll
    for (int x = 0; x < KX; x++) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int tile = from_tile; tile < last; tile += STEP) {
      const int r = tile * 16 + n16;
      const float f_row = fr, z0 = ref;
      f32x4 s[KX];
#pragma unroll
      for (int x = 0; x < KX; x++) s[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = PARTS * KS - 1; k >= 0; k--)       // (the smaller parts first)
#pragma unroll
        for (int x = 0; x < KX; x++) s[x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[x][k % KS].v, next[k].v, s[x], 0, 0, 0);
      if (tile + STEP < last) load_rows(tile + STEP);
#pragma unroll
      for (int x = 0; x < KX; x++) {
        const float f = f_row * sk[x];
#pragma unroll
        for (int e = 0; e < 4; e++) s[x][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][e], f, -z0));
      }
      if (tile < clear || tile == last - 1) {
        asm volatile("; masked");                     // (a branch, not selects for every tile)
        const int limit = r < R ? kv_seen(d, r / G, length, count) : 0;
#pragma unroll
        for (int x = 0; x < KX; x++)
#pragma unroll
          for (int e = 0; e < 4; e++) s[x][e] = n0 + 16 * x + 4 * g + e < limit ? s[x][e] : 0.f;
      }
#pragma unroll
      for (int x = 0; x < KX; x++) acc[x] += s[x];
    }
    // over the 16 rows' lanes, by way of LDS: a lane then has a key
    float (&to)[kKeysOf][17] = sums[wave];
#pragma unroll
    for (int x = 0; x < KX; x++)
#pragma unroll
      for (int e = 0; e < 4; e++) to[16 * x + 4 * g + e][n16] = acc[x][e];
    if (SHARE)
      __syncthreads();
    else
      __builtin_amdgcn_wave_barrier();                // (a wave's LDS operations are in order)
    const int from = lane % kKeysOf;
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < STEP; w++)
#pragma unroll
      for (int i = 0; i < 16; i++) part[i % 4] += (SHARE ? sums[w] : to)[from][i];
    sum = (part[0] + part[1]) + (part[2] + part[3]);
  }
  const int n = n0 + lane;
  if ((SHARE && wave > 0) || lane >= kKeysOf || n >= c.capacity || (n >= length && w_in == w_out)) return;
  const int64_t at = row * c.capacity + n;
  w_out[at] = (w_in ? w_in[at] : 0.f) + sum;
}

// Few rows: the operands of QT tiles of them stay in registers, and a wave takes `steps` times 32 keys, the next ones' codes on their way.
template <int PARTS, int CODE, int D, int QT>
__global__ __launch_bounds__(256, 2) void kv_weights_stream_kernel(ns_kv_cache c, ns_kv_attn_desc d, const int32_t *lengths, const int32_t *counts,
                                                                   const Frag *frags, const float *factors, const float *lse2, const float *w_in,
                                                                   float *w_out, int steps) {
  constexpr int KS = D / 32, KX = 2, kKeysOf = 16 * KX;
  const int lane = threadIdx.x & 63, n16 = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = d.heads / c.heads_kv, R = G * d.tokens, tiles = (R + 15) / 16, lblock = 31 - __clz(c.block);
  const int h = blockIdx.y, b = blockIdx.z;
  __shared__ float sums[4][kKeysOf][17];
  const int length = kv_length(lengths, b, c.capacity), count = kv_count(counts, b, d.tokens);
  const int64_t row = (int64_t)b * c.heads_kv + h;
  int n0 = ((int)blockIdx.x * steps * 4 + wave) * kKeysOf;
  const int end = min(n0 + steps * 4 * kKeysOf, c.capacity), seen = w_in == w_out ? min(end, length) : end;
  if (n0 >= seen) return;

  const uint8_t *kb = static_cast<const uint8_t *>(c.k) + b * c.stride_b + h * c.stride_h;
  const uint32_t off = (uint32_t)n16 * (uint32_t)c.stride_t + 16 * g;
  u32x4 kw[KX][D / 64];
  float next_sk, next_w = 0.f;
  auto fetch = [&](int n) {
    if (w_in && n + lane % kKeysOf < seen) next_w = w_in[row * c.capacity + n + lane % kKeysOf];
    if (n >= length) return;
    const uint8_t *kp = kb + (int64_t)n * c.stride_t;
    const uint32_t o = (uint32_t)opaque((int)off);
#pragma unroll
    for (int x = 0; x < KX; x++)
#pragma unroll
      for (int i = 0; i < D / 64; i++) kw[x][i] = *reinterpret_cast<const u32x4 *>(kp + (int64_t)16 * x * c.stride_t + 64 * i + o);
    next_sk = c.k_scale[row * (c.capacity >> lblock) + (n >> lblock)];
  };
  fetch(n0);
  Frag qf[QT][PARTS * KS];
  float fr[QT], ref[QT];
  int limit[QT];
#pragma unroll
  for (int t = 0; t < QT; t++) {
    const int tile = min(t, tiles - 1), r = t * 16 + n16;
    const Frag *qp = frags + ((row * tiles + tile) * PARTS) * KS * 64 + lane;
#pragma unroll
    for (int k = 0; k < PARTS * KS; k++) qf[t][k] = qp[k * 64];
    limit[t] = r < R ? kv_seen(d, r / G, length, count) : 0;
    fr[t] = factors[row * tiles * 16 + tile * 16 + n16];
    ref[t] = lse2[row * R + min(r, R - 1)];
  }
  for (; n0 < seen; n0 += 4 * kKeysOf) {
    f32x4 acc[KX];
#pragma unroll
    for (int x = 0; x < KX; x++) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float before = next_w;
    if (n0 < length) {
      Frag kf[KX][KS];
#pragma unroll
      for (int x = 0; x < KX; x++)
#pragma unroll
        for (int k = 0; k < KS; k++) kf[x][k] = kv_frag<CODE>(kw[x][k / 2][2 * (k % 2)], kw[x][k / 2][2 * (k % 2) + 1]);
      const float sk = next_sk;
      if (n0 + 4 * kKeysOf < seen) fetch(n0 + 4 * kKeysOf);
#pragma unroll
      for (int t = 0; t < QT; t++) {
        const float f = fr[t] * sk;
#pragma unroll
        for (int x = 0; x < KX; x++) {
          f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = PARTS * KS - 1; k >= 0; k--) s = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[x][k % KS].v, qf[t][k].v, s, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 4; e++) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], f, -ref[t]));
            acc[x][e] += n0 + 16 * x + 4 * g + e < limit[t] ? p : 0.f;
          }
        }
      }
    } else if (n0 + 4 * kKeysOf < seen) {
      fetch(n0 + 4 * kKeysOf);
    }
    // over the 16 rows' lanes, by way of LDS: a lane then has a key
    float (&to)[kKeysOf][17] = sums[wave];
    __builtin_amdgcn_wave_barrier();                  // (a wave's LDS operations are in order)
#pragma unroll
    for (int x = 0; x < KX; x++)
#pragma unroll
      for (int e = 0; e < 4; e++) to[16 * x + 4 * g + e][n16] = acc[x][e];
    __builtin_amdgcn_wave_barrier();
    const int key = lane % kKeysOf, part = lane / kKeysOf * 8;        // two lanes a key, eight rows each
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) sum += to[key][part + i];
    sum = half_swap_sum(sum);
    const int n = n0 + key;
    if (lane < kKeysOf && n < seen) w_out[row * c.capacity + n] = before + sum;
  }
}

// ---- host side

// Waves of a workgroup: a tile's conversion serves the rows of all of them.  128 channels, 8 waves against two workgroups of 4: 245 us against
// 270 for the prompts of 2 x 4096 tokens, fp32 530 against 565.  64 channels have three workgroups of 4 instead (a tile is 16 codes for each
// thread of 4 waves), 256 channels registers for one wave a SIMD.
constexpr int waves_of(int D) { return D == 128 ? 8 : 4; }

// Workgroups of the prompt kernel that a CU holds
constexpr int per_cu(int D, int dtype) { return D == 64 ? dtype == NS_F32 ? 2 : 3 : 1; }

int splits_of(const ns_kv_cache &c, const ns_kv_attn_desc &d) {
  const int64_t rows = (int64_t)d.heads / c.heads_kv * d.tokens, per = waves_of(c.head_dim) * 32;
  const int64_t wgs = (rows + per - 1) / per * c.heads_kv * c.batch, cus = device_cu_count();
  // as many parts of the keys as fill the chip once, of 512 keys at least, or 256 of 128 channels (256 queries of 16 heads, 2048 tokens: bf16
  // 31 -> 28 us, fp32 41 -> 33; 1024 queries and tokens of 64 channels: 24 us with 512 and 27 with 256; fp32 of 256 channels 55 and 70)
  return (int)std::max<int64_t>(1, std::min<int64_t>({per_cu(c.head_dim, d.dtype) * cus / wgs, (int64_t)c.capacity / (c.head_dim == 128 ? 256 : 512), 64}));
}

struct Layout { size_t o, ml, lse2, frags, factors, tickets, total; int splits; };
Layout layout_of(const ns_kv_cache &c, const ns_kv_attn_desc &d, bool weights) {
  Layout w;
  w.splits = splits_of(c, d);
  const size_t rows = (size_t)(d.heads / c.heads_kv) * d.tokens, heads = (size_t)c.batch * c.heads_kv;
  size_t off = 0;
  w.o = off;
  if (w.splits > 1) off += align_up(w.splits * heads * rows * c.head_dim * 4, 256);
  w.ml = off;
  if (w.splits > 1) off += align_up(w.splits * heads * rows * 8, 256);
  w.lse2 = off;
  if (weights) off += align_up(heads * rows * 4, 256);
  w.frags = off;
  if (weights) off += kv_rows_frag_bytes(c, d);
  w.factors = off;
  if (weights) off += kv_rows_factor_bytes(c, d);
  w.tickets = off;
  w.total = off + 256;
  return w;
}

template <typename T, int CODE, int D, bool FACTOR>
ns_status launch(const KvAttnArgs &a) {
  constexpr int WAVES = waves_of(D), DV = sizeof(T) == 4 && D == 256 ? 128 : D;
  const ns_kv_cache &c = a.c;
  const Layout w = layout_of(c, a.d, a.w_out != nullptr);
  const int rows = a.d.heads / c.heads_kv * a.d.tokens, tiles = (rows + WAVES * 32 - 1) / (WAVES * 32);
  PromptArgs p{reinterpret_cast<float *>(a.ws + w.o), reinterpret_cast<float *>(a.ws + w.ml),
               a.w_out ? reinterpret_cast<float *>(a.ws + w.lse2) : nullptr, w.splits, 0, nullptr};
  // two tiles, or one and the second part of the queries
  const int tile_lds = kKeys * (D + DV) * 2, lds = DV == D ? 2 * tile_lds : tile_lds + WAVES * 32 * D * 2;
  const T *q = static_cast<const T *>(a.q);
  T *out = static_cast<T *>(a.out);
  ns_status st = reserve_lds_once(reinterpret_cast<const void *>(kv_prompt_kernel<T, CODE, D, DV, WAVES, FACTOR>), lds);
  if (st != NS_OK) return st;
  const int64_t items = (int64_t)tiles * w.splits * (D / DV) * c.heads_kv * c.batch;
  if (items > 0x7fffffff - 65536) return fail(NS_ERR_UNSUPPORTED, "too many rows");
  const int workgroups = (int)std::min<int64_t>(items, (int64_t)per_cu(D, a.d.dtype) * device_cu_count());
  p.items = (int)items;                               // (with room for the numbers that are drawn in vain)
  if (items > workgroups) {
    p.tickets = reinterpret_cast<int *>(a.ws + w.tickets);
    hipLaunchKernelGGL(kv_no_tickets_kernel, dim3(1), dim3(1), 0, a.stream, p.tickets);
    if ((st = check_launch("kv_no_tickets_kernel")) != NS_OK) return st;
  }
  hipLaunchKernelGGL((kv_prompt_kernel<T, CODE, D, DV, WAVES, FACTOR>), dim3((unsigned)workgroups), dim3(WAVES * 64), lds, a.stream, c, a.d, q, a.lengths, a.counts, out,
                     a.lse, p);
  st = check_launch("kv_prompt_kernel");
  Frag *frags = reinterpret_cast<Frag *>(a.ws + w.frags);
  float *factors = reinterpret_cast<float *>(a.ws + w.factors);
  if (st == NS_OK && w.splits > 1) {
    const int per = 1024 / D, more = a.w_out ? (rows + 63) / 64 : 0;
    hipLaunchKernelGGL((kv_prompt_join_kernel<T>), dim3((unsigned)((rows + per - 1) / per + more), (unsigned)c.heads_kv, (unsigned)c.batch), dim3(256), 0,
                       a.stream, c, a.d, q, p, out, a.lse, frags, factors);
    st = check_launch("kv_prompt_join_kernel");
  }
  if (st != NS_OK || !a.w_out) return st;
  return launch_kv_weights_again(a, frags, factors, p.lse2, w.splits == 1);
}

template <typename T, int CODE, bool FACTOR> ns_status launch_d(const KvAttnArgs &a) {
  return a.c.head_dim == 64 ? launch<T, CODE, 64, FACTOR>(a) : a.c.head_dim == 128 ? launch<T, CODE, 128, FACTOR>(a) : launch<T, CODE, 256, FACTOR>(a);
}
template <typename T, int CODE> ns_status launch_any(const KvAttnArgs &a) {
  if constexpr (sizeof(T) == 2)
    if (a.c.capacity > kFewKeys) return launch_d<T, CODE, false>(a);
  return launch_d<T, CODE, true>(a);
}

template <int PARTS, int CODE>
ns_status weights_sum(const KvAttnArgs &a, const Frag *frags, const float *factors, const float *lse2) {
  const int R = a.d.heads / a.c.heads_kv * a.d.tokens;
  // registers for the operands of that many tiles of rows (64 of them), or 64 keys a wave
  const int tiles = R <= 32 ? 2 : R <= 64 ? 4 : 1 << 20;
  if (tiles * PARTS * a.c.head_dim <= 512) {
    // steps of 32 keys a wave: so many that all waves are on the chip at once, four at most
    const int64_t pieces = (int64_t)(a.c.capacity / 32) * a.c.heads_kv * a.c.batch;
    const int steps = (int)std::max<int64_t>(1, std::min<int64_t>(4, pieces / ((int64_t)device_cu_count() * 16)));
    const dim3 grid((unsigned)((a.c.capacity + 128 * steps - 1) / (128 * steps)), (unsigned)a.c.heads_kv, (unsigned)a.c.batch);
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(256), 0, a.stream, a.c, a.d, a.lengths, a.counts, frags, factors, lse2, a.w_in, a.w_out, steps);
      return check_launch("kv_weights_stream_kernel");
    };
    if (a.c.head_dim == 64) return tiles == 2 ? go(kv_weights_stream_kernel<PARTS, CODE, 64, 2>) : go(kv_weights_stream_kernel<PARTS, CODE, 64, 4>);
    if constexpr (PARTS == 1) {
      if (a.c.head_dim == 256) return go(kv_weights_stream_kernel<PARTS, CODE, 256, 2>);
      if (tiles == 4) return go(kv_weights_stream_kernel<PARTS, CODE, 128, 4>);
    }
    return go(kv_weights_stream_kernel<PARTS, CODE, 128, 2>);
  }
  // a wave has the operands of 64 keys, or 32, in registers.  Its workgroup the same ones, with the rows shared out, where there are fewer
  // than CUs of workgroups with keys of their own (16 heads of 64, 576 rows and keys, all of the call: 35 -> 27 us; 2048 rows, 320 keys: 65 -> 36).
  // Around that border, 512 rows of 16 heads of 64, 128 and 256 channels, all of the call: 240 workgroups 43, 54, 113 us, shared 40, 55, 112; 256 of them
  // 42, 55, 117 and 39, 56, 117; 512 of them 55, 75, 173 and 57, 82, 193; 1040 of them 93, 131, 318 and 95, 140, 348
  constexpr int KX256 = PARTS == 2 ? 2 : 4;
  const int most = a.c.head_dim == 256 ? 64 * KX256 : 256;
  const bool share = (int64_t)((a.c.capacity + most - 1) / most) * a.c.heads_kv * a.c.batch < device_cu_count();
  const int keys = share ? most / 4 : most;
  const dim3 grid((unsigned)((a.c.capacity + keys - 1) / keys), (unsigned)a.c.heads_kv, (unsigned)a.c.batch);
  auto go = [&](auto kernel, auto shared) {
    hipLaunchKernelGGL(share ? shared : kernel, grid, dim3(256), 0, a.stream, a.c, a.d, a.lengths, a.counts, frags, factors, lse2, a.w_in, a.w_out);
    return check_launch("kv_weights_sum_kernel");
  };
  return a.c.head_dim == 64    ? go(kv_weights_sum_kernel<PARTS, CODE, 64, 4, false>, kv_weights_sum_kernel<PARTS, CODE, 64, 4, true>)
         : a.c.head_dim == 128 ? go(kv_weights_sum_kernel<PARTS, CODE, 128, 4, false>, kv_weights_sum_kernel<PARTS, CODE, 128, 4, true>)
                               : go(kv_weights_sum_kernel<PARTS, CODE, 256, KX256, false>, kv_weights_sum_kernel<PARTS, CODE, 256, KX256, true>);
}

}  // namespace

ns_status launch_kv_weights_again(const KvAttnArgs &a, Frag *frags, float *factors, const float *lse2, bool rows) {
  if (rows) {
    const int R = a.d.heads / a.c.heads_kv * a.d.tokens;
    const dim3 grid((unsigned)((R + 63) / 64), (unsigned)a.c.heads_kv, (unsigned)a.c.batch);
    if (a.d.dtype == NS_F32)
      hipLaunchKernelGGL((kv_weights_rows_kernel<float>), grid, dim3(256), 0, a.stream, a.c, a.d, static_cast<const float *>(a.q), frags, factors);
    else
      hipLaunchKernelGGL((kv_weights_rows_kernel<bf16_t>), grid, dim3(256), 0, a.stream, a.c, a.d, static_cast<const bf16_t *>(a.q), frags, factors);
    const ns_status st = check_launch("kv_weights_rows_kernel");
    if (st != NS_OK) return st;
  }
  if (a.d.dtype == NS_F32)
    return a.c.code == NS_CODE_I8 ? weights_sum<2, NS_CODE_I8>(a, frags, factors, lse2) : weights_sum<2, NS_CODE_E4M3>(a, frags, factors, lse2);
  return a.c.code == NS_CODE_I8 ? weights_sum<1, NS_CODE_I8>(a, frags, factors, lse2) : weights_sum<1, NS_CODE_E4M3>(a, frags, factors, lse2);
}

size_t kv_prompt_workspace_bytes(const ns_kv_cache &c, const ns_kv_attn_desc &d, bool weights) { return layout_of(c, d, weights).total; }

ns_status launch_kv_prompt(const KvAttnArgs &a) {
  if (a.d.dtype == NS_F32) return a.c.code == NS_CODE_I8 ? launch_any<float, NS_CODE_I8>(a) : launch_any<float, NS_CODE_E4M3>(a);
  return a.c.code == NS_CODE_I8 ? launch_any<bf16_t, NS_CODE_I8>(a) : launch_any<bf16_t, NS_CODE_E4M3>(a);
}

}  // namespace ns
