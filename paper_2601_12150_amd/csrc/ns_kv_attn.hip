// Attention over the 8-bit key/value cache for few query rows per key/value head (single tokens of a group of heads, a few
// drafted tokens): bound by the reads of the cache.
//
// The rows of a key/value head, r = token * group + head in the group, are the columns of the products
//     S^T = K Q^T   (16 keys x 32 channels  by  32 channels x 16 rows)
//     O^T = V^T P^T (16 channels x 32 keys  by  32 keys x 16 rows)
// so that a lane of the result of the first one holds logits of one row for four keys of every 16, and 32 keys' weights
// are the operand of the second one as they stand: its k index 8 g + j stands for key 4 g + j (j < 4) and 16 + 4 g + j - 4.
// All a wave needs of V then are eight tokens' bytes for its own channels, which it loads as they lie and turns with
// byte permutations; nothing goes through LDS in the loop.  K's channels are taken in an order that makes a lane's 16 bytes two
// operands.
//
// A launch has as many workgroups as the chip holds at once, and each takes an equal share of all sequences' tokens
// (tiles of 128, counted in device memory, so that a recorded graph follows the lengths): partial results of a head that
// several workgroups share are joined by kv_attn_join_kernel.  Small caches are not shared out: a workgroup of eight waves per
// head writes its result itself, in one launch.
//
// The weights that positions are given need the rows' sums, which are known at the end: few rows leave their logits (4 bytes a row and
// key, written and read), more rows have K read again (D bytes a key) by kv_weights_sum_kernel.
#include "ns_kv.h"
#include <algorithm>

namespace ns {

namespace {

constexpr int kThreads = 256, kWaves = 4, kSub = 32, kTile = kWaves * kSub, kMostParts = 1024;

// Sums over the lanes up to and including each
__device__ __forceinline__ int wave_upto(int x, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    x += lane >= o ? y : 0;
  }
  return x;
}
__device__ __forceinline__ int tiles_of(const int32_t *lengths, int b, int batch, int capacity) {
  return b < batch ? (kv_length(lengths, b, capacity) + kTile - 1) / kTile : 0;
}

// The tiles of all sequences and heads, in the order sequence, head, token, shared out over the workgroups (there are fewer than 2^31;
// the host sees to that).  The whole wave calls, with uniform arguments.
struct Tiles {
  const int32_t *lengths;
  int batch, capacity, heads_kv, lane;
  int mine, upto;                                 // of the first 64 sequences: this lane's tiles per head, and with those before
  __device__ __forceinline__ Tiles(const int32_t *lengths, const ns_kv_cache &c, int lane)
      : lengths(lengths), batch(c.batch), capacity(c.capacity), heads_kv(c.heads_kv), lane(lane) {
    mine = tiles_of(lengths, lane, batch, capacity);
    upto = wave_upto(mine, lane);
  }
  // ... of a later 64
  __device__ __forceinline__ void later(int b, int &n, int &to) const {
    n = tiles_of(lengths, b + lane, batch, capacity);
    to = wave_upto(n, lane);
  }
  __device__ __forceinline__ int all() const {
    int sum = __builtin_amdgcn_readlane(upto, 63);
    for (int b = 64; b < batch; b += 64) {
      int n, to;
      later(b, n, to);
      sum += __builtin_amdgcn_readlane(to, 63);
    }
    return sum * heads_kv;
  }
  // tiles per workgroup
  __device__ __forceinline__ int share(int workgroups) const { return kv_share(all(), workgroups); }
  // the tiles of the sequences before b
  __device__ __forceinline__ int before(int b) const {
    if (b == 0) return 0;
    int sum = __builtin_amdgcn_readlane(upto, min(b, 64) - 1);
    for (int x = 64; x < b; x += 64) {
      int n, to;
      later(x, n, to);
      sum += __builtin_amdgcn_readlane(to, min(b - x, 64) - 1);
    }
    return sum * heads_kv;
  }
  // where a tile lies: sequence b, whose tiles of all heads begin at `first`, and its number of tiles per head
  __device__ __forceinline__ void place(int tile, int &b, int &tiles, int &first) const {
    first = 0;
    int n = mine, to = upto;
    for (int x = 0; x < batch; x += 64) {
      if (x) later(x, n, to);
      const unsigned long long past = __ballot(first + to * heads_kv > tile);
      if (past) {
        const int at = __ffsll((long long)past) - 1;
        tiles = __builtin_amdgcn_readlane(n, at);
        first += (__builtin_amdgcn_readlane(to, at) - tiles) * heads_kv;
        b = x + at;
        return;
      }
      first += __builtin_amdgcn_readlane(to, 63) * heads_kv;
    }
    b = 0;                                        // (not reached: the tile is one of them)
    tiles = 1;
  }
};

// What the launches leave for each other.
struct SplitArgs {
  float *part_o, *part_ml;         // records [workgroup + head][R] of D floats / (reference, sum)
  float *lse2;                     // [B Hkv][R]: log2 of the rows' sums, +inf for a row that sees nothing
  float *logits;                   // nullable [B Hkv][R][capacity], times log2 e
  Frag *frags;                     // nullable: operands and factors of the weights' second pass
  float *factors;
  const float *w_in;
  float *w_out;
  int workgroups;
};

// The weights of the positions n0 .. n0 + 3 from the rows' logits.
__device__ __forceinline__ void weigh(const ns_kv_cache &c, const ns_kv_attn_desc &d, const SplitArgs &a, int64_t row, int n0, int length, int count,
                                      const float *lse2 /* [R], in LDS */) {
  const int G = d.heads / c.heads_kv, R = G * d.tokens;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  if (n0 < length) {
    int t = 0, g = 0;
    for (int r = 0; r < R; r++) {
      const int limit = kv_seen(d, t, length, count);
      const f32x4 z = *reinterpret_cast<const f32x4 *>(a.logits + (row * R + r) * c.capacity + n0);
#pragma unroll
      for (int i = 0; i < 4; i++) sum[i] += n0 + i < limit ? __builtin_amdgcn_exp2f(z[i] - lse2[r]) : 0.f;
      if (++g == G) g = 0, t++;
    }
  }
  const int64_t at = row * c.capacity + n0;
#pragma unroll
  for (int i = 0; i < 4; i++)
    if (n0 + i < length || a.w_in != a.w_out) a.w_out[at + i] = (a.w_in ? a.w_in[at + i] : 0.f) + sum[i];
}

// Workgroups of four waves that a CU holds, by registers: more of them have more loads on their way.
constexpr int per_cu(bool f32, int D, int NT) { return NT * D <= 128 || (!f32 && D == 128 && NT == 2) ? 2 : 1; }

// T: float takes its queries, and the weights, as the sum of two fp16 numbers.  ALONE: a workgroup has a head to itself.
// Measured, bf16, 128 channels, 4 rows a head: 131001 tokens of 8 heads 46 us (268 MB and 17 MB of logits, 6.2 TB/s); a workgroup for each of
// 8 heads of 32 sequences of 63708 tokens together 33 us (131 MB, 3.9 TB/s; the longest one sets it).  32 rows: 58990 tokens of 8 heads 32 us (121 MB, 3.7).
template <typename T, int CODE, int D, int NT, int WAVES, bool ALONE>
__global__ __launch_bounds__(WAVES * 64, ALONE ? (D == 256 ? 1 : 2) : per_cu(sizeof(T) == 4, D, NT))
void kv_attn_split_kernel(ns_kv_cache c, ns_kv_attn_desc d, const T *q, const int32_t *lengths, const int32_t *counts, T *out, float *lse, SplitArgs a) {
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1, KS = D / 32, DT = D / 16, VW = D / 64;   // k steps, channel tiles, dwords of V a token
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int G = d.heads / c.heads_kv, R = G * d.tokens;
  __shared__ __attribute__((aligned(16))) float sh_o[WAVES][16][D + 4];
  __shared__ float sh_m[WAVES][16], sh_l[WAVES][16], sh_lse2[ALONE ? 16 * NT : 1];

  const int lblock = 31 - __clz(c.block);
  const Tiles tiles_all(lengths, c, lane);
  int u = 0, u_end = 1;
  if constexpr (!ALONE) {
    const int share = tiles_all.share(gridDim.x), total = tiles_all.all();
    if ((int)blockIdx.x > (total - 1) / share || total == 0) return;
    u = share * (int)blockIdx.x;
    u_end = total - u < share ? total : u + share;
  }

  // ---- the piece of a head's tokens in hand, and codes on their way
  int b = 0, h = 0, n_lo = 0, n_hi = 0, done = 1, length = 0, count = 0;
  int64_t row = 0;
  const uint8_t *kb = nullptr, *vb = nullptr;
  const float *ks = nullptr, *vs = nullptr;
  auto piece_at = [&](int tile) {
    if constexpr (ALONE) {
      b = (int)blockIdx.y;
      h = (int)blockIdx.x;
      length = kv_length(lengths, b, c.capacity);
      n_hi = length;
    } else {
      int tiles, first;
      tiles_all.place(tile, b, tiles, first);
      h = (int)((unsigned)(tile - first) / (unsigned)tiles);
      const int t0 = tile - first - h * tiles;
      done = min(tiles - t0, u_end - tile);
      length = kv_length(lengths, b, c.capacity);
      n_lo = t0 * kTile;
      n_hi = min(length, (t0 + done) * kTile);
    }
    count = kv_count(counts, b, d.tokens);
    row = (int64_t)b * c.heads_kv + h;
    kb = static_cast<const uint8_t *>(c.k) + b * c.stride_b + h * c.stride_h;
    vb = static_cast<const uint8_t *>(c.v) + b * c.stride_b + h * c.stride_h;
    ks = c.k_scale + row * (c.capacity >> lblock);
    vs = c.v_scale + row * (c.capacity >> lblock);
  };
  const uint32_t k_off = (uint32_t)n16 * (uint32_t)c.stride_t + 16 * g, v_off = 4 * (uint32_t)g * (uint32_t)c.stride_t + (uint32_t)n16 * (D / 16);
  u32x4 kw[2][D / 64];
  uint32_t vw[8][VW];
  float skey, sval;
  auto fetch = [&](int n0) {
    // (uniform bases and one offset: else the compiler advances an address of 64 bits for every load)
    const uint8_t *kp = kb + (int64_t)n0 * c.stride_t, *vp = vb + (int64_t)n0 * c.stride_t;
    const uint32_t ko = (uint32_t)opaque((int)k_off), vo = (uint32_t)opaque((int)v_off);
#pragma unroll
    for (int x = 0; x < 2; x++)
#pragma unroll
      for (int i = 0; i < D / 64; i++) kw[x][i] = *reinterpret_cast<const u32x4 *>(kp + (int64_t)x * 16 * c.stride_t + 64 * i + ko);
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const uint8_t *p = vp + (int64_t)((j >> 2) * 16 + (j & 3)) * c.stride_t + vo;
      if constexpr (VW == 1) {
        vw[j][0] = *reinterpret_cast<const uint32_t *>(p);
      } else if constexpr (VW == 2) {
        const u32x2 w = *reinterpret_cast<const u32x2 *>(p);
        vw[j][0] = w[0]; vw[j][1] = w[1];
      } else {
        const u32x4 w = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
        for (int i = 0; i < 4; i++) vw[j][i] = w[i];
      }
    }
    skey = ks[n0 >> lblock];
    sval = vs[n0 >> lblock];
  };
  constexpr int kStep = WAVES * kSub;
  int n0 = 0;
  auto begin = [&](int tile) {
    piece_at(tile);
    n0 = n_lo + wave * kSub;
    if (n0 < n_hi) fetch(n0);
  };
  begin(u);
  while (true) {

    // ---- the rows' queries
    Frag qf[NT][PARTS][KS];
    float factor[NT];
    int limit[NT], least = 0x7fffffff;            // least: keys from here on are masked in some row
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      const int r = nt * 16 + n16;
      const bool real = r < R;
      const int t = real ? r / G : 0;
      limit[nt] = real ? kv_seen(d, t, length, count) : 0;
      if (real) least = min(least, limit[nt]);
      const T *p = q + b * d.q_stride_b + (int64_t)(h * G + (real ? r - t * G : 0)) * d.q_stride_h + (int64_t)t * d.q_stride_t;
      f32x4 x[D / 16];
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < D / 16; i++) {
        x[i] = load4(p + 64 * (i / 4) + 16 * g + 4 * (i % 4));
#pragma unroll
        for (int j = 0; j < 4; j++) {
          x[i][j] = real ? x[i][j] : 0.f;
          most = max(most, __float_as_uint(x[i][j]) & 0x7fffffffu);
        }
      }
      most = max(most, (uint32_t)__shfl_xor((int)most, 16));
      most = max(most, (uint32_t)__shfl_xor((int)most, 32));
      const int shift = kv_row_shift(most);
      factor[nt] = ldexpf(d.scale, -shift) * kLog2e;
#pragma unroll
      for (int i = 0; i < D / 16; i++)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const float x0 = ldexpf(x[i][j], shift), x1 = ldexpf(x[i][j + 1], shift);
          const uint32_t hi = pack_f16(x0, x1);
          qf[nt][0][i / 2].w[(i % 2) * 2 + j / 2] = hi;
          if (PARTS == 2) {
            const f16x2 w = __builtin_bit_cast(f16x2, hi);
            qf[nt][PARTS - 1][i / 2].w[(i % 2) * 2 + j / 2] = pack_f16(x0 - (float)w[0], x1 - (float)w[1]);
          }
        }
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) least = min(least, __shfl_xor(least, o));
    least = __builtin_amdgcn_readfirstlane(least);

    // ---- its tokens, 32 at a time
    f32x4 o[NT][DT];
    float m[NT], l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      m[nt] = -INFINITY;
      l[nt] = 0.f;
#pragma unroll
      for (int i = 0; i < DT; i++) o[nt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (; n0 < n_hi; n0 += kStep) {
      const bool edge = n0 + kSub > least;
      uint32_t vt[VW][8];                           // V's dwords on to other registers, so that the next tokens' loads can be under way
#pragma unroll
      for (int j = 0; j < 8; j++)
#pragma unroll
        for (int i = 0; i < VW; i++) vt[i][j] = vw[j][i];
      if (edge) {                                   // what lies behind the length may be NaN
        asm volatile("; edge");                     // (a branch, not selects in every step)
#pragma unroll
        for (int j = 0; j < 8; j++)
#pragma unroll
          for (int i = 0; i < VW; i++) vt[i][j] = n0 + (j >> 2) * 16 + 4 * g + (j & 3) < length ? vt[i][j] : 0u;
      }
      const float sk = skey, sv = sval;
      f32x4 sx[NT][2];
#pragma unroll
      for (int x = 0; x < 2; x++) {
        Frag kf[KS];
#pragma unroll
        for (int k = 0; k < KS; k++) kf[k] = kv_frag<CODE>(kw[x][k / 2][2 * (k % 2)], kw[x][k / 2][2 * (k % 2) + 1]);
        if (x == 1 && n0 + kStep < n_hi) fetch(n0 + kStep);      // (two steps ahead instead of one: no faster)
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
          sx[nt][x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int pt = PARTS - 1; pt >= 0; pt--)
#pragma unroll
            for (int k = 0; k < KS; k++) sx[nt][x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[k].v, qf[nt][pt][k].v, sx[nt][x], 0, 0, 0);
        }
        if (NT > 1) __builtin_amdgcn_sched_barrier(0);
      }

      Frag pf[NT][PARTS];
      float svr[NT];
#pragma unroll
      for (int nt = 0; nt < NT; nt++) {
        const f32x4 (&s)[2] = sx[nt];
        const float f = factor[nt] * sk;
        if (a.logits && nt * 16 + n16 < R) {
#pragma unroll
          for (int x = 0; x < 2; x++)
            *reinterpret_cast<f32x4 *>(a.logits + (row * R + nt * 16 + n16) * c.capacity + n0 + 16 * x + 4 * g) = s[x] * f;
        }
        const bool fresh = m[nt] == -INFINITY;                                         // this row has seen no key yet
        const float ref = fresh ? 0.f : m[nt];
        float z[8], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; i++) z[i] = __builtin_fmaf(s[i / 4][i % 4], f, -ref);
        svr[nt] = sv * (1.f / Lift<true>::factor);
        if (edge) {
          asm volatile("; edge");
#pragma unroll
          for (int i = 0; i < 8; i++) z[i] = n0 + (i / 4) * 16 + 4 * g + i % 4 < limit[nt] ? z[i] : -INFINITY;
          svr[nt] = n0 >= limit[nt] ? 0.f : svr[nt];                                   // a NaN block is NaN for those who see it
        }
#pragma unroll
        for (int i = 0; i < 8; i++) top = fmaxf(top, z[i]);
        if (__any(top > Lift<true>::room || (fresh && top > -INFINITY))) {
          top = half_swap_max(row_swap_max(top));
          const bool moved = top > Lift<true>::room || (fresh && top > -INFINITY);
          const float move = moved ? top : 0.f;
          // (a fresh row's sums are 0, or NaN: not times a factor beyond fp32 where its logits are far below 0)
          const float fade = __builtin_amdgcn_exp2f(fminf(-move, 0.f));
#pragma unroll
          for (int i = 0; i < 8; i++) z[i] -= move;
          if (moved) m[nt] = ref + move;
          l[nt] *= fade;
#pragma unroll
          for (int i = 0; i < DT; i++) o[nt][i] *= fade;
        }
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
          p[i] = __builtin_amdgcn_exp2f(z[i]);
          l[nt] += p[i];
          p[i] *= Lift<true>::factor;
        }
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const uint32_t hi = pack_f16(p[i], p[i + 1]);
          pf[nt][0].w[i / 2] = hi;
          if (PARTS == 2) {
            const f16x2 w = __builtin_bit_cast(f16x2, hi);
            pf[nt][PARTS - 1].w[i / 2] = pack_f16(p[i] - (float)w[0], p[i + 1] - (float)w[1]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < VW; i++) {
        Frag vf[4];
        kv_frags_t<CODE>(vt[i], vf);
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
          for (int nt = 0; nt < NT; nt++) {
            f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int pt = PARTS - 1; pt >= 0; pt--) y = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[j].v, pf[nt][pt].v, y, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; e++) o[nt][4 * i + j][e] = __builtin_fmaf(y[e], svr[nt], o[nt][4 * i + j][e]);
          }
        if (VW > 1) __builtin_amdgcn_sched_barrier(0);
      }
    }

    // ---- the next piece's first tokens on their way; the waves' results together, and out: record (blockIdx.x + row) of the joined head
    const int64_t out_row = row, slot = (int64_t)blockIdx.x + row;
    const int out_b = b, out_h = h, out_length = length, out_count = count;
    u += done;
    if (!ALONE && u < u_end) begin(u);
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      const float ls = half_swap_sum(row_swap_sum(l[nt]));
      if (g == 0) {
        sh_m[wave][n16] = m[nt] == -INFINITY && ls != ls ? 0.f : m[nt];      // a row of NaN is not an empty one
        sh_l[wave][n16] = ls;
      }
      // a lane's channels: (4 g + e) * DT + i
#pragma unroll
      for (int e = 0; e < 4; e++)
#pragma unroll
        for (int i = 0; i < DT; i += 4)
          *reinterpret_cast<f32x4 *>(&sh_o[wave][n16][(4 * g + e) * DT + i]) = f32x4{o[nt][i][e], o[nt][i + 1][e], o[nt][i + 2][e], o[nt][i + 3][e]};
      __syncthreads();
      for (int x = tid; x < 16 * D / 4; x += WAVES * 64) {
        const int n = x / (D / 4), dd = x % (D / 4) * 4, r = nt * 16 + n;
        if (r < R) {
          float M = sh_m[0][n];
#pragma unroll
          for (int w = 1; w < WAVES; w++) M = fmaxf(M, sh_m[w][n]);
          f32x4 y = {0.f, 0.f, 0.f, 0.f};
          float ll = 0.f;
#pragma unroll
          for (int w = 0; w < WAVES; w++) {
            const float fade = __builtin_amdgcn_exp2f(sh_m[w][n] - M);
            if (sh_m[w][n] != -INFINITY) {
              y += *reinterpret_cast<const f32x4 *>(&sh_o[w][n][dd]) * fade;
              ll += sh_l[w][n] * fade;
            }
          }
          if constexpr (ALONE) {
            const bool some = M != -INFINITY;
            const int t = r / G, hq = out_h * G + r - t * G;
            const float inv = some ? 1.f / ll : 0.f;
#pragma unroll
            for (int e = 0; e < 4; e++) y[e] = some ? y[e] * inv : 0.f;
            store4(out + out_b * d.out_stride_b + (int64_t)hq * d.out_stride_h + (int64_t)t * d.out_stride_t + dd, y);
            if (dd == 0) {
              const float z2 = some ? M + __log2f(ll) : -INFINITY;
              if (lse) lse[((int64_t)out_b * d.heads + hq) * d.tokens + t] = z2 * kLn2;
              sh_lse2[r] = some ? z2 : INFINITY;
              if (a.frags) a.lse2[out_row * R + r] = sh_lse2[r];
            }
          } else {
            *reinterpret_cast<f32x4 *>(a.part_o + (slot * R + r) * D + dd) = y;
            if (dd == 0) *reinterpret_cast<f32x2 *>(a.part_ml + (slot * R + r) * 2) = f32x2{M, ll};
          }
        }
      }
      __syncthreads();
    }
    if constexpr (ALONE) {
      if (a.logits)
        for (int n = tid * 4; n < c.capacity && (n < out_length || a.w_in != a.w_out); n += WAVES * 64 * 4)
          weigh(c, d, a, out_row, n, out_length, out_count, sh_lse2);
    }
    if (ALONE || u >= u_end) break;
  }
}

// The first R workgroups of a head: a row's joined result each.  The others: the weights of 1024 positions each from the rows'
// logits, or the operands for the weights' second pass.  Bound by latency: 8 to 10 us.
template <typename T>
__global__ __launch_bounds__(kThreads) void kv_attn_join_kernel(ns_kv_cache c, ns_kv_attn_desc d, const T *q, const int32_t *lengths,
                                                                const int32_t *counts, T *out, float *lse, SplitArgs a) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, D = c.head_dim;
  const int G = d.heads / c.heads_kv, R = G * d.tokens;
  const int x = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int64_t row = (int64_t)b * c.heads_kv + h;
  __shared__ __attribute__((aligned(16))) float sh[kThreads * 4];
  __shared__ float fades[kMostParts], sh_w[2 * kWaves], lse2[64];
  if (x >= R && a.frags) {
    const int tile = (x - R) * kWaves + wave;
    if (tile < (R + 15) / 16) kv_rows_tile(c, d, q, b, h, tile, lane, a.frags, a.factors);
    return;
  }

  // this head's records
  const Tiles tiles_all(lengths, c, lane);
  const int share = tiles_all.share(a.workgroups);
  const int tiles = tiles_of(lengths, b, c.batch, c.capacity), lo = tiles_all.before(b) + h * tiles;
  const int first = lo / share, parts = tiles ? (lo + tiles - 1) / share - first + 1 : 0;
  const int64_t slot = first + row;

  if (x >= R) {
    for (int r = wave; r < R; r += kWaves) {
      float M = -INFINITY, L = 0.f;
      for (int p = lane; p < parts; p += 64) M = fmaxf(M, a.part_ml[((slot + p) * R + r) * 2]);
      M = wave_max(M);
      for (int p = lane; p < parts; p += 64) {
        const f32x2 ml = *reinterpret_cast<const f32x2 *>(a.part_ml + ((slot + p) * R + r) * 2);
        L += ml[0] == -INFINITY ? 0.f : ml[1] * __builtin_amdgcn_exp2f(ml[0] - M);
      }
      L = wave_sum(L);
      if (lane == 0) lse2[r] = M == -INFINITY ? INFINITY : M + __log2f(L);
    }
    __syncthreads();
    const int n = ((x - R) * kThreads + tid) * 4, length = kv_length(lengths, b, c.capacity);
    if (n < c.capacity && (n < length || a.w_in != a.w_out)) weigh(c, d, a, row, n, length, kv_count(counts, b, d.tokens), lse2);
    return;
  }

  const int r = x, quads = D / 4, slices = kThreads / quads, s = tid / quads, dd = tid % quads * 4;
  const float *records = a.part_o + (slot * R + r) * D + dd, *mls = a.part_ml + (slot * R + r) * 2;
  constexpr int kAhead = 4;                         // records that are loaded before it is known what they are multiplied with
  f32x4 v[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; i++) v[i] = s + i * slices < parts ? *reinterpret_cast<const f32x4 *>(records + (int64_t)(s + i * slices) * R * D) : f32x4{0.f, 0.f, 0.f, 0.f};
  float M = -INFINITY, L = 0.f;
  f32x2 own = {-INFINITY, 0.f};                     // (as a rule there are no more records than threads)
  for (int p = tid; p < parts; p += kThreads) {
    own = *reinterpret_cast<const f32x2 *>(mls + (int64_t)p * R * 2);
    M = fmaxf(M, own[0]);
  }
  M = wave_max(M);
  if (lane == 0) sh_w[wave] = M;
  __syncthreads();
  M = fmaxf(fmaxf(sh_w[0], sh_w[1]), fmaxf(sh_w[2], sh_w[3]));
  for (int p = tid; p < parts; p += kThreads) {
    if (parts > kThreads) own = *reinterpret_cast<const f32x2 *>(mls + (int64_t)p * R * 2);
    const float fade = own[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(own[0] - M);
    fades[p] = fade;
    L += own[0] == -INFINITY ? 0.f : own[1] * fade;
  }
  L = wave_sum(L);
  if (lane == 0) sh_w[kWaves + wave] = L;
  __syncthreads();
  L = (sh_w[kWaves] + sh_w[kWaves + 1]) + (sh_w[kWaves + 2] + sh_w[kWaves + 3]);
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kAhead; i++)
    if (s + i * slices < parts) y += v[i] * fades[s + i * slices];
#pragma unroll 4
  for (int p = s + kAhead * slices; p < parts; p += slices) y += *reinterpret_cast<const f32x4 *>(records + (int64_t)p * R * D) * fades[p];
  *reinterpret_cast<f32x4 *>(&sh[tid * 4]) = y;
  __syncthreads();
  if (tid < quads) {
    for (int i = 1; i < slices; i++) y += *reinterpret_cast<const f32x4 *>(&sh[(i * quads + tid) * 4]);
    const bool some = M != -INFINITY;
    const float inv = some ? 1.f / L : 0.f;
    const int t = r / G, hq = h * G + r - t * G;
#pragma unroll
    for (int e = 0; e < 4; e++) y[e] = some ? y[e] * inv : 0.f;
    store4(out + b * d.out_stride_b + (int64_t)hq * d.out_stride_h + (int64_t)t * d.out_stride_t + dd, y);
    if (tid == 0) {
      const float z2 = some ? M + __log2f(L) : -INFINITY;
      if (lse) lse[((int64_t)b * d.heads + hq) * d.tokens + t] = z2 * kLn2;
      if (a.frags) a.lse2[row * R + r] = some ? z2 : INFINITY;
    }
  }
}

// ---- host side

int rows_of(const ns_kv_cache &c, const ns_kv_attn_desc &d) { return d.heads / c.heads_kv * d.tokens; }

// Row tiles of 16 that there are registers for
constexpr int most_tiles(int head_dim) { return head_dim == 256 ? 1 : head_dim == 128 ? 2 : 4; }
// More rows are a prompt: the operands of another tile have no registers here.  Both kernels, 32 heads' 16384 tokens: 16 and 32 rows of 64
// channels 20 and 23 us against a prompt's 29 and 29, of 128 30 and 35 against 52 and 53, 16 of 256 54 against 128; 8 heads' 8192 tokens 32 rows of
// 128 20.7 against 21.1 (fp32 19 against 25), 16 of 256 19 against 40.  What this does not tell apart: 17 to 32 rows of very many heads with few
// tokens each, where a prompt would be faster (512 heads' 512 tokens, 32 rows: 46 against 16 us of 64 channels, 54 against 35 of 128).
// Of channels of 64 three and four tiles are bound by the products here, which prompts share out better: 45 us against 33
// for 64 heads' 8192 tokens, 41 against 13 for 256 heads' 512.  Where there are few heads of many tokens this has more workgroups, by which its
// finer shares win: 19 us against 37 for one head's 65536 tokens, 17 against 20 for 8 heads' 8192, 14 against 16 for 8 heads' 1024.
bool few_rows(const ns_kv_cache &c, const ns_kv_attn_desc &d) {
  const int tiles = (rows_of(c, d) + 15) / 16;
  if (tiles <= 2) return tiles <= most_tiles(c.head_dim);
  return tiles <= most_tiles(c.head_dim) && c.capacity >= 1024 && (int64_t)c.batch * c.heads_kv * 16 < device_cu_count();
}

// Weights: logits are 8 bytes a row and key, written and read; K read again is D bytes a key, its products and a launch.  32 heads' 16384
// tokens, logits against K again: 8 rows of 64 channels 26.5 us against 28.5, 16 rows 35.9 against 29.2; of 128 channels 36.6 against 44.8 and
// 46.1 against 45.7 (8 heads' 131072: 4 rows 56 against 76, 16 rows 87 against 77); 16 rows of 256 channels 77 against 82.
bool by_logits(const ns_kv_cache &c, const ns_kv_attn_desc &d) { return rows_of(c, d) <= (c.head_dim == 256 ? 16 : 10); }
// A workgroup per sequence and head, which spares the records and their join: where a head's tokens are few (8 heads' 1024 of 64 channels 7.5 us
// against 9.1 shared out, 2048: 11.1 against 9.2; 512 of 128 channels 8.2 against 9.8, 1024: 11.0 against 9.8), and where there is one
// for every CU (256 heads' 4096 of 128 channels 43.5 against 49.8; of more tokens, still 98.5 against 104.9 for 8192, a single long sequence
// among short ones would have its heads' workgroups run alone for too long).  That happens with room for 4096 as well, where the lengths are
// that far apart: 32 sequences' 8 heads of 128 channels, all 4096 tokens long 43 us against 50 shared out, all 2048 24 against 30, all 102 6
// against 12, but one of 4096 among 31 of 102 28 against 13 (256 channels: 94 and 102, 44 and 52, 7 and 14, 58 and 19).
bool alone(const ns_kv_cache &c, const ns_kv_attn_desc &d) {
  return rows_of(c, d) <= 16 && ((int64_t)c.capacity * c.head_dim <= 65536 || (c.capacity <= 4096 && (int64_t)c.batch * c.heads_kv >= device_cu_count()));
}

struct Layout { size_t o, ml, lse2, logits, frags, factors, total; int workgroups; };
Layout layout_of(const ns_kv_cache &c, const ns_kv_attn_desc &d, bool weights) {
  Layout w{};
  const bool shared = !alone(c, d), logits = weights && by_logits(c, d), again = weights && !logits;
  const size_t rows = rows_of(c, d), heads = (size_t)c.batch * c.heads_kv;
  const int nt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  w.workgroups = std::min(per_cu(d.dtype == NS_F32, c.head_dim, nt) * device_cu_count(), kMostParts);
  const size_t slots = (size_t)w.workgroups + heads;
  size_t off = 0;
  auto take = [&](bool wanted, size_t bytes) {
    const size_t was = off;
    off += wanted ? align_up(bytes, 256) : 0;
    return was;
  };
  w.o = take(shared, slots * rows * c.head_dim * 4);
  w.ml = take(shared, slots * rows * 8);
  w.lse2 = take(again, heads * rows * 4);
  w.logits = take(logits, heads * rows * (size_t)c.capacity * 4);
  w.frags = take(again, again ? kv_rows_frag_bytes(c, d) : 0);
  w.factors = take(again, again ? kv_rows_factor_bytes(c, d) : 0);
  w.total = off;
  return w;
}

template <typename T, int CODE, int D, int NT>
ns_status launch_split(const KvAttnArgs &a) {
  const ns_kv_cache &c = a.c;
  const bool weights = a.w_out != nullptr, logits = weights && by_logits(c, a.d), again = weights && !logits;
  const Layout w = layout_of(c, a.d, weights);
  auto at = [&](size_t off) { return reinterpret_cast<float *>(a.ws + off); };
  SplitArgs s{at(w.o), at(w.ml), at(w.lse2), logits ? at(w.logits) : nullptr, again ? reinterpret_cast<Frag *>(a.ws + w.frags) : nullptr, at(w.factors),
              a.w_in, a.w_out, w.workgroups};
  const T *q = static_cast<const T *>(a.q);
  T *out = static_cast<T *>(a.out);
  if constexpr (NT == 1)
    if (alone(c, a.d)) {
      constexpr int WAVES = D == 256 ? 4 : 8;       // (LDS)
      hipLaunchKernelGGL((kv_attn_split_kernel<T, CODE, D, NT, WAVES, true>), dim3((unsigned)c.heads_kv, (unsigned)c.batch), dim3(WAVES * 64), 0, a.stream, c, a.d, q,
                         a.lengths, a.counts, out, a.lse, s);
      const ns_status st = check_launch("kv_attn_split_kernel");
      if (st != NS_OK || !again) return st;
      return launch_kv_weights_again(a, s.frags, s.factors, s.lse2, true);
    }
  hipLaunchKernelGGL((kv_attn_split_kernel<T, CODE, D, NT, kWaves, false>), dim3((unsigned)w.workgroups), dim3(kThreads), 0, a.stream, c, a.d, q, a.lengths,
                     a.counts, out, a.lse, s);
  ns_status st = check_launch("kv_attn_split_kernel");
  if (st != NS_OK) return st;
  const int rows = rows_of(c, a.d), more = logits ? (c.capacity + 4 * kThreads - 1) / (4 * kThreads) : again ? 1 : 0;
  hipLaunchKernelGGL((kv_attn_join_kernel<T>), dim3((unsigned)(rows + more), (unsigned)c.heads_kv, (unsigned)c.batch), dim3(kThreads), 0, a.stream,
                     c, a.d, q, a.lengths, a.counts, out, a.lse, s);
  st = check_launch("kv_attn_join_kernel");
  if (st != NS_OK || !again) return st;
  return launch_kv_weights_again(a, s.frags, s.factors, s.lse2, false);
}

template <typename T, int CODE, int D>
ns_status launch_tiles(const KvAttnArgs &a) {
  constexpr int most = most_tiles(D);
  const int nt = (rows_of(a.c, a.d) + 15) / 16;
  if constexpr (most >= 4)
    if (nt > 2) return launch_split<T, CODE, D, 4>(a);
  if constexpr (most >= 2)
    if (nt > 1) return launch_split<T, CODE, D, 2>(a);
  return launch_split<T, CODE, D, 1>(a);
}

template <typename T, int CODE>
ns_status launch_any(const KvAttnArgs &a) {
  if (!few_rows(a.c, a.d)) return launch_kv_prompt(a);
  return a.c.head_dim == 64 ? launch_tiles<T, CODE, 64>(a) : a.c.head_dim == 128 ? launch_tiles<T, CODE, 128>(a) : launch_tiles<T, CODE, 256>(a);
}

}  // namespace

size_t kv_attn_workspace_bytes(const ns_kv_cache &c, const ns_kv_attn_desc &d, bool weights) {
  return few_rows(c, d) ? layout_of(c, d, weights).total : kv_prompt_workspace_bytes(c, d, weights);
}

ns_status launch_kv_attn(const KvAttnArgs &a) {
  if (a.d.dtype == NS_F32) return a.c.code == NS_CODE_I8 ? launch_any<float, NS_CODE_I8>(a) : launch_any<float, NS_CODE_E4M3>(a);
  return a.c.code == NS_CODE_I8 ? launch_any<bf16_t, NS_CODE_I8>(a) : launch_any<bf16_t, NS_CODE_E4M3>(a);
}

}  // namespace ns
