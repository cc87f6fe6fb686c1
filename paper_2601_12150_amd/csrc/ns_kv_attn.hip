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
// Every launch has as many workgroups as the chip holds at once, and each takes an equal share of all sequences' tokens
// (tiles of 128, counted in device memory, so that a recorded graph follows the lengths): partial results of a head that
// several workgroups share are joined by kv_attn_join_kernel.
#include "ns_kv.h"

namespace ns {

namespace {

constexpr int kThreads = 256, kWaves = 4, kSub = 32, kTile = kWaves * kSub;
// Weights are 2^(z - m + 11) in fp16, m a logit near the largest so far, which is moved up before they pass 2^15: a weight that is the
// largest one's 2^-25 or more keeps its 11 bits, and below it all are within 2^-36 of the largest.
constexpr float kLift = 11.f, kRoom = 15.f;

struct Span { int64_t lo, hi; };                  // tiles of this workgroup

// Sum over the wave of a small count
__device__ __forceinline__ int wave_total(int x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

__device__ __forceinline__ int tiles_of(const int32_t *lengths, int b, int batch, int capacity) {
  return b < batch ? (kv_length(lengths, b, capacity) + kTile - 1) / kTile : 0;
}

// Tiles of all sequences (one head).  The whole wave calls.
__device__ __forceinline__ int64_t all_tiles(const int32_t *lengths, int batch, int capacity, int lane) {
  int64_t sum = 0;
  for (int b = 0; b < batch; b += 64) sum += wave_total(tiles_of(lengths, b + lane, batch, capacity));
  return sum;
}

// Where a tile lies: sequence b, whose tiles of all heads begin at `first`, and its number of tiles per head.
struct Place { int b, tiles; int64_t first; };
__device__ __forceinline__ Place place_of(const int32_t *lengths, int batch, int capacity, int heads_kv, int64_t tile, int lane) {
  int64_t first = 0;
  for (int b = 0; b < batch; b += 64) {
    const int mine = tiles_of(lengths, b + lane, batch, capacity);
    int upto = mine;                              // tiles of this lane's sequence and those before
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o);
      upto += lane >= o ? x : 0;
    }
    const unsigned long long past = __ballot(first + (int64_t)upto * heads_kv > tile);
    if (past) {
      const int at = __ffsll((long long)past) - 1, n = __shfl(mine, at);
      return Place{b + at, n, first + (int64_t)(__shfl(upto, at) - n) * heads_kv};
    }
    first += (int64_t)__shfl(upto, 63) * heads_kv;
  }
  return Place{batch, 0, first};
}

// tiles per workgroup
__device__ __forceinline__ int64_t share_of(int64_t total, int workgroups) { return (total + workgroups - 1) / workgroups; }

template <typename T> __device__ __forceinline__ f32x4 load4(const T *p);
template <> __device__ __forceinline__ f32x4 load4<float>(const float *p) { return *reinterpret_cast<const f32x4 *>(p); }
template <> __device__ __forceinline__ f32x4 load4<bf16_t>(const bf16_t *p) {
  const u32x2 w = *reinterpret_cast<const u32x2 *>(p);
  return f32x4{bf16_lo(w[0]), bf16_hi(w[0]), bf16_lo(w[1]), bf16_hi(w[1])};
}

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
}

// PARTS: 1 for bf16 queries, 2 for fp32 ones (a number as the sum of two in fp16)
template <typename T, int CODE, int D, int NT>
__global__ __launch_bounds__(kThreads, NT * D <= 128 ? 2 : 1) void kv_attn_split_kernel(ns_kv_cache c, ns_kv_attn_desc d, const T *q, const int32_t *lengths,
                                                                    const int32_t *counts, float *part_o, float *part_ml, float *logits) {
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1, KS = D / 32, DT = D / 16, VW = D / 64;   // k steps, channel tiles, dwords of V a token
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int G = d.heads / c.heads_kv, R = G * d.tokens;
  __shared__ __attribute__((aligned(16))) float sh_o[kWaves][16][D + 4];
  __shared__ float sh_m[kWaves][16], sh_l[kWaves][16];

  const int64_t total = all_tiles(lengths, c.batch, c.capacity, lane) * c.heads_kv;
  const int64_t share = share_of(total, gridDim.x);
  int64_t u = share * blockIdx.x;
  const int64_t u_end = min(u + share, total);
  if (u >= u_end) return;
  Place at = place_of(lengths, c.batch, c.capacity, c.heads_kv, u, lane);

  while (u < u_end) {
    if (u >= at.first + (int64_t)at.tiles * c.heads_kv) at = place_of(lengths, c.batch, c.capacity, c.heads_kv, u, lane);
    const int b = __builtin_amdgcn_readfirstlane(at.b), tiles = __builtin_amdgcn_readfirstlane(at.tiles);
    const int h = __builtin_amdgcn_readfirstlane((int)((u - at.first) / tiles));
    const int t0 = __builtin_amdgcn_readfirstlane((int)((u - at.first) - (int64_t)h * tiles));
    const int t1 = (int)min((int64_t)tiles, t0 + (u_end - u));
    const int length = kv_length(lengths, b, c.capacity), count = kv_count(counts, b, d.tokens);
    const int64_t row = (int64_t)b * c.heads_kv + h;

    // ---- the rows' queries
    Frag qf[NT][PARTS][KS];
    float factor[NT];
    int limit[NT];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      const int r = nt * 16 + n16;
      const bool real = r < R;
      const int t = real ? r / G : 0;
      limit[nt] = real ? kv_seen(d, t, length, count) : 0;
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
      factor[nt] = ldexpf(d.scale * kLog2e, -shift);
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
    int least = limit[0];                         // keys from here on are masked in some row
#pragma unroll
    for (int nt = 0; nt < NT; nt++)
      if (nt * 16 + n16 < R) least = min(least, limit[nt]);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) least = min(least, __shfl_xor(least, o));
    least = __builtin_amdgcn_readfirstlane(least);

    // ---- its tokens, 32 at a time
    const uint8_t *kb = static_cast<const uint8_t *>(c.k) + b * c.stride_b + h * c.stride_h;
    const uint8_t *vb = static_cast<const uint8_t *>(c.v) + b * c.stride_b + h * c.stride_h;
    const float *ks = c.k_scale + row * (c.capacity / c.block), *vs = c.v_scale + row * (c.capacity / c.block);
    const int lblock = 31 - __clz(c.block);
    f32x4 o[NT][DT];
    float m[NT], l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      m[nt] = -INFINITY;
      l[nt] = 0.f;
#pragma unroll
      for (int i = 0; i < DT; i++) o[nt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const uint32_t koff = (uint32_t)n16 * (uint32_t)c.stride_t + 16 * g, voff = 4 * (uint32_t)g * (uint32_t)c.stride_t + (uint32_t)n16 * (D / 16);
    u32x4 kw[2][D / 64];
    uint32_t vw[8][VW];
    float skey, sval;
    auto fetch = [&](int n0) {
      const uint8_t *kp = kb + (int64_t)n0 * c.stride_t, *vp = vb + (int64_t)n0 * c.stride_t;
#pragma unroll
      for (int x = 0; x < 2; x++)
#pragma unroll
        for (int i = 0; i < D / 64; i++) kw[x][i] = *reinterpret_cast<const u32x4 *>(kp + (int64_t)x * 16 * c.stride_t + koff + 64 * i);
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const uint8_t *p = vp + (int64_t)((j >> 2) * 16 + (j & 3)) * c.stride_t + voff;
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
    const int end = min(length, t1 * kTile);
    int n0 = t0 * kTile + wave * kSub;
    if (n0 < end) fetch(n0);
    for (; n0 < end; n0 += kTile) {
      // K to fp16; V's dwords on to other registers, so that the next tokens' loads can be under way
      Frag kf[2][KS];
#pragma unroll
      for (int x = 0; x < 2; x++)
#pragma unroll
        for (int s = 0; s < KS; s++) kf[x][s] = kv_frag<CODE>(kw[x][s / 2][2 * (s % 2)], kw[x][s / 2][2 * (s % 2) + 1]);
      const bool edge = n0 + kSub > least;
      uint32_t vt[VW][8];
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const bool there = !edge || n0 + (j >> 2) * 16 + 4 * g + (j & 3) < length;    // what lies behind may be NaN
#pragma unroll
        for (int i = 0; i < VW; i++) vt[i][j] = there ? vw[j][i] : 0u;
      }
      const float sk = skey, sv = sval;
      if (n0 + kTile < end) fetch(n0 + kTile);

      Frag pf[NT][PARTS];
      float svr[NT];
#pragma unroll
      for (int nt = 0; nt < NT; nt++) {
        f32x4 s[2];
#pragma unroll
        for (int x = 0; x < 2; x++) {
          s[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int pt = PARTS - 1; pt >= 0; pt--)
#pragma unroll
            for (int k = 0; k < KS; k++) s[x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[x][k].v, qf[nt][pt][k].v, s[x], 0, 0, 0);
        }
        const float f = factor[nt] * sk;
        if (logits && nt * 16 + n16 < R) {
#pragma unroll
          for (int x = 0; x < 2; x++)
            *reinterpret_cast<f32x4 *>(logits + (row * R + nt * 16 + n16) * c.capacity + n0 + 16 * x + 4 * g) = s[x] * f;
        }
        const bool fresh = m[nt] == -INFINITY;                                         // this row has seen no key yet
        const float ref = fresh ? 0.f : m[nt];
        float z[8], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; i++) {
          z[i] = __builtin_fmaf(s[i / 4][i % 4], f, -ref);
          if (edge) z[i] = n0 + (i / 4) * 16 + 4 * g + i % 4 < limit[nt] ? z[i] : -INFINITY;
          top = fmaxf(top, z[i]);
        }
        svr[nt] = edge && n0 >= limit[nt] ? 0.f : sv;                                  // a NaN block is NaN for those who see it
        if (__any(top > kRoom || (fresh && top > -INFINITY))) {
          top = half_swap_max(row_swap_max(top));
          const bool moved = top > kRoom || (fresh && top > -INFINITY);
          const float move = moved ? top - kLift : 0.f;
          const float fade = __builtin_amdgcn_exp2f(-move);
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
            f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int pt = PARTS - 1; pt >= 0; pt--) a = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[j].v, pf[nt][pt].v, a, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; e++) o[nt][4 * i + j][e] = __builtin_fmaf(a[e], svr[nt], o[nt][4 * i + j][e]);
          }
      }
    }

    // ---- the four waves' results together, and out: record (blockIdx.x + row) of the joined head
    const int64_t slot = (int64_t)blockIdx.x + row;
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
      const int tid = threadIdx.x;
      for (int x = tid; x < 16 * D / 4; x += kThreads) {
        const int n = x / (D / 4), dd = x % (D / 4) * 4, r = nt * 16 + n;
        if (r < R) {
          float M = sh_m[0][n];
#pragma unroll
          for (int w = 1; w < kWaves; w++) M = fmaxf(M, sh_m[w][n]);
          f32x4 a = {0.f, 0.f, 0.f, 0.f};
          float ll = 0.f;
#pragma unroll
          for (int w = 0; w < kWaves; w++) {
            const float fade = sh_m[w][n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sh_m[w][n] - M);
            if (sh_m[w][n] != -INFINITY) a += *reinterpret_cast<const f32x4 *>(&sh_o[w][n][dd]) * fade;
            ll += sh_l[w][n] * fade;
          }
          *reinterpret_cast<f32x4 *>(part_o + (slot * R + r) * D + dd) = a;
          if (dd == 0) *reinterpret_cast<f32x2 *>(part_ml + (slot * R + r) * 2) = f32x2{M, ll};
        }
      }
      __syncthreads();
    }
    u += t1 - t0;
  }
}

// One workgroup per row: the joined result of its head's partial ones.
template <typename T>
__global__ __launch_bounds__(kThreads) void kv_attn_join_kernel(ns_kv_cache c, ns_kv_attn_desc d, const int32_t *lengths, int workgroups,
                                                                const float *part_o, const float *part_ml, T *out, float *lse, float *lse2) {
  const int tid = threadIdx.x, lane = tid & 63, D = c.head_dim;
  const int G = d.heads / c.heads_kv, R = G * d.tokens;
  const int r = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int64_t row = (int64_t)b * c.heads_kv + h;
  __shared__ float sh[kThreads * 4], sh_ml[kThreads * 2];

  const int64_t total = all_tiles(lengths, c.batch, c.capacity, lane) * c.heads_kv;
  const int64_t share = max((int64_t)1, share_of(total, workgroups));
  int64_t before = 0;
  for (int x = 0; x < b; x += 64) before += wave_total(x + lane < b ? tiles_of(lengths, x + lane, c.batch, c.capacity) : 0);
  const int tiles = tiles_of(lengths, b, c.batch, c.capacity);
  const int64_t lo = before * c.heads_kv + (int64_t)h * tiles;
  const int first = (int)(lo / share), parts = tiles ? (int)((lo + tiles - 1) / share) - first + 1 : 0;
  const int64_t slot = first + row;

  // the largest reference and the sum, by the wave's lanes, the same in every wave
  float M = -INFINITY;
  for (int p = lane; p < parts; p += 64) M = fmaxf(M, part_ml[((slot + p) * R + r) * 2]);
  M = wave_max(M);
  const int quads = D / 4, slices = kThreads / quads, s = tid / quads, dd = tid % quads * 4;
  f32x4 a = {0.f, 0.f, 0.f, 0.f};
  float L = 0.f;
  for (int p = s; p < parts; p += slices) {
    const float *ml = part_ml + ((slot + p) * R + r) * 2;
    if (ml[0] != -INFINITY) {
      const float fade = __builtin_amdgcn_exp2f(ml[0] - M);
      a += *reinterpret_cast<const f32x4 *>(part_o + ((slot + p) * R + r) * D + dd) * fade;
      L += ml[1] * fade;
    }
  }
  *reinterpret_cast<f32x4 *>(&sh[tid * 4]) = a;
  sh_ml[tid] = L;
  __syncthreads();
  if (tid < quads) {
    L = sh_ml[tid];
    for (int x = 1; x < slices; x++) {
      a += *reinterpret_cast<const f32x4 *>(&sh[(x * quads + tid) * 4]);
      L += sh_ml[x * quads + tid];
    }
    const bool some = M != -INFINITY;
    const float inv = some ? 1.f / L : 0.f;
    const int t = r / G, hq = h * G + r - t * G;
    T *to = out + b * d.out_stride_b + (int64_t)hq * d.out_stride_h + (int64_t)t * d.out_stride_t + dd;
#pragma unroll
    for (int e = 0; e < 4; e++) a[e] = some ? a[e] * inv : 0.f;
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<f32x4 *>(to) = a;
    } else {
      *reinterpret_cast<u32x2 *>(to) = u32x2{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3])};
    }
    if (tid == 0) {
      const float z2 = some ? M + __log2f(L) : -INFINITY;
      if (lse) lse[((int64_t)b * d.heads + hq) * d.tokens + t] = z2 * kLn2;
      if (lse2) lse2[row * R + r] = z2;
    }
  }
}

// The weights that every position was given, from the rows' logits; four positions a thread.
__global__ __launch_bounds__(kThreads) void kv_weights_kernel(ns_kv_cache c, ns_kv_attn_desc d, const int32_t *lengths, const int32_t *counts,
                                                              const float *logits, const float *lse2, const float *w_in, float *w_out) {
  const int h = blockIdx.y, b = blockIdx.z, n0 = (int)(blockIdx.x * kThreads + threadIdx.x) * 4;
  const int G = d.heads / c.heads_kv, R = G * d.tokens;
  const int length = kv_length(lengths, b, c.capacity), count = kv_count(counts, b, d.tokens);
  if (n0 >= c.capacity || (n0 >= length && w_in == w_out)) return;
  const int64_t row = (int64_t)b * c.heads_kv + h;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  if (n0 < length)
    for (int r = 0; r < R; r++) {
      const int limit = kv_seen(d, r / G, length, count);
      const f32x4 z = *reinterpret_cast<const f32x4 *>(logits + (row * R + r) * c.capacity + n0);
      const float ref = lse2[row * R + r];
#pragma unroll
      for (int i = 0; i < 4; i++) sum[i] += n0 + i < limit ? __builtin_amdgcn_exp2f(z[i] - ref) : 0.f;
    }
  const int64_t at = row * c.capacity + n0;
  for (int i = 0; i < 4; i++)
    if (n0 + i < length || w_in != w_out) w_out[at + i] = (w_in ? w_in[at + i] : 0.f) + sum[i];
}

// ---- host side of the split kernel

int rows_of(const ns_kv_cache &c, const ns_kv_attn_desc &d) { return d.heads / c.heads_kv * d.tokens; }

// Row tiles of 16 that the split kernel has registers for
int most_tiles(int head_dim, int dtype) {
  if (dtype == NS_F32) return head_dim == 64 ? 4 : head_dim == 128 ? 2 : 1;
  return head_dim == 256 ? 1 : 4;
}
bool few_rows(const ns_kv_cache &c, const ns_kv_attn_desc &d) { return rows_of(c, d) <= 16 * most_tiles(c.head_dim, d.dtype); }

struct SplitLayout { size_t o, ml, lse2, logits, total; int workgroups; };
SplitLayout split_layout(const ns_kv_cache &c, const ns_kv_attn_desc &d, bool weights) {
  SplitLayout w;
  w.workgroups = ((rows_of(c, d) + 15) / 16 * c.head_dim <= 128 ? 2 : 1) * device_cu_count();
  const size_t rows = rows_of(c, d), heads = (size_t)c.batch * c.heads_kv, slots = (size_t)w.workgroups + heads;
  size_t off = 0;
  w.o = off;
  off += align_up(slots * rows * c.head_dim * 4, 256);
  w.ml = off;
  off += align_up(slots * rows * 8, 256);
  w.lse2 = off;
  off += align_up(heads * rows * 4, 256);
  w.logits = off;
  if (weights) off += align_up(heads * rows * (size_t)c.capacity * 4, 256);
  w.total = off;
  return w;
}

template <typename T, int CODE, int D, int NT>
ns_status launch_split(const KvAttnArgs &a) {
  const SplitLayout w = split_layout(a.c, a.d, a.w_out != nullptr);
  float *po = reinterpret_cast<float *>(a.ws + w.o), *pml = reinterpret_cast<float *>(a.ws + w.ml);
  float *lse2 = reinterpret_cast<float *>(a.ws + w.lse2), *logits = a.w_out ? reinterpret_cast<float *>(a.ws + w.logits) : nullptr;
  hipLaunchKernelGGL((kv_attn_split_kernel<T, CODE, D, NT>), dim3((unsigned)w.workgroups), dim3(kThreads), 0, a.stream, a.c, a.d,
                     static_cast<const T *>(a.q), a.lengths, a.counts, po, pml, logits);
  ns_status st = check_launch("kv_attn_split_kernel");
  if (st != NS_OK) return st;
  hipLaunchKernelGGL((kv_attn_join_kernel<T>), dim3((unsigned)rows_of(a.c, a.d), (unsigned)a.c.heads_kv, (unsigned)a.c.batch), dim3(kThreads), 0, a.stream,
                     a.c, a.d, a.lengths, w.workgroups, po, pml, static_cast<T *>(a.out), a.lse, lse2);
  st = check_launch("kv_attn_join_kernel");
  if (st != NS_OK || !a.w_out) return st;
  hipLaunchKernelGGL(kv_weights_kernel, dim3((unsigned)((a.c.capacity + 4 * kThreads - 1) / (4 * kThreads)), (unsigned)a.c.heads_kv, (unsigned)a.c.batch),
                     dim3(kThreads), 0, a.stream, a.c, a.d, a.lengths, a.counts, logits, lse2, a.w_in, a.w_out);
  return check_launch("kv_weights_kernel");
}

template <typename T, int CODE, int D>
ns_status launch_tiles(const KvAttnArgs &a) {
  constexpr int most = sizeof(T) == 4 ? (D == 64 ? 4 : D == 128 ? 2 : 1) : D == 256 ? 1 : 4;
  const int nt = (rows_of(a.c, a.d) + 15) / 16;
  if (nt <= 1) return launch_split<T, CODE, D, 1>(a);
  if constexpr (most >= 4)
    if (nt > 2) return launch_split<T, CODE, D, 4>(a);
  if constexpr (most >= 2) return launch_split<T, CODE, D, 2>(a);
  return NS_ERR_UNSUPPORTED;
}

template <typename T, int CODE>
ns_status launch_any(const KvAttnArgs &a) {
  if (!few_rows(a.c, a.d)) return launch_kv_prompt(a);
  return a.c.head_dim == 64 ? launch_tiles<T, CODE, 64>(a) : a.c.head_dim == 128 ? launch_tiles<T, CODE, 128>(a) : launch_tiles<T, CODE, 256>(a);
}

}  // namespace

size_t kv_attn_workspace_bytes(const ns_kv_cache &c, const ns_kv_attn_desc &d, bool weights) {
  if (!few_rows(c, d)) return kv_prompt_workspace_bytes(c, d, weights);
  return split_layout(c, d, weights).total;
}

ns_status launch_kv_attn(const KvAttnArgs &a) {
  if (a.d.dtype == NS_F32) return a.c.code == NS_CODE_I8 ? launch_any<float, NS_CODE_I8>(a) : launch_any<float, NS_CODE_E4M3>(a);
  return a.c.code == NS_CODE_I8 ? launch_any<bf16_t, NS_CODE_I8>(a) : launch_any<bf16_t, NS_CODE_E4M3>(a);
}

}  // namespace ns
