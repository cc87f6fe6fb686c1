// The 8-bit key/value cache: what its translation units share.
#pragma once
#include "ns_common.h"

namespace ns {

struct KvAttnArgs {
  ns_kv_cache c;
  ns_kv_attn_desc d;
  const void *q;
  const int32_t *lengths, *counts;
  void *out;
  float *lse;
  const float *w_in;
  float *w_out;
  unsigned char *ws;
  hipStream_t stream;
};

ns_status launch_kv_append(const ns_kv_cache &c, int tokens, int dtype, const void *k, const void *v, int64_t sb, int64_t sh,
                           int64_t st, const int32_t *start, const int32_t *counts, hipStream_t s);
ns_status launch_kv_read(const ns_kv_cache &c, const int32_t *lengths, int first, int tokens, int dtype, void *k_out, void *v_out,
                         hipStream_t s);
size_t kv_attn_workspace_bytes(const ns_kv_cache &c, const ns_kv_attn_desc &d, bool weights);
ns_status launch_kv_attn(const KvAttnArgs &a);
// ... of many rows per key/value head (ns_kv_prompt.hip)
size_t kv_prompt_workspace_bytes(const ns_kv_cache &c, const ns_kv_attn_desc &d, bool weights);
ns_status launch_kv_prompt(const KvAttnArgs &a);
size_t kv_evict_workspace_bytes(const ns_kv_cache &from, int keep);
ns_status launch_kv_evict(const ns_kv_cache &from, const ns_kv_cache &to, const float *weights, const int32_t *lengths, int keep,
                          int n_global, int n_recent, int32_t *kept, float *w_out, int32_t *lengths_out, void *ws, hipStream_t s);

// ---- counts that live in device memory, taken into the range that the kernels can work with
__device__ __forceinline__ int kv_length(const int32_t *lengths, int b, int capacity) { return min(max(lengths[b], 0), capacity); }
__device__ __forceinline__ int kv_count(const int32_t *counts, int b, int tokens) {
  return counts ? min(max(counts[b], 0), tokens) : tokens;
}

// Tiles per workgroup where `tiles` of them (up to 2^31 - 1) are shared out
__host__ __device__ constexpr int kv_share(int tiles, int workgroups) { return tiles ? (tiles - 1) / workgroups + 1 : 1; }

// ---- codes.  CODE: ns_kv_code
// the four values of a dword of codes (int8: bytes c + 128 have a conversion of their own)
template <int CODE>
__device__ __forceinline__ f32x4 kv_decode4(uint32_t w) {
  if (CODE == NS_CODE_I8) {
    const uint32_t u = w ^ 0x80808080u;
    return f32x4{(float)(u & 0xffu) - 128.f, (float)((u >> 8) & 0xffu) - 128.f, (float)((u >> 16) & 0xffu) - 128.f, (float)(u >> 24) - 128.f};
  }
  return f32x4{__builtin_amdgcn_cvt_f32_fp8((int)w, 0), __builtin_amdgcn_cvt_f32_fp8((int)w, 1),
               __builtin_amdgcn_cvt_f32_fp8((int)w, 2), __builtin_amdgcn_cvt_f32_fp8((int)w, 3)};
}
// The nearest codes (ties to even) of x * f, which the codes' range holds.  int8: added to 1.5 2^23 in the multiplication itself, whose one
// rounding is then the one to a whole number, in two's complement in the low byte.
template <int CODE>
__device__ __forceinline__ uint32_t kv_encode4(f32x4 x, float f) {
  if (CODE == NS_CODE_I8) {
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; i++) y[i] = __float_as_uint(__builtin_fmaf(x[i], f, 12582912.f));
    const uint32_t lo = __builtin_amdgcn_perm(y[1], y[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(y[3], y[2], 0x04000c0cu);
    return lo | hi;
  }
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * f, x[1] * f, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * f, x[3] * f, w, true);
}

// a power of two (whose reciprocal is one too), or 0
__device__ __forceinline__ bool kv_is_pow2(float s) { return (__float_as_uint(s) & 0x7fffffu) == 0; }

// x * f for a rounding to far fewer bits that is the only one: of a product that fp32 does not hold, the neighbour whose last bit is 1.  No
// border between codes has that bit, so that the product lies on the same side of all of them.
__device__ __forceinline__ float kv_mul_odd(float x, float f) {
  const float p = x * f, off = __builtin_fmaf(x, f, -p);               // (off: exact)
  const uint32_t u = __float_as_uint(p);
  return off == 0.f || (u & 1u) ? p : __uint_as_float((off < 0.f) == (p < 0.f) ? u + 1 : u - 1);
}
// The nearest codes of codes times any ratio f.  (int8's rounding in kv_encode4 is one already.)
template <int CODE> __device__ __forceinline__ uint32_t kv_recode4(uint32_t w, float f) {
  f32x4 x = kv_decode4<CODE>(w);
  if (CODE == NS_CODE_I8 || kv_is_pow2(f)) return kv_encode4<CODE>(x, f);
#pragma unroll
  for (int i = 0; i < 4; i++) x[i] = kv_mul_odd(x[i], f);
  return kv_encode4<CODE>(x, 1.f);
}

template <int CODE> __device__ __forceinline__ constexpr float kv_limit() { return CODE == NS_CODE_I8 ? 127.f : 448.f; }   // the largest code
constexpr uint32_t kInfBits = 0x7f800000u, kNanBits = 0x7fc00000u;
// The scale of a block whose largest magnitude has these bits: 2^e, e the smallest with most <= 127 * 2^e (448 * 2^e), at
// least -100; NaN for a NaN or an infinity.  With most = 1.f * 2^x (f the fraction's bits): 127 = 1.984375 * 2^6 and
// 448 = 1.75 * 2^8, so e = x - 6 (x - 8), one more where 1.f is above 1.984375 (1.75).
template <int CODE>
__device__ __forceinline__ float kv_scale_for(uint32_t most) {
  if (most >= kInfBits) return __uint_as_float(kNanBits);
  const int x = (int)(most >> 23) - 127, f = (int)(most & 0x7fffffu);
  const int e = CODE == NS_CODE_I8 ? x - 6 + (f > 0x7e0000) : x - 8 + (f > 0x600000);
  return __uint_as_float((uint32_t)(max(e, -100) + 127) << 23);
}
__device__ __forceinline__ bool kv_is_nan(float s) { return !(s == s); }

// ---- matrix products over codes
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
union Frag {                               // one lane's operand of a 16x16x32 or 32x32x16 product
  f16x8 v;
  uint32_t w[4];
};

// Codes as fp16, which holds every one of them exactly.  int8: the byte c + 128 (the code with its top bit turned) below the
// byte 0x64 is 1024 + 128 + c in fp16, from which 1152 is taken: with the byte permutation one and a half instructions for two codes.
// e4m3: a conversion of two.  The operand is one dword of codes prepared by kv_raw.
template <int CODE> __device__ __forceinline__ uint32_t kv_raw(uint32_t w) { return CODE == NS_CODE_I8 ? w ^ 0x80808080u : w; }
template <int CODE, int HALF> __device__ __forceinline__ uint32_t kv_f16x2(uint32_t raw) {      // the codes 2 HALF, 2 HALF + 1
  if (CODE == NS_CODE_I8) {
    const uint32_t u = __builtin_amdgcn_perm(0x64646464u, raw, HALF ? 0x07030602u : 0x05010400u);
    const f16x2 c = __builtin_bit_cast(f16x2, u) - f16x2{(_Float16)1152, (_Float16)1152};
    return __builtin_bit_cast(uint32_t, c);
  }
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)raw, 1.f, HALF));
}
// The same times f, a power of two that leaves them exact: in the instruction that makes them.  kv_by<CODE>(f) is what the conversion takes.
template <int CODE> struct By { f16x2 f, bias; float scale; };
template <int CODE> __device__ __forceinline__ By<CODE> kv_by(float f) {
  const _Float16 h = (_Float16)f, b = (_Float16)(-1152.f * f);
  return By<CODE>{f16x2{h, h}, f16x2{b, b}, f};
}
template <int CODE, int HALF> __device__ __forceinline__ uint32_t kv_f16x2_by(uint32_t raw, const By<CODE> &by) {
  if (CODE == NS_CODE_I8) {
    const uint32_t u = __builtin_amdgcn_perm(0x64646464u, raw, HALF ? 0x07030602u : 0x05010400u);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, u), by.f, by.bias));
  }
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)raw, by.scale, HALF));
}
// eight consecutive codes
template <int CODE> __device__ __forceinline__ Frag kv_frag(uint32_t lo, uint32_t hi) {
  lo = kv_raw<CODE>(lo);
  hi = kv_raw<CODE>(hi);
  return Frag{.w = {kv_f16x2<CODE, 0>(lo), kv_f16x2<CODE, 1>(lo), kv_f16x2<CODE, 0>(hi), kv_f16x2<CODE, 1>(hi)}};
}
// The transpose: of eight tokens' dwords (four channels each) the four channels' fragments, tokens in order.
template <int CODE> __device__ __forceinline__ void kv_frags_t(const uint32_t (&t)[8], Frag (&f)[4]) {
#pragma unroll
  for (int j = 0; j < 4; j++) {
    const uint32_t a = kv_raw<CODE>(t[2 * j]), b = kv_raw<CODE>(t[2 * j + 1]);
    const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x05010400u), hi = __builtin_amdgcn_perm(b, a, 0x07030602u);   // a0 b0 a1 b1, a2 b2 a3 b3
    f[0].w[j] = kv_f16x2<CODE, 0>(lo);
    f[1].w[j] = kv_f16x2<CODE, 1>(lo);
    f[2].w[j] = kv_f16x2<CODE, 0>(hi);
    f[3].w[j] = kv_f16x2<CODE, 1>(hi);
  }
}

// ---- queries as fp16.  A row is scaled by a power of two that brings its largest magnitude to 2^14 .. 2^15: what lies 28 binades
// below it keeps its 11 bits (bf16 has 8).  fp32 is taken as the sum of two such numbers, each the nearest, which is off by 2^-23 of the
// value at most (fp32's own step is 2^-23 of it, or less); what lies 2^-16 below the largest or further is off by at most 2^-39 of the largest.
__device__ __forceinline__ int kv_row_shift(uint32_t most) { return most >= kInfBits ? 0 : 141 - (int)(most >> 23); }   // q is taken times 2^this

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
}
template <typename T> __device__ __forceinline__ f32x4 load4(const T *p);
template <> __device__ __forceinline__ f32x4 load4<float>(const float *p) { return *reinterpret_cast<const f32x4 *>(p); }
template <> __device__ __forceinline__ f32x4 load4<bf16_t>(const bf16_t *p) {
  const u32x2 w = *reinterpret_cast<const u32x2 *>(p);
  return f32x4{bf16_lo(w[0]), bf16_hi(w[0]), bf16_lo(w[1]), bf16_hi(w[1])};
}
__device__ __forceinline__ void store4(float *p, f32x4 v) { *reinterpret_cast<f32x4 *>(p) = v; }
__device__ __forceinline__ void store4(bf16_t *p, f32x4 v) { *reinterpret_cast<u32x2 *>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}; }

// Weights are 2^(z - m + 11) in fp16, m a logit near the largest so far, which is moved up before they pass 2^15: a weight that is the
// largest one's 2^-25 or more keeps its 11 bits, and below it all are within 2^-36 of the largest.  (Two parts, where the call is in fp32: 2^-23
// of itself from 2^-13 of the largest on, and 2^-36 of the largest below.)  The sums of the weights take them as they were before that rounding.
// Where the 11 is part of the exponent its last bits are 2^-20, and every weight is off by up to 3 10^-7 of itself: what bf16 calls of many rows
// take in caches of more than kFewKeys tokens, where log-sums are seldom near 0 (they are off by that much at most, whatever their size).  Elsewhere
// 2^11 is a factor of the weight behind the exponential, and so of none of its sums: another instruction for each, of which long prompts would be 4
// to 6 % slower (4096 tokens of 64 heads of 64 channels 491 -> 514 us); 2048 queries of 16 heads on 320 tokens take 13.5 us with it, 13.2 without.
constexpr int kFewKeys = 512;
template <bool FACTOR> struct Lift {
  static constexpr float exponent = FACTOR ? 0.f : 11.f, factor = FACTOR ? 2048.f : 1.f, room = exponent + 4.f;
};

// positions that query t sees: 0 .. limit - 1
__device__ __forceinline__ int kv_seen(const ns_kv_attn_desc &d, int t, int length, int count) {
  return t >= count ? 0 : d.causal ? max(length - count + t + 1, 0) : length;
}

// ---- the weights' second pass over K (ns_kv_prompt.hip): its operands, 16 rows of queries r = token * group + head at a time.  Channels of the
// step s = 2 i + f that lane (n, g) has: 64 i + 16 g + 8 f + j, so that 16 bytes of codes are two operands.  One wave.
template <typename T>
__device__ __forceinline__ void kv_rows_tile(const ns_kv_cache &c, const ns_kv_attn_desc &d, const T *q, int b, int h, int tile, int lane, Frag *frags,
                                             float *factors) {
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1;
  const int n16 = lane & 15, g = lane >> 4, KS = c.head_dim / 32;
  const int G = d.heads / c.heads_kv, R = G * d.tokens, tiles = (R + 15) / 16;
  const int64_t row = (int64_t)b * c.heads_kv + h;
  const int r = tile * 16 + n16;
  const bool real = r < R;
  const int t = real ? r / G : 0;
  const T *p = q + b * d.q_stride_b + (int64_t)(h * G + (real ? r - t * G : 0)) * d.q_stride_h + (int64_t)t * d.q_stride_t + 16 * g;
  uint32_t most = 0;
  for (int i = 0; i < KS / 2; i++)
#pragma unroll
    for (int k = 0; k < 4; k++) {
      const f32x4 x = load4(p + 64 * i + 4 * k);
#pragma unroll
      for (int j = 0; j < 4; j++) most = max(most, __float_as_uint(x[j]) & 0x7fffffffu);
    }
  most = max(most, (uint32_t)__shfl_xor((int)most, 16));
  most = max(most, (uint32_t)__shfl_xor((int)most, 32));
  const int shift = kv_row_shift(most);
  if (g == 0) factors[row * tiles * 16 + r] = real ? ldexpf(d.scale, -shift) * kLog2e : 0.f;
  for (int s = 0; s < KS; s++) {
    Frag f[PARTS];
#pragma unroll
    for (int k = 0; k < 2; k++) {
      const f32x4 x = load4(p + 64 * (s / 2) + 8 * (s % 2) + 4 * k);
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        const float x0 = real ? ldexpf(x[j], shift) : 0.f, x1 = real ? ldexpf(x[j + 1], shift) : 0.f;
        f[0].w[2 * k + j / 2] = pack_f16(x0, x1);
        if (PARTS == 2) {
          const f16x2 w = __builtin_bit_cast(f16x2, f[0].w[2 * k + j / 2]);
          f[PARTS - 1].w[2 * k + j / 2] = pack_f16(x0 - (float)w[0], x1 - (float)w[1]);
        }
      }
    }
#pragma unroll
    for (int pt = 0; pt < PARTS; pt++) frags[(((row * tiles + tile) * PARTS + pt) * KS + s) * 64 + lane] = f[pt];
  }
}
inline size_t kv_rows_padded(const ns_kv_cache &c, const ns_kv_attn_desc &d) {
  return (size_t)c.batch * c.heads_kv * (((size_t)(d.heads / c.heads_kv) * d.tokens + 15) / 16) * 16;
}
inline size_t kv_rows_frag_bytes(const ns_kv_cache &c, const ns_kv_attn_desc &d) {
  return align_up(kv_rows_padded(c, d) * c.head_dim * 2 * (d.dtype == NS_F32 ? 2 : 1), 256);
}
inline size_t kv_rows_factor_bytes(const ns_kv_cache &c, const ns_kv_attn_desc &d) { return align_up(kv_rows_padded(c, d) * 4, 256); }
// lse2 [B Hkv][R]: log2 of the rows' sums, +inf for a row that sees nothing; rows: the operands are yet to be made
ns_status launch_kv_weights_again(const KvAttnArgs &a, Frag *frags, float *factors, const float *lse2, bool rows);

}  // namespace ns
