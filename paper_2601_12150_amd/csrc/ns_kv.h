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
size_t kv_evict_workspace_bytes(const ns_kv_cache &from, int keep);
ns_status launch_kv_evict(const ns_kv_cache &from, const ns_kv_cache &to, const float *weights, const int32_t *lengths, int keep,
                          int n_global, int n_recent, int32_t *kept, float *w_out, int32_t *lengths_out, void *ws, hipStream_t s);

// ---- counts that live in device memory, taken into the range that the kernels can work with
__device__ __forceinline__ int kv_length(const int32_t *lengths, int b, int capacity) { return min(max(lengths[b], 0), capacity); }
__device__ __forceinline__ int kv_count(const int32_t *counts, int b, int tokens) {
  return counts ? min(max(counts[b], 0), tokens) : tokens;
}

// ---- codes.  CODE: ns_kv_code
// the four values of a dword of codes
template <int CODE>
__device__ __forceinline__ f32x4 kv_decode4(uint32_t w) {
  if (CODE == NS_CODE_I8)
    return f32x4{(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24)};
  return f32x4{__builtin_amdgcn_cvt_f32_fp8((int)w, 0), __builtin_amdgcn_cvt_f32_fp8((int)w, 1),
               __builtin_amdgcn_cvt_f32_fp8((int)w, 2), __builtin_amdgcn_cvt_f32_fp8((int)w, 3)};
}
// the nearest codes (ties to even) of values within the codes' range
template <int CODE>
__device__ __forceinline__ uint32_t kv_encode4(f32x4 y) {
  if (CODE == NS_CODE_I8) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) w |= ((uint32_t)(int)__builtin_rintf(y[i]) & 0xffu) << (8 * i);
    return w;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
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

}  // namespace ns
