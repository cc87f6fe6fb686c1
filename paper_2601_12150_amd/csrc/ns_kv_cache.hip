// The 8-bit key/value cache: tokens in (kv_append_kernel), values out (kv_read_kernel).
#include "ns_kv.h"

namespace ns {

namespace {

constexpr int kThreads = 256;
constexpr int kMostBlocks = 1 << 23;    // of one launch: a grid's threads along an axis are counted in 32 bits

template <typename T> struct Row8;      // eight consecutive elements as they lie in memory
template <> struct Row8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float *p) { a = reinterpret_cast<const f32x4 *>(p)[0]; b = reinterpret_cast<const f32x4 *>(p)[1]; }
  __device__ __forceinline__ void zero() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ f32x4 half(int i) const { return i ? b : a; }
};
template <> struct Row8<bf16_t> {
  u32x4 w;
  __device__ __forceinline__ void load(const bf16_t *p) { w = *reinterpret_cast<const u32x4 *>(p); }
  __device__ __forceinline__ void zero() { w = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ f32x4 half(int i) const { return f32x4{bf16_lo(w[2 * i]), bf16_hi(w[2 * i]), bf16_lo(w[2 * i + 1]), bf16_hi(w[2 * i + 1])}; }
};
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// One workgroup per block of tokens that a sequence's new tokens may touch, head, and keys or values.  The scale needs the
// largest magnitude of all new values of the block: a thread has its up to PIECES times 8 in registers until it is known, so that they are
// read once.  Bound by the reads and writes: 8404 tokens of 8 heads of 128 channels in bf16, 52 MB, 16 us (3.2 TB/s); one token 3.5 us.
template <typename T, int CODE, int PIECES>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(ns_kv_cache c, int first, int tokens, const T *k, const T *v, int64_t sb, int64_t sh,
                                                             int64_t st, const int32_t *start, const int32_t *counts) {
  const int b = blockIdx.z, h = blockIdx.y >> 1, value = blockIdx.y & 1, tid = threadIdx.x;
  const int from = kv_length(start, b, c.capacity), to = min(from + kv_count(counts, b, tokens), c.capacity);
  const int lblock = 31 - __clz(c.block), block = (from >> lblock) + first + (int)blockIdx.x, begin = block << lblock;
  if (block >= c.capacity >> lblock) return;
  const int lo = max(from, begin), hi = min(to, begin + c.block);
  if (lo >= hi) return;
  const T *x = (value ? v : k) + b * sb + h * sh;
  uint8_t *codes = static_cast<uint8_t *>(value ? c.v : c.k) + b * c.stride_b + h * c.stride_h;
  float *scale = (value ? c.v_scale : c.k_scale) + ((int64_t)b * c.heads_kv + h) * (c.capacity >> lblock) + block;
  const bool live = from > begin;                                      // tokens before the new ones are in this block
  const float old = live ? *scale : 0.f;
  const int lpieces = 31 - __clz(c.head_dim / 8), step = kThreads >> lpieces;      // pieces of a token; tokens between a thread's
  const int n0 = lo + (tid >> lpieces), d = (tid & ((1 << lpieces) - 1)) * 8;

  Row8<T> y[PIECES];
#pragma unroll
  for (int i = 0; i < PIECES; i++) {
    const int n = n0 + i * step;
    y[i].zero();
    if (n < hi) y[i].load(x + (int64_t)(n - from) * st + d);
  }
  uint32_t most = 0;                                                   // magnitudes order like their bits; NaN above all
#pragma unroll
  for (int i = 0; i < PIECES; i++)
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const f32x4 z = y[i].half(j);
      most = max(max(most, max(abs_bits(z[0]), abs_bits(z[1]))), max(abs_bits(z[2]), abs_bits(z[3])));
    }
  __shared__ uint32_t largest[kThreads / 64];
#pragma unroll
  for (int o = 32; o; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
  if (tid % 64 == 0) largest[tid / 64] = most;
  __syncthreads();
  most = max(max(largest[0], largest[1]), max(largest[2], largest[3]));
  float s = kv_scale_for<CODE>(most);
  // (the comparison is false for a NaN on either side: a NaN block stays one, a NaN among the new tokens makes it one)
  // (the sign of limit * old - most is exact this way)
  if (live && (kv_is_nan(old) || (most < kInfBits && __builtin_fmaf(kv_limit<CODE>(), old, -__uint_as_float(most)) >= 0.f))) s = old;
  if (live && s > old) {                                               // (not with a NaN: the codes no longer matter)
    const float ratio = old / s;
    for (int n = begin + (tid >> lpieces); n < from; n += step) {
      u32x2 *w = reinterpret_cast<u32x2 *>(codes + n * c.stride_t + d);
      const u32x2 was = *w;
      *w = u32x2{kv_recode4<CODE>(was[0], ratio), kv_recode4<CODE>(was[1], ratio)};
    }
  }
  const bool plain = kv_is_pow2(s);                                    // else one of the caller's own: the quotient is rounded, then the code
  const bool none = kv_is_nan(s) || s == 0.f;                          // (0: the caller's own for a block of zeros, which zeros have entered)
  const float inv = plain ? 1.f / s : 1.f;
#pragma unroll
  for (int i = 0; i < PIECES; i++) {
    const int n = n0 + i * step;
    if (n < hi) {
      u32x2 w;
#pragma unroll
      for (int j = 0; j < 2; j++) {
        f32x4 z = y[i].half(j);
        if (!plain) z /= s;
        w[j] = none ? 0u : kv_encode4<CODE>(z, inv);
      }
      *reinterpret_cast<u32x2 *>(codes + n * c.stride_t + d) = w;
    }
  }
  if (tid == 0) *scale = s;
}

// 16 codes per thread.  Bound by the writes: 16384 positions of 8 heads of 128 channels in bf16, 84 MB, 15 us (5.5 TB/s).
template <typename T, int CODE>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(ns_kv_cache c, const int32_t *lengths, int first, int tokens, T *k_out, T *v_out) {
  const int b = blockIdx.z, h = blockIdx.y >> 1, value = blockIdx.y & 1;
  const int pieces = c.head_dim / 16;
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int t = (int)(at / pieces), d = (int)(at % pieces) * 16;
  if (t >= tokens) return;
  const int n = first + t;
  T *out = (value ? v_out : k_out) + (((int64_t)b * c.heads_kv + h) * tokens + t) * c.head_dim + d;
  u32x4 w = {0, 0, 0, 0};
  float s = 0.f;
  if (n < kv_length(lengths, b, c.capacity)) {
    w = *reinterpret_cast<const u32x4 *>(static_cast<const uint8_t *>(value ? c.v : c.k) + b * c.stride_b + h * c.stride_h + n * c.stride_t + d);
    s = (value ? c.v_scale : c.k_scale)[((int64_t)b * c.heads_kv + h) * (c.capacity / c.block) + n / c.block];
  }
#pragma unroll
  for (int i = 0; i < 4; i++) store4(out + 4 * i, kv_decode4<CODE>(w[i]) * s);
}

template <typename T, int CODE>
void append(int blocks, hipStream_t s, const ns_kv_cache &c, int tokens, const void *k, const void *v, int64_t sb, int64_t sh, int64_t st,
            const int32_t *start, const int32_t *counts) {
  auto go = [&](auto kernel) {
    for (int first = 0; first < blocks; first += kMostBlocks)
      hipLaunchKernelGGL(kernel, dim3((unsigned)min(blocks - first, kMostBlocks), (unsigned)c.heads_kv * 2, (unsigned)c.batch), dim3(kThreads), 0, s, c, first,
                         tokens, static_cast<const T *>(k), static_cast<const T *>(v), sb, sh, st, start, counts);
  };
  // what a thread has to hold: the block's values, or all the new ones
  const int values = (min(c.block, tokens) * c.head_dim + 8 * kThreads - 1) / (8 * kThreads);
  values <= 1 ? go(kv_append_kernel<T, CODE, 1>) : values <= 4 ? go(kv_append_kernel<T, CODE, 4>) : go(kv_append_kernel<T, CODE, 16>);
}

}  // namespace

ns_status launch_kv_append(const ns_kv_cache &c, int tokens, int dtype, const void *k, const void *v, int64_t sb, int64_t sh,
                           int64_t st, const int32_t *start, const int32_t *counts, hipStream_t s) {
  // the blocks that so many tokens touch where they begin at a block's last position
  const int blocks = min((tokens + c.block - 2) / c.block + 1, c.capacity / c.block);
  if (dtype == NS_F32)
    c.code == NS_CODE_I8 ? append<float, NS_CODE_I8>(blocks, s, c, tokens, k, v, sb, sh, st, start, counts)
                         : append<float, NS_CODE_E4M3>(blocks, s, c, tokens, k, v, sb, sh, st, start, counts);
  else
    c.code == NS_CODE_I8 ? append<bf16_t, NS_CODE_I8>(blocks, s, c, tokens, k, v, sb, sh, st, start, counts)
                         : append<bf16_t, NS_CODE_E4M3>(blocks, s, c, tokens, k, v, sb, sh, st, start, counts);
  return check_launch("kv_append_kernel");
}

ns_status launch_kv_read(const ns_kv_cache &c, const int32_t *lengths, int first, int tokens, int dtype, void *k_out, void *v_out,
                         hipStream_t s) {
  const int64_t pieces = (int64_t)tokens * (c.head_dim / 16);
  const dim3 grid((unsigned)((pieces + kThreads - 1) / kThreads), (unsigned)c.heads_kv * 2, (unsigned)c.batch);
  auto go = [&](auto kernel, auto *kp, auto *vp) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, c, lengths, first, tokens, kp, vp); };
  if (dtype == NS_F32) {
    float *kp = static_cast<float *>(k_out), *vp = static_cast<float *>(v_out);
    c.code == NS_CODE_I8 ? go(kv_read_kernel<float, NS_CODE_I8>, kp, vp) : go(kv_read_kernel<float, NS_CODE_E4M3>, kp, vp);
  } else {
    bf16_t *kp = static_cast<bf16_t *>(k_out), *vp = static_cast<bf16_t *>(v_out);
    c.code == NS_CODE_I8 ? go(kv_read_kernel<bf16_t, NS_CODE_I8>, kp, vp) : go(kv_read_kernel<bf16_t, NS_CODE_E4M3>, kp, vp);
  }
  return check_launch("kv_read_kernel");
}

}  // namespace ns
