// The 8-bit key/value cache: tokens in (kv_append_kernel), values out (kv_read_kernel).
#include "ns_kv.h"

namespace ns {

namespace {

constexpr int kThreads = 256;

template <typename T> struct Row4;      // four consecutive elements
template <> struct Row4<float> {
  static __device__ __forceinline__ f32x4 load(const float *p) { return *reinterpret_cast<const f32x4 *>(p); }
  static __device__ __forceinline__ void store(float *p, f32x4 v) { *reinterpret_cast<f32x4 *>(p) = v; }
};
template <> struct Row4<bf16_t> {
  static __device__ __forceinline__ f32x4 load(const bf16_t *p) {
    const u32x2 w = *reinterpret_cast<const u32x2 *>(p);
    return f32x4{bf16_lo(w[0]), bf16_hi(w[0]), bf16_lo(w[1]), bf16_hi(w[1])};
  }
  static __device__ __forceinline__ void store(bf16_t *p, f32x4 v) {
    *reinterpret_cast<u32x2 *>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  }
};

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// One workgroup per block of tokens that a sequence's new tokens may touch, head, and keys or values.  The scale needs the
// largest magnitude of all new values of the block, so they are read twice; the second time they come from the L2.
template <typename T, int CODE>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(ns_kv_cache c, int tokens, const T *k, const T *v, int64_t sb, int64_t sh,
                                                             int64_t st, const int32_t *start, const int32_t *counts) {
  const int b = blockIdx.z, h = blockIdx.y >> 1, value = blockIdx.y & 1, tid = threadIdx.x;
  const int from = kv_length(start, b, c.capacity), to = min(from + kv_count(counts, b, tokens), c.capacity);
  const int block = from / c.block + (int)blockIdx.x;
  const int lo = max(from, block * c.block), hi = min(to, (block + 1) * c.block);
  if (lo >= hi) return;
  const int quads = c.head_dim / 4;                                    // a power of two: 16, 32 or 64
  const T *x = (value ? v : k) + b * sb + h * sh;
  uint8_t *codes = static_cast<uint8_t *>(value ? c.v : c.k) + b * c.stride_b + h * c.stride_h;
  float *scale = (value ? c.v_scale : c.k_scale) + ((int64_t)b * c.heads_kv + h) * (c.capacity / c.block) + block;
  const int d = tid % quads * 4, step = kThreads / quads;

  uint32_t most = 0;                                                   // magnitudes order like their bits; NaN above all
  for (int n = lo + tid / quads; n < hi; n += step) {
    const f32x4 y = Row4<T>::load(x + (int64_t)(n - from) * st + d);
    most = max(max(most, max(abs_bits(y[0]), abs_bits(y[1]))), max(abs_bits(y[2]), abs_bits(y[3])));
  }
  __shared__ uint32_t largest[kThreads / 64];
#pragma unroll
  for (int o = 32; o; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
  if (tid % 64 == 0) largest[tid / 64] = most;
  const bool live = from > block * c.block;                            // tokens before the new ones are in this block
  const float old = live ? *scale : 0.f;
  __syncthreads();
  most = max(max(largest[0], largest[1]), max(largest[2], largest[3]));
  float s = kv_scale_for<CODE>(most);
  // (the comparison is false for a NaN on either side: a NaN block stays one, a NaN among the new tokens makes it one)
  if (live && (kv_is_nan(old) || (most < kInfBits && __uint_as_float(most) <= kv_limit<CODE>() * old))) s = old;
  if (live && s > old) {                                               // (not with a NaN: the codes no longer matter)
    const float ratio = old / s;
    for (int n = block * c.block + tid / quads; n < from; n += step) {
      uint32_t *w = reinterpret_cast<uint32_t *>(codes + n * c.stride_t + d);
      *w = kv_encode4<CODE>(kv_decode4<CODE>(*w) * ratio);
    }
  }
  for (int n = lo + tid / quads; n < hi; n += step) {
    const f32x4 y = Row4<T>::load(x + (int64_t)(n - from) * st + d);
    *reinterpret_cast<uint32_t *>(codes + n * c.stride_t + d) = kv_is_nan(s) ? 0u : kv_encode4<CODE>(y / s);
  }
  if (tid == 0) *scale = s;
}

// 16 codes per thread.
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
  for (int i = 0; i < 4; i++) Row4<T>::store(out + 4 * i, kv_decode4<CODE>(w[i]) * s);
}

}  // namespace

ns_status launch_kv_append(const ns_kv_cache &c, int tokens, int dtype, const void *k, const void *v, int64_t sb, int64_t sh,
                           int64_t st, const int32_t *start, const int32_t *counts, hipStream_t s) {
  // the blocks that so many tokens touch where they begin at a block's last position
  const int blocks = min((tokens + c.block - 2) / c.block + 1, c.capacity / c.block);
  const dim3 grid((unsigned)blocks, (unsigned)c.heads_kv * 2, (unsigned)c.batch);
  auto go = [&](auto kernel, auto *kp, auto *vp) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, c, tokens, kp, vp, sb, sh, st, start, counts); };
  if (dtype == NS_F32) {
    const float *kp = static_cast<const float *>(k), *vp = static_cast<const float *>(v);
    c.code == NS_CODE_I8 ? go(kv_append_kernel<float, NS_CODE_I8>, kp, vp) : go(kv_append_kernel<float, NS_CODE_E4M3>, kp, vp);
  } else {
    const bf16_t *kp = static_cast<const bf16_t *>(k), *vp = static_cast<const bf16_t *>(v);
    c.code == NS_CODE_I8 ? go(kv_append_kernel<bf16_t, NS_CODE_I8>, kp, vp) : go(kv_append_kernel<bf16_t, NS_CODE_E4M3>, kp, vp);
  }
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
