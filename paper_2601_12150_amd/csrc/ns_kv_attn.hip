// Attention over the 8-bit key/value cache: one workgroup per query row, in plain fp32.
#include "ns_kv.h"

namespace ns {

namespace {

constexpr int kThreads = 256;

// <q, codes> of one key, fp32
template <int CODE>
__device__ __forceinline__ float dot_codes(const float *q, const uint8_t *codes, int D) {
  float a = 0.f;
  for (int d = 0; d < D; d += 16) {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(codes + d);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const f32x4 c = kv_decode4<CODE>(w[i]);
#pragma unroll
      for (int j = 0; j < 4; j++) a = __builtin_fmaf(q[d + 4 * i + j], c[j], a);
    }
  }
  return a;
}

// positions that query t sees: 0 .. limit - 1
__device__ __forceinline__ int seen_by(const ns_kv_attn_desc &d, int t, int length, int count) {
  return t >= count ? 0 : d.causal ? max(length - count + t + 1, 0) : length;
}

template <typename T> __device__ __forceinline__ T to_out(float x);
template <> __device__ __forceinline__ float to_out<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16_t to_out<bf16_t>(float x) { return (bf16_t)x; }

__device__ __forceinline__ float group_max(float x, float *tmp, int tid) {
  x = wave_max(x);
  __syncthreads();
  if (tid % 64 == 0) tmp[tid / 64] = x;
  __syncthreads();
  return fmaxf(fmaxf(tmp[0], tmp[1]), fmaxf(tmp[2], tmp[3]));
}

template <typename T, int CODE>
__global__ __launch_bounds__(kThreads) void kv_attn_row_kernel(ns_kv_cache c, ns_kv_attn_desc d, const T *q, const int32_t *lengths,
                                                               const int32_t *counts, T *out, float *lse) {
  const int t = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, D = c.head_dim;
  const int h = hq / (d.heads / c.heads_kv);
  const int limit = seen_by(d, t, kv_length(lengths, b, c.capacity), kv_count(counts, b, d.tokens));
  const uint8_t *k = static_cast<const uint8_t *>(c.k) + b * c.stride_b + h * c.stride_h;
  const uint8_t *v = static_cast<const uint8_t *>(c.v) + b * c.stride_b + h * c.stride_h;
  const int64_t blocks = ((int64_t)b * c.heads_kv + h) * (c.capacity / c.block);
  __shared__ float row[256], p[kThreads], tmp[4];
  if (tid < D) row[tid] = (float)q[b * d.q_stride_b + hq * d.q_stride_h + t * d.q_stride_t + tid];
  __syncthreads();
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int at = 0; at < limit; at += kThreads) {
    const int n = at + tid;
    const float z = n < limit ? dot_codes<CODE>(row, k + n * c.stride_t, D) * (c.k_scale[blocks + n / c.block] * d.scale) : -INFINITY;
    const float next = fmaxf(m, group_max(z, tmp, tid));
    const float ref = next == -INFINITY ? 0.f : next, fade = __expf(m - ref);
    p[tid] = z == -INFINITY ? 0.f : __expf(z - ref);
    __syncthreads();
    l *= fade;
    o *= fade;
    const int here = min(kThreads, limit - at);
    for (int j = 0; j < here; j++) {
      l += p[j];
      if (tid < D) {
        const uint32_t w = v[(at + j) * c.stride_t + tid];
        o = __builtin_fmaf(p[j] * c.v_scale[blocks + (at + j) / c.block], kv_decode4<CODE>(w)[0], o);
      }
    }
    m = next;
  }
  if (tid < D) out[b * d.out_stride_b + hq * d.out_stride_h + t * d.out_stride_t + tid] = to_out<T>(limit ? o / l : 0.f);
  if (tid == 0 && lse) lse[((int64_t)b * d.heads + hq) * d.tokens + t] = limit ? m + __logf(l) : -INFINITY;
}

// One thread per position: the sum over all rows that read its head.
template <typename T, int CODE>
__global__ __launch_bounds__(kThreads) void kv_weights_kernel(ns_kv_cache c, ns_kv_attn_desc d, const T *q, const int32_t *lengths,
                                                              const int32_t *counts, const float *lse, const float *w_in, float *w_out) {
  const int n = blockIdx.x * kThreads + threadIdx.x, h = blockIdx.y, b = blockIdx.z, D = c.head_dim, G = d.heads / c.heads_kv;
  const int length = kv_length(lengths, b, c.capacity), count = kv_count(counts, b, d.tokens);
  __shared__ float row[256];
  float sum = 0.f;
  for (int g = 0; g < G; g++)
    for (int t = 0; t < count; t++) {
      __syncthreads();
      if ((int)threadIdx.x < D) row[threadIdx.x] = (float)q[b * d.q_stride_b + (h * G + g) * d.q_stride_h + t * d.q_stride_t + threadIdx.x];
      __syncthreads();
      if (n < seen_by(d, t, length, count)) {
        const float s = c.k_scale[((int64_t)b * c.heads_kv + h) * (c.capacity / c.block) + n / c.block] * d.scale;
        sum += __expf(dot_codes<CODE>(row, static_cast<const uint8_t *>(c.k) + b * c.stride_b + h * c.stride_h + n * c.stride_t, D) * s -
                      lse[((int64_t)b * d.heads + h * G + g) * d.tokens + t]);
      }
    }
  const int64_t at = ((int64_t)b * c.heads_kv + h) * c.capacity + n;
  if (n < c.capacity && (n < length || w_in != w_out)) w_out[at] = (w_in ? w_in[at] : 0.f) + sum;
}

template <typename T, int CODE>
ns_status launch(const KvAttnArgs &a) {
  const T *q = static_cast<const T *>(a.q);
  float *lse = a.lse ? a.lse : reinterpret_cast<float *>(a.ws);
  hipLaunchKernelGGL((kv_attn_row_kernel<T, CODE>), dim3((unsigned)a.d.tokens, (unsigned)a.d.heads, (unsigned)a.c.batch), dim3(kThreads), 0,
                     a.stream, a.c, a.d, q, a.lengths, a.counts, static_cast<T *>(a.out), lse);
  const ns_status st = check_launch("kv_attn_row_kernel");
  if (st != NS_OK || !a.w_out) return st;
  hipLaunchKernelGGL((kv_weights_kernel<T, CODE>), dim3((unsigned)((a.c.capacity + kThreads - 1) / kThreads), (unsigned)a.c.heads_kv, (unsigned)a.c.batch),
                     dim3(kThreads), 0, a.stream, a.c, a.d, q, a.lengths, a.counts, lse, a.w_in, a.w_out);
  return check_launch("kv_weights_kernel");
}

}  // namespace

size_t kv_attn_workspace_bytes(const ns_kv_cache &c, const ns_kv_attn_desc &d, bool weights) {
  return weights ? align_up((size_t)c.batch * d.heads * d.tokens * 4, 256) : 0;
}

ns_status launch_kv_attn(const KvAttnArgs &a) {
  if (a.d.dtype == NS_F32) return a.c.code == NS_CODE_I8 ? launch<float, NS_CODE_I8>(a) : launch<float, NS_CODE_E4M3>(a);
  return a.c.code == NS_CODE_I8 ? launch<bf16_t, NS_CODE_I8>(a) : launch<bf16_t, NS_CODE_E4M3>(a);
}

}  // namespace ns
