// Eviction from the 8-bit key/value cache by added-up weight: which tokens stay (kv_select_kernel), and their move into
// another cache, where every block gets the scale that its tokens need (kv_move_kernel).
#include "ns_kv.h"

namespace ns {

namespace {

constexpr int kSelect = 1024, kMove = 256;

// larger weight <=> larger key; -0 and +0 alike, NaN above everything.  0 is nobody's key.
__device__ __forceinline__ uint32_t rank_key(float w) {
  if (!(w == w)) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// One workgroup per sequence and head: the key of the last token that stays, by four digits of 8 bits (radix select), then the
// kept tokens in order of their positions, among equal keys the first ones.
__global__ __launch_bounds__(kSelect) void kv_select_kernel(const float *weights, const int32_t *lengths, int capacity, int keep, int n_global,
                                                            int n_recent, int heads_kv, int to_capacity, int32_t *kept, float *w_out,
                                                            int32_t *lengths_out) {
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int length = kv_length(lengths, b, capacity);
  const int64_t row = (int64_t)b * heads_kv + h;
  const float *w = weights + row * capacity;
  kept += row * keep;
  w_out += row * to_capacity;
  if (h == 0 && tid == 0) lengths_out[b] = min(length, keep);
  if (length <= keep) {
    for (int i = tid; i < to_capacity; i += kSelect) {
      if (i < keep) kept[i] = i < length ? i : -1;
      w_out[i] = i < length ? w[i] : 0.f;
    }
    return;
  }
  const int first = n_global, last = length - n_recent;                // the ranked ones: first <= n < last
  __shared__ uint32_t hist[256], total[kSelect / 64], found[2];
  uint32_t prefix = 0, mask = 0, need = (uint32_t)(keep - n_global - n_recent);
  for (int shift = 24; need && shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int n = first + tid; n < last; n += kSelect) {
      const uint32_t key = rank_key(w[n]);
      if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      int digit = 255;
      uint32_t above = 0;
      while (above + hist[digit] < need) above += hist[digit--];
      found[0] = (uint32_t)digit;
      found[1] = need - above;
    }
    __syncthreads();
    prefix |= found[0] << shift;
    mask |= 255u << shift;
    need = found[1];
    __syncthreads();
  }
  // prefix: the key of the last token that stays; need: how many of those with this very key stay
  uint32_t placed = 0, equal = 0;
  const bool ranked = keep > n_global + n_recent;
  for (int at = 0; at < length; at += kSelect) {
    const int n = at + tid;
    const float x = n < length ? w[n] : 0.f;
    const bool in = n >= first && n < last;
    const uint32_t key = rank_key(x);
    const bool eq = ranked && in && key == prefix;
    const unsigned long long eqs = __ballot(eq);
    __syncthreads();
    if (lane == 0) total[wave] = (uint32_t)__popcll(eqs);
    __syncthreads();
    uint32_t before = equal, all = 0;
    for (int i = 0; i < kSelect / 64; i++) {
      before += i < wave ? total[i] : 0u;
      all += total[i];
    }
    equal += all;
    const bool stays = n < length && (!in || (ranked && (key > prefix || (eq && before + (uint32_t)__popcll(eqs & ((1ull << lane) - 1)) < need))));
    const unsigned long long st = __ballot(stays);
    __syncthreads();
    if (lane == 0) total[wave] = (uint32_t)__popcll(st);
    __syncthreads();
    before = placed;
    all = 0;
    for (int i = 0; i < kSelect / 64; i++) {
      before += i < wave ? total[i] : 0u;
      all += total[i];
    }
    placed += all;
    if (stays) {
      const uint32_t to = before + (uint32_t)__popcll(st & ((1ull << lane) - 1));
      kept[to] = n;
      w_out[to] = x;
    }
  }
  for (int i = keep + tid; i < to_capacity; i += kSelect) w_out[i] = 0.f;
}

// One workgroup per block of the new cache, head, and keys or values.
template <int CODE>
__global__ __launch_bounds__(kMove) void kv_move_kernel(ns_kv_cache from, ns_kv_cache to, const int32_t *lengths, const int32_t *kept, int keep) {
  const int b = blockIdx.z, h = blockIdx.y >> 1, value = blockIdx.y & 1, tid = threadIdx.x, block = blockIdx.x;
  const int lo = block * to.block, hi = min(lo + to.block, min(kv_length(lengths, b, from.capacity), keep));
  if (lo >= hi) return;
  const int64_t row = (int64_t)b * to.heads_kv + h;
  const int quads = to.head_dim / 4, d = tid % quads * 4, step = kMove / quads;
  const uint8_t *src = static_cast<const uint8_t *>(value ? from.v : from.k) + b * from.stride_b + h * from.stride_h + d;
  const float *src_scale = (value ? from.v_scale : from.k_scale) + row * (from.capacity / from.block);
  uint8_t *dst = static_cast<uint8_t *>(value ? to.v : to.k) + b * to.stride_b + h * to.stride_h + d;
  kept += row * keep;
  uint32_t most = 0;
  for (int i = lo + tid / quads; i < hi; i += step) {
    const int n = kept[i];
    const f32x4 x = kv_decode4<CODE>(*reinterpret_cast<const uint32_t *>(src + n * from.stride_t)) * src_scale[n / from.block];
#pragma unroll
    for (int j = 0; j < 4; j++) most = max(most, __float_as_uint(x[j]) & 0x7fffffffu);
  }
  __shared__ uint32_t largest[kMove / 64];
#pragma unroll
  for (int o = 32; o; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
  if (tid % 64 == 0) largest[tid / 64] = most;
  __syncthreads();
  most = max(max(largest[0], largest[1]), max(largest[2], largest[3]));
  const float s = kv_scale_for<CODE>(most);
  for (int i = lo + tid / quads; i < lo + to.block; i += step) {
    uint32_t w = 0;
    if (i < hi && !kv_is_nan(s)) {
      const int n = kept[i];
      w = kv_encode4<CODE>(kv_decode4<CODE>(*reinterpret_cast<const uint32_t *>(src + n * from.stride_t)) * src_scale[n / from.block] / s);
    }
    *reinterpret_cast<uint32_t *>(dst + i * to.stride_t) = w;
  }
  if (tid == 0) (value ? to.v_scale : to.k_scale)[row * (to.capacity / to.block) + block] = s;
}

}  // namespace

size_t kv_evict_workspace_bytes(const ns_kv_cache &, int) { return 0; }

ns_status launch_kv_evict(const ns_kv_cache &from, const ns_kv_cache &to, const float *weights, const int32_t *lengths, int keep,
                          int n_global, int n_recent, int32_t *kept, float *w_out, int32_t *lengths_out, void *, hipStream_t s) {
  hipLaunchKernelGGL(kv_select_kernel, dim3((unsigned)from.heads_kv, (unsigned)from.batch), dim3(kSelect), 0, s, weights, lengths, from.capacity,
                     keep, n_global, n_recent, from.heads_kv, to.capacity, kept, w_out, lengths_out);
  const ns_status st = check_launch("kv_select_kernel");
  if (st != NS_OK) return st;
  const dim3 grid((unsigned)((keep + to.block - 1) / to.block), (unsigned)to.heads_kv * 2, (unsigned)to.batch);
  if (to.code == NS_CODE_I8)
    hipLaunchKernelGGL(kv_move_kernel<NS_CODE_I8>, grid, dim3(kMove), 0, s, from, to, lengths, kept, keep);
  else
    hipLaunchKernelGGL(kv_move_kernel<NS_CODE_E4M3>, grid, dim3(kMove), 0, s, from, to, lengths, kept, keep);
  return check_launch("kv_move_kernel");
}

}  // namespace ns
