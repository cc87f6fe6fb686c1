// C ABI of the 8-bit key/value cache: host-side validation and dispatch.  No kernel lives here.
#include "ns_kv.h"

namespace ns {
namespace {

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline int64_t elt_size(int dtype) { return dtype == NS_F32 ? 4 : 2; }

ns_status validate_cache(const ns_kv_cache *c) {
  if (!c) return fail(NS_ERR_INVALID_ARG, "cache is NULL");
  if (c->batch < 1 || c->heads_kv < 1 || c->head_dim < 1 || c->capacity < 1 || c->block < 1)
    return fail(NS_ERR_INVALID_ARG, "the cache's batch, heads_kv, head_dim, capacity and block must be positive");
  if (c->code != NS_CODE_I8 && c->code != NS_CODE_E4M3) return fail(NS_ERR_INVALID_ARG, "code must be NS_CODE_I8 or NS_CODE_E4M3");
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
    return fail(NS_ERR_UNSUPPORTED, "head_dim %d: only 64, 128 and 256 are implemented", c->head_dim);
  if (c->block != 32 && c->block != 64 && c->block != 128)
    return fail(NS_ERR_UNSUPPORTED, "blocks of %d tokens: only 32, 64 and 128 are implemented", c->block);
  if (c->capacity % c->block) return fail(NS_ERR_INVALID_ARG, "capacity (%d) must be a multiple of block (%d)", c->capacity, c->block);
  if (c->capacity > (1 << 30)) return fail(NS_ERR_UNSUPPORTED, "capacity above 2^30");
  if (c->batch > 65535) return fail(NS_ERR_UNSUPPORTED, "batch above 65535");
  if (c->heads_kv > 1024) return fail(NS_ERR_UNSUPPORTED, "more than 1024 key/value heads");
  if (c->stride_t > (1 << 25)) return fail(NS_ERR_UNSUPPORTED, "tokens more than 2^25 bytes apart");
  if (c->stride_t < c->head_dim || c->stride_t % 16 || c->stride_h % 16 || c->stride_b % 16 || c->stride_h < 0 || c->stride_b < 0)
    return fail(NS_ERR_INVALID_ARG, "the cache's strides must be non-negative multiples of 16 bytes, stride_t >= head_dim");
  return NS_OK;
}

ns_status validate_cache_memory(const ns_kv_cache *c) {
  const ns_status st = validate_cache(c);
  if (st != NS_OK) return st;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale) return fail(NS_ERR_INVALID_ARG, "the cache's k, v, k_scale and v_scale must not be NULL");
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return fail(NS_ERR_INVALID_ARG, "the cache's k and v must be 16-byte aligned");
  if (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return fail(NS_ERR_INVALID_ARG, "the cache's scales are misaligned");
  if (c->k == c->v || c->k_scale == c->v_scale) return fail(NS_ERR_INVALID_ARG, "the cache's keys and values must not share memory");
  return NS_OK;
}

// rows that a call writes lie apart (rows that it only reads may be one and the same, as a prefix that all sequences share)
ns_status validate_apart(int64_t sb, int64_t sh, int batch, int heads, int D, const char *what) {
  if ((batch > 1 && sb < D) || (heads > 1 && sh < D))
    return fail(NS_ERR_INVALID_ARG, "%s is written: sequences and heads must not share rows", what);
  return NS_OK;
}

ns_status validate_dtype(int dtype) {
  return dtype == NS_F32 || dtype == NS_BF16 ? NS_OK : fail(NS_ERR_INVALID_ARG, "dtype must be NS_F32 or NS_BF16");
}

ns_status validate_rows(int64_t sb, int64_t sh, int64_t st, int dtype, int D, const char *what) {
  const int64_t unit = 16 / elt_size(dtype);
  if (st < D || sb < 0 || sh < 0 || sb % unit || sh % unit || st % unit)
    return fail(NS_ERR_INVALID_ARG, "%s strides must be non-negative, rows 16-byte aligned, stride_t >= head_dim", what);
  return NS_OK;
}

ns_status validate_counts(const int32_t *needed, const int32_t *optional) {
  if (!needed) return fail(NS_ERR_INVALID_ARG, "start / lengths must not be NULL");
  if (!aligned(needed, 4) || !aligned(optional, 4)) return fail(NS_ERR_INVALID_ARG, "start / lengths / counts misaligned");
  return NS_OK;
}

ns_status validate_attn(const ns_kv_cache *c, const ns_kv_attn_desc *d) {
  ns_status st = validate_cache(c);
  if (st != NS_OK) return st;
  if (!d) return fail(NS_ERR_INVALID_ARG, "descriptor is NULL");
  if (d->heads < 1 || d->tokens < 1) return fail(NS_ERR_INVALID_ARG, "heads and tokens must be positive");
  if (d->heads % c->heads_kv) return fail(NS_ERR_INVALID_ARG, "heads (%d) must be a multiple of heads_kv (%d)", d->heads, c->heads_kv);
  if (d->heads > 1024) return fail(NS_ERR_UNSUPPORTED, "more than 1024 query heads");
  if ((int64_t)d->heads * d->tokens > (1 << 24)) return fail(NS_ERR_UNSUPPORTED, "heads x tokens above 2^24");
  if ((int64_t)c->batch * c->heads_kv * ((c->capacity + 127) / 128) > 0x7fffffff) return fail(NS_ERR_UNSUPPORTED, "batch x heads_kv x capacity above 2^38");
  if ((st = validate_dtype(d->dtype)) != NS_OK) return st;
  if (!(d->scale - d->scale == 0.f)) return fail(NS_ERR_INVALID_ARG, "scale must be finite");
  if ((st = validate_rows(d->q_stride_b, d->q_stride_h, d->q_stride_t, d->dtype, c->head_dim, "q")) != NS_OK) return st;
  if ((st = validate_rows(d->out_stride_b, d->out_stride_h, d->out_stride_t, d->dtype, c->head_dim, "out")) != NS_OK) return st;
  return validate_apart(d->out_stride_b, d->out_stride_h, c->batch, d->heads, c->head_dim, "out");
}

ns_status check_workspace(const void *ws, size_t have, size_t need) {
  if (!need) return NS_OK;
  if (!ws) return fail(NS_ERR_WORKSPACE, "workspace is NULL, %zu bytes needed", need);
  if (!aligned(ws, 256)) return fail(NS_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (have < need) return fail(NS_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", have, need);
  return NS_OK;
}

ns_status validate_evict(const ns_kv_cache *from, int32_t keep) {
  const ns_status st = validate_cache(from);
  if (st != NS_OK) return st;
  if (keep < 1 || keep > from->capacity) return fail(NS_ERR_INVALID_ARG, "keep (%d) must be in [1, capacity = %d]", keep, from->capacity);
  return NS_OK;
}

}  // namespace
}  // namespace ns

using namespace ns;

extern "C" {

ns_status kv_cache_append(const ns_kv_cache *cache, int32_t tokens, int32_t dtype, const void *k, const void *v, int64_t stride_b,
                          int64_t stride_h, int64_t stride_t, const int32_t *start, const int32_t *counts, void *stream) {
  ns_status st = validate_cache_memory(cache);
  if (st != NS_OK) return st;
  if ((st = validate_apart(cache->stride_b, cache->stride_h, cache->batch, cache->heads_kv, cache->head_dim, "the cache")) != NS_OK) return st;
  if (tokens < 1) return fail(NS_ERR_INVALID_ARG, "tokens must be positive");
  if (tokens > (1 << 30)) return fail(NS_ERR_UNSUPPORTED, "more than 2^30 tokens");
  if ((st = validate_dtype(dtype)) != NS_OK) return st;
  if (!k || !v) return fail(NS_ERR_INVALID_ARG, "k and v must not be NULL");
  if (!aligned(k, 16) || !aligned(v, 16)) return fail(NS_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
  if (k == cache->k || v == cache->v || k == cache->v || v == cache->k) return fail(NS_ERR_INVALID_ARG, "the cache must not alias an input");
  if ((st = validate_rows(stride_b, stride_h, stride_t, dtype, cache->head_dim, "k/v")) != NS_OK) return st;
  if ((st = validate_counts(start, counts)) != NS_OK) return st;
  return launch_kv_append(*cache, tokens, dtype, k, v, stride_b, stride_h, stride_t, start, counts, static_cast<hipStream_t>(stream));
}

ns_status kv_cache_read(const ns_kv_cache *cache, const int32_t *lengths, int32_t first, int32_t tokens, int32_t dtype, void *k_out,
                        void *v_out, void *stream) {
  ns_status st = validate_cache_memory(cache);
  if (st != NS_OK) return st;
  if (first < 0 || tokens < 1 || tokens > cache->capacity || first > cache->capacity - tokens)
    return fail(NS_ERR_INVALID_ARG, "positions %d .. %lld are not within the capacity (%d)", first, (long long)first + tokens - 1, cache->capacity);
  if ((st = validate_dtype(dtype)) != NS_OK) return st;
  if ((st = validate_counts(lengths, nullptr)) != NS_OK) return st;
  if (!k_out || !v_out) return fail(NS_ERR_INVALID_ARG, "k_out and v_out must not be NULL");
  if (!aligned(k_out, 16) || !aligned(v_out, 16)) return fail(NS_ERR_INVALID_ARG, "k_out and v_out must be 16-byte aligned");
  if (k_out == v_out || k_out == cache->k || k_out == cache->v || v_out == cache->k || v_out == cache->v)
    return fail(NS_ERR_INVALID_ARG, "k_out and v_out must have memory of their own");
  return launch_kv_read(*cache, lengths, first, tokens, dtype, k_out, v_out, static_cast<hipStream_t>(stream));
}

size_t kv_cache_attn_workspace_bytes(const ns_kv_cache *cache, const ns_kv_attn_desc *desc, int32_t want_weights) {
  if (validate_attn(cache, desc) != NS_OK) return 0;
  return kv_attn_workspace_bytes(*cache, *desc, want_weights != 0);
}

ns_status kv_cache_attn(const ns_kv_cache *cache, const ns_kv_attn_desc *desc, const void *q, const int32_t *lengths,
                        const int32_t *counts, void *out, float *lse, const float *weights_in, float *weights_out,
                        void *workspace, size_t workspace_bytes, void *stream) {
  ns_status st = validate_attn(cache, desc);
  if (st == NS_OK) st = validate_cache_memory(cache);
  if (st == NS_OK) st = validate_counts(lengths, counts);
  if (st != NS_OK) return st;
  if (!q || !out) return fail(NS_ERR_INVALID_ARG, "q and out must not be NULL");
  if (!aligned(q, 16) || !aligned(out, 16)) return fail(NS_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
  if (!aligned(lse, 4) || !aligned(weights_in, 4) || !aligned(weights_out, 4)) return fail(NS_ERR_INVALID_ARG, "lse / weights misaligned");
  if (out == q || out == cache->k || out == cache->v) return fail(NS_ERR_INVALID_ARG, "out must not alias an input");
  if (weights_in && !weights_out) return fail(NS_ERR_INVALID_ARG, "weights_in without weights_out");
  st = check_workspace(workspace, workspace_bytes, kv_attn_workspace_bytes(*cache, *desc, weights_out != nullptr));
  if (st != NS_OK) return st;
  return launch_kv_attn(KvAttnArgs{*cache, *desc, q, lengths, counts, out, lse, weights_in, weights_out,
                                   static_cast<unsigned char *>(workspace), static_cast<hipStream_t>(stream)});
}

size_t kv_cache_evict_workspace_bytes(const ns_kv_cache *from, int32_t keep) {
  return validate_evict(from, keep) == NS_OK ? kv_evict_workspace_bytes(*from, keep) : 0;
}

ns_status kv_cache_evict(const ns_kv_cache *from, const ns_kv_cache *to, const float *weights, const int32_t *lengths, int32_t keep,
                         int32_t n_global, int32_t n_recent, int32_t *kept_idx, float *weights_out, int32_t *lengths_out,
                         void *workspace, size_t workspace_bytes, void *stream) {
  ns_status st = validate_evict(from, keep);
  if (st == NS_OK) st = validate_cache_memory(from);
  if (st == NS_OK) st = validate_cache_memory(to);
  if (st == NS_OK) st = validate_counts(lengths, nullptr);
  if (st != NS_OK) return st;
  if (to->batch != from->batch || to->heads_kv != from->heads_kv || to->head_dim != from->head_dim || to->block != from->block || to->code != from->code)
    return fail(NS_ERR_INVALID_ARG, "both caches must have the same batch, heads_kv, head_dim, block and code");
  if ((st = validate_apart(to->stride_b, to->stride_h, to->batch, to->heads_kv, to->head_dim, "the new cache")) != NS_OK) return st;
  if (to->capacity < keep) return fail(NS_ERR_INVALID_ARG, "the new cache has room for %d tokens, keep is %d", to->capacity, keep);
  if (n_global < 0 || n_recent < 0 || (int64_t)n_global + n_recent > keep)
    return fail(NS_ERR_INVALID_ARG, "n_global and n_recent must not be negative, nor their sum above keep");
  if (!weights || !kept_idx || !weights_out || !lengths_out)
    return fail(NS_ERR_INVALID_ARG, "weights, kept_idx, weights_out and lengths_out must not be NULL");
  if (!aligned(weights, 4) || !aligned(kept_idx, 4) || !aligned(weights_out, 4) || !aligned(lengths_out, 4))
    return fail(NS_ERR_INVALID_ARG, "misaligned pointer");
  if (weights_out == weights || lengths_out == lengths || to->k == from->k || to->v == from->v || to->k == from->v || to->v == from->k ||
      to->k_scale == from->k_scale || to->v_scale == from->v_scale || to->k_scale == from->v_scale || to->v_scale == from->k_scale)
    return fail(NS_ERR_INVALID_ARG, "the new cache and the outputs must have memory of their own");
  st = check_workspace(workspace, workspace_bytes, kv_evict_workspace_bytes(*from, keep));
  if (st != NS_OK) return st;
  return launch_kv_evict(*from, *to, weights, lengths, keep, n_global, n_recent, kept_idx, weights_out, lengths_out, workspace,
                         static_cast<hipStream_t>(stream));
}

}  // extern "C"
