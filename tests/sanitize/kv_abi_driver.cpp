// Walks the host side of the key/value cache's entry points (validation, workspace sizes and layout, messages) at the ends of what their
// arguments hold, without touching a GPU: every call below only computes a size or is refused before anything is launched.  Built with
// -fsanitize=address,undefined on the host pass by tests/test_kv_sanitizers_cpu.py.
#include <initializer_list>
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "../../include/nsattn.h"

static int fails = 0;
#define EXPECT(cond)                                                     \
  do {                                                                   \
    if (!(cond)) { printf("FAILED line %d: %s\n", __LINE__, #cond); fails++; } \
  } while (0)

static void *at(int i) { return reinterpret_cast<void *>((uintptr_t)0x100000000 * (uintptr_t)(i + 1)); }

static ns_kv_cache cache(int batch, int heads, int D, int capacity, int block, int code, int where = 0) {
  ns_kv_cache c;
  memset(&c, 0, sizeof(c));
  c.batch = batch; c.heads_kv = heads; c.head_dim = D; c.capacity = capacity; c.block = block; c.code = code;
  c.stride_t = D; c.stride_h = (int64_t)capacity * D; c.stride_b = c.stride_h * heads;
  c.k = at(where); c.v = at(where + 1);
  c.k_scale = static_cast<float *>(at(where + 2)); c.v_scale = static_cast<float *>(at(where + 3));
  return c;
}
static ns_kv_attn_desc desc(int heads, int tokens, int D, int dtype) {
  ns_kv_attn_desc d;
  memset(&d, 0, sizeof(d));
  d.heads = heads; d.tokens = tokens; d.dtype = dtype; d.causal = 1; d.scale = 0.1f;
  d.q_stride_t = d.out_stride_t = D; d.q_stride_h = d.out_stride_h = (int64_t)tokens * D; d.q_stride_b = d.out_stride_b = d.q_stride_h * heads;
  return d;
}

int main() {
  const int32_t *counts = static_cast<const int32_t *>(at(20));
  float *w = static_cast<float *>(at(21)), *w2 = static_cast<float *>(at(22));
  int32_t *kept = static_cast<int32_t *>(at(23)), *left = static_cast<int32_t *>(at(24));
  // sizes, from one token to the most, and what a workspace that is too small, misplaced or missing is called
  for (int D : {64, 128, 256})
    for (int block : {32, 128})
      for (int code : {(int)NS_CODE_I8, (int)NS_CODE_E4M3})
        for (int capacity : {128, 4096, 16384, 16512, 131072, 1 << 30})
          for (int batch : {1, 7, 65535})
            for (int heads : {1, 8, 1024}) {
              const ns_kv_cache c = cache(batch, heads, D, capacity, block, code);
              const bool many = (int64_t)batch * heads * ((capacity + 127) / 128) > INT32_MAX;
              for (int group : {1, 8})
                for (int tokens : {1, 2, 5, 33, 4096, 1 << 14})
                  for (int dtype : {(int)NS_F32, (int)NS_BF16})
                    for (int weights : {0, 1}) {
                      if (heads * group > 1024) continue;
                      const ns_kv_attn_desc d = desc(heads * group, tokens, D, dtype);
                      const size_t need = kv_cache_attn_workspace_bytes(&c, &d, weights);
                      EXPECT(!many || need == 0);
                      EXPECT(need % 256 == 0);
                      if (!need) continue;
                      EXPECT(kv_cache_attn(&c, &d, at(10), counts, nullptr, at(11), nullptr, nullptr, weights ? w : nullptr, nullptr, 0, nullptr) == NS_ERR_WORKSPACE);
                      EXPECT(kv_cache_attn(&c, &d, at(10), counts, nullptr, at(11), nullptr, nullptr, weights ? w : nullptr, at(12), need - 1, nullptr) == NS_ERR_WORKSPACE);
                    }
              for (int keep : {1, 100, capacity}) {
                const size_t need = kv_cache_evict_workspace_bytes(&c, keep);
                EXPECT((need == 0) == (capacity <= 16384));
                if (!need) continue;
                const ns_kv_cache to = cache(batch, heads, D, capacity, block, code, 4);
                EXPECT(kv_cache_evict(&c, &to, w, counts, keep, 0, 0, kept, w2, left, nullptr, 0, nullptr) == NS_ERR_WORKSPACE);
                EXPECT(kv_cache_evict(&c, &to, w, counts, keep, 0, 0, kept, w2, left, at(12), need - 1, nullptr) == NS_ERR_WORKSPACE);
                EXPECT(kv_cache_evict(&c, &to, w, counts, keep, INT_MAX, INT_MAX, kept, w2, left, at(12), need, nullptr) == NS_ERR_INVALID_ARG);
                EXPECT(kv_cache_evict(&c, &to, w, counts, keep, INT_MIN, INT_MAX, kept, w2, left, at(12), need, nullptr) == NS_ERR_INVALID_ARG);
              }
            }
  // numbers at the ends of their types
  const int ends[] = {INT_MIN, -1, 0, INT_MAX};
  const ns_kv_cache good = cache(2, 4, 128, 256, 64, NS_CODE_I8);
  const ns_kv_attn_desc plain = desc(8, 3, 128, NS_BF16);
  for (int x : ends) {
    for (int field = 0; field < 6; field++) {
      ns_kv_cache c = good;
      int32_t *const fields[] = {&c.batch, &c.heads_kv, &c.head_dim, &c.capacity, &c.block, &c.code};
      *fields[field] = x;
      if (field == 5 && x == 0) continue;
      EXPECT(kv_cache_append(&c, 1, NS_BF16, at(10), at(11), 128, 128, 128, counts, nullptr, nullptr) != NS_OK);
      EXPECT(kv_cache_read(&c, counts, 0, 1, NS_BF16, at(10), at(11), nullptr) != NS_OK);
      EXPECT(kv_cache_attn_workspace_bytes(&c, &plain, 1) == 0);
      EXPECT(kv_cache_evict_workspace_bytes(&c, 10) == 0);
    }
    EXPECT(kv_cache_append(&good, x, x ? NS_BF16 : 9, at(10), at(11), 128, 128, 128, counts, nullptr, nullptr) != NS_OK);
    EXPECT(kv_cache_read(&good, counts, x, INT_MAX, NS_F32, at(10), at(11), nullptr) != NS_OK);
    EXPECT(kv_cache_read(&good, counts, INT_MAX, x, NS_F32, at(10), at(11), nullptr) != NS_OK);
    EXPECT(kv_cache_evict_workspace_bytes(&good, x) == 0);
    for (int field = 0; field < 3; field++) {
      ns_kv_attn_desc d = plain;
      int32_t *const fields[] = {&d.heads, &d.tokens, &d.dtype};
      *fields[field] = x;
      if (field == 2 && x == 0) continue;
      EXPECT(kv_cache_attn(&good, &d, at(10), counts, nullptr, at(11), nullptr, nullptr, nullptr, at(12), (size_t)1 << 40, nullptr) != NS_OK);
    }
  }
  for (int64_t x : {INT64_MIN, (int64_t)-16, (int64_t)8, INT64_MAX}) {
    for (int field = 0; field < 3; field++) {
      ns_kv_cache c = good;
      int64_t *const fields[] = {&c.stride_b, &c.stride_h, &c.stride_t};
      *fields[field] = x;
      EXPECT(kv_cache_read(&c, counts, 0, 1, NS_BF16, at(10), at(11), nullptr) != NS_OK);
    }
    for (int field = 0; field < 6; field++) {
      ns_kv_attn_desc d = plain;
      int64_t *const fields[] = {&d.q_stride_b, &d.q_stride_h, &d.q_stride_t, &d.out_stride_b, &d.out_stride_h, &d.out_stride_t};
      *fields[field] = x == 8 ? 4 : x;
      EXPECT(kv_cache_attn_workspace_bytes(&good, &d, 1) == 0);
      EXPECT(kv_cache_append(&good, 3, NS_F32, at(10), at(11), field == 0 ? x | 1 : 512, field == 1 ? x | 1 : 512, field == 2 ? x | 1 : 127, counts, nullptr, nullptr) != NS_OK);
    }
  }
  for (float x : {INFINITY, -INFINITY, NAN}) {
    ns_kv_attn_desc d = plain;
    d.scale = x;
    EXPECT(kv_cache_attn_workspace_bytes(&good, &d, 0) == 0);
  }
  EXPECT(kv_cache_attn_workspace_bytes(nullptr, &plain, 0) == 0 && kv_cache_attn_workspace_bytes(&good, nullptr, 0) == 0);
  EXPECT(kv_cache_evict_workspace_bytes(nullptr, 1) == 0);
  EXPECT(strlen(ns_last_error()) > 0);
  if (fails) return 1;
  printf("key/value cache sanitizer run ok\n");
  return 0;
}
