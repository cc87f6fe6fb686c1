// Eviction from the 8-bit key/value cache by added-up weight: which tokens stay, and their move into another cache, where every block
// gets the scale that its tokens need.
//
// The tokens that stay are found by the key (an order-preserving integer image of the weight) of the last of them: digits of 11,
// 11 and 10 bits, each from a histogram of the keys that share the digits before it (radix select).  Then all tokens with a larger
// key stay, and of those with this very key the first ones.
//   kv_select_kernel: caches of up to 16384 tokens; one workgroup per sequence and head has all keys in registers, one launch.
//   kv_digit_kernel, kv_place_kernel: longer ones, a workgroup per 8192 tokens, or as many times that as leave 64 of them; a launch for every digit
//     and one that places.
//   kv_move_kernel: a workgroup per block of the new cache; its codes are read once and stay in registers until the scale is known.
// Measured: selection among 577 tokens 7.6 us, among 16000 (64 sequences and heads) 23 us, both bound by the barriers between the passes; among
// 131001 (8 heads) 7 + 9 + 9 + 12 us, bound by launches and the sums over all workgroups' histograms.  The move: 32768 tokens of 8 heads of 128
// channels 33 us (134 MB, 4.1 TB/s), bound by the reads and writes of rows of 128 bytes.
#include "ns_kv.h"

namespace ns {

namespace {

constexpr int kSelect = 1024, kWaves = kSelect / 64;
constexpr int kBits[3] = {11, 11, 10}, kShift[3] = {21, 10, 0}, kBins = 2048;
// Tokens that one workgroup selects from: 8 heads' 16384 to 1000 take 21 us with, 31 without (the move included); one of 32768 would take
// 34 against 32.
constexpr int kHeld = 16384;
constexpr int kChunkKeys = 8, kPiece = kSelect * kChunkKeys;
// Chunks of a sequence and head, each with a workgroup and one piece or several: every workgroup reads all chunks' histograms, which without
// an end to their number would be work that grows with the square of the capacity (8 heads' 2^20 tokens to 4096: 119 us, 259 with a workgroup
// for every piece; 2^22: 244 and 3206).
constexpr int kMostChunks = 64;

// larger weight <=> larger key; -0 and +0 alike, NaN above everything
__device__ __forceinline__ uint32_t rank_key(float w) {
  if (!(w == w)) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ uint32_t digit_of(uint32_t key, int pass) { return (key >> kShift[pass]) & ((1u << kBits[pass]) - 1); }

struct Choice { uint32_t digit, need, above; };   // the digit, how many of its keys are needed, how many keys lie above it

// The digit that the need-th largest key has, need >= 1; thread t brings the counts of the digits 2 t and 2 t + 1.  All threads call.
__device__ __forceinline__ Choice choose(uint32_t n0, uint32_t n1, uint32_t need, int tid, uint32_t *shared /* [kWaves + 3] */) {
  const int lane = tid & 63, wave = tid >> 6;
  uint32_t from = n0 + n1;                        // of this lane's digits and those above, in the wave
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = (uint32_t)__shfl_down((int)from, o);
    from += lane + o < 64 ? x : 0u;
  }
  if (lane == 0) shared[wave] = from;
  __syncthreads();
  uint32_t above = from - n0 - n1;
  for (int w = wave + 1; w < kWaves; w++) above += shared[w];
  if (above < need && need <= above + n1) {
    shared[kWaves] = 2 * tid + 1; shared[kWaves + 1] = need - above; shared[kWaves + 2] = above;
  } else if (above + n1 < need && need <= above + n1 + n0) {
    shared[kWaves] = 2 * tid; shared[kWaves + 1] = need - above - n1; shared[kWaves + 2] = above + n1;
  }
  __syncthreads();
  const Choice c{shared[kWaves], shared[kWaves + 1], shared[kWaves + 2]};
  __syncthreads();
  return c;
}

struct SelectArgs {
  const float *weights;
  const int32_t *lengths;
  int capacity, keep, n_global, n_recent, heads_kv, to_capacity;
  int pieces;                                     // of a chunk
  int32_t *kept;
  float *w_out;
  int32_t *lengths_out;
};

// A sequence that stays whole; true if it is one.  part of parts: which share of the outputs.
__device__ __forceinline__ bool all_stay(const SelectArgs &a, int64_t row, int length, int part, int parts, int tid) {
  if (length > a.keep) {
    for (int i = a.keep + part * kSelect + tid; i < a.to_capacity; i += parts * kSelect) a.w_out[row * a.to_capacity + i] = 0.f;
    return false;
  }
  for (int i = part * kSelect + tid; i < a.to_capacity; i += parts * kSelect) {
    if (i < a.keep) a.kept[row * a.keep + i] = i < length ? i : -1;
    a.w_out[row * a.to_capacity + i] = i < length ? a.weights[row * a.capacity + i] : 0.f;
  }
  return true;
}

// Writes the tokens that stay of KPT * 1024 tokens from `base`: thread's token i is base + wave * 64 KPT + 64 i + lane.  placed, equal: how
// many stay, and how many have the border's key, before these; those of these are added where more follow.
template <int KPT>
__device__ __forceinline__ void place(const SelectArgs &a, int64_t row, const float *w, const uint32_t (&key)[KPT], int base, int length,
                                      uint32_t border, uint32_t need, bool ranked, uint32_t &placed, uint32_t &equal, bool more, int tid,
                                      uint32_t *shared /* [2 kWaves] */) {
  const int lane = tid & 63, wave = tid >> 6;
  const int first = a.n_global, last = length - a.n_recent;
  const unsigned long long below = (1ull << lane) - 1;
  const int n0 = base + wave * 64 * KPT + lane;
  uint32_t sure = 0, eqs = 0;                     // of the wave: tokens that stay in any case, and with the border's key
#pragma unroll
  for (int i = 0; i < KPT; i++) {
    const int n = n0 + 64 * i;
    const bool in = n >= first && n < last;
    sure += (uint32_t)__popcll(__ballot(n < length && (!in || (ranked && key[i] > border))));
    eqs += (uint32_t)__popcll(__ballot(in && ranked && key[i] == border));
  }
  if (lane == 0) {
    shared[wave] = sure;
    shared[kWaves + wave] = eqs;
  }
  __syncthreads();
  // all tokens before this wave that stay: the sure ones, and of those with the border's key the first `need`
  uint32_t at = placed, eq = equal;
  for (int x = 0; x < wave; x++) {
    at += shared[x];
    eq += shared[kWaves + x];
  }
  for (int x = 0; more && x < kWaves; x++) {
    placed += shared[x];
    equal += shared[kWaves + x];
  }
#pragma unroll
  for (int i = 0; i < KPT; i++) {
    const int n = n0 + 64 * i;
    const bool in = n >= first && n < last;
    const bool is_sure = n < length && (!in || (ranked && key[i] > border)), is_eq = in && ranked && key[i] == border;
    const unsigned long long s = __ballot(is_sure), e = __ballot(is_eq);
    const uint32_t eq_here = eq + (uint32_t)__popcll(e & below);
    if (is_sure || (is_eq && eq_here < need)) {
      const uint32_t to = at + (uint32_t)__popcll(s & below) + min(eq_here, need);
      a.kept[row * a.keep + to] = n;
      a.w_out[row * a.to_capacity + to] = w[n];
    }
    at += (uint32_t)__popcll(s);
    eq += (uint32_t)__popcll(e);
  }
}

template <int KPT>
__global__ __launch_bounds__(kSelect) void kv_select_kernel(SelectArgs a) {
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int length = kv_length(a.lengths, b, a.capacity);
  const int64_t row = (int64_t)b * a.heads_kv + h;
  if (h == 0 && tid == 0) a.lengths_out[b] = min(length, a.keep);
  if (all_stay(a, row, length, 0, 1, tid)) return;
  const float *w = a.weights + row * a.capacity;
  __shared__ __attribute__((aligned(8))) uint32_t hist[kBins];
  __shared__ uint32_t shared[2 * kWaves + 3];
  const int first = a.n_global, last = length - a.n_recent;
  uint32_t key[KPT];
#pragma unroll
  for (int i = 0; i < KPT; i++) {
    const int n = wave * 64 * KPT + 64 * i + lane;
    key[i] = n < length ? rank_key(w[n]) : 0u;
  }
  uint32_t prefix = 0, need = (uint32_t)(a.keep - a.n_global - a.n_recent);
  const bool ranked = need > 0;
  if (ranked) {
#pragma unroll
    for (int pass = 0; pass < 3; pass++) {
      *reinterpret_cast<u32x2 *>(&hist[2 * tid]) = u32x2{0, 0};
      __syncthreads();
      const uint32_t mask = pass == 0 ? 0u : ~0u << kShift[pass - 1];
#pragma unroll
      for (int i = 0; i < KPT; i++) {
        const int n = wave * 64 * KPT + 64 * i + lane;
        if (n >= first && n < last && (key[i] & mask) == prefix) atomicAdd(&hist[digit_of(key[i], pass)], 1u);
      }
      __syncthreads();
      const u32x2 counts = *reinterpret_cast<const u32x2 *>(&hist[2 * tid]);
      const Choice c = choose(counts[0], counts[1], need, tid, shared);
      prefix |= c.digit << kShift[pass];
      need = c.need;
    }
  }
  uint32_t placed = 0, equal = 0;
  place<KPT>(a, row, w, key, 0, length, prefix, need, ranked, placed, equal, false, tid, shared);
}

// ---- longer caches.  Scratch of a sequence and head: a histogram for every digit and chunk, the border's digits so far, and how many of each
// chunk's keys lie above them.
struct Scratch {
  uint32_t *hist;       // [3][chunks][kBins]
  uint32_t *border;     // [3][2]: after the digit: the key's digits, and how many of its keys are needed
  uint32_t *above;      // [2][chunks]: keys above the first digit; those that share it above the second
};
inline __host__ __device__ size_t scratch_words(int chunks) { return (size_t)3 * chunks * kBins + 8 + 2 * (size_t)chunks; }
__device__ __forceinline__ Scratch scratch_of(uint32_t *ws, int64_t row, int chunks) {
  uint32_t *p = ws + row * scratch_words(chunks);
  return Scratch{p, p + (size_t)3 * chunks * kBins, p + (size_t)3 * chunks * kBins + 8};
}

// The keys of a piece, in the places that place() has them
__device__ __forceinline__ void load_keys(const float *w, int base, int length, int wave, int lane, uint32_t (&key)[kChunkKeys]) {
  const int n0 = base + wave * 64 * kChunkKeys + lane;
#pragma unroll
  for (int i = 0; i < kChunkKeys; i++) key[i] = n0 + 64 * i < length ? rank_key(w[n0 + 64 * i]) : 0u;
}

// Sums over the workgroup
__device__ __forceinline__ u32x2 group_sum(u32x2 x, int tid, uint32_t *shared /* [2 kWaves] */) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += u32x2{(uint32_t)__shfl_xor((int)x[0], o), (uint32_t)__shfl_xor((int)x[1], o)};
  if ((tid & 63) == 0) {
    shared[tid >> 6] = x[0];
    shared[kWaves + (tid >> 6)] = x[1];
  }
  __syncthreads();
  u32x2 sum = {0, 0};
  for (int w = 0; w < kWaves; w++) sum += u32x2{shared[w], shared[kWaves + w]};
  __syncthreads();
  return sum;
}

// The border after digit `pass`, from all chunks' histograms; the first workgroup leaves it for the next launch.  own, before: the
// counts of the thread's digits in this chunk and in those before it.
__device__ __forceinline__ void border_after(const Scratch &s, int pass, int chunks, int chunk, uint32_t need0, int tid, uint32_t *shared, uint32_t &prefix,
                                             uint32_t &need, u32x2 &own, u32x2 &before) {
  prefix = pass ? s.border[2 * (pass - 1)] : 0u;
  need = pass ? s.border[2 * (pass - 1) + 1] : need0;
  const u32x2 *hist = reinterpret_cast<const u32x2 *>(s.hist + (size_t)pass * chunks * kBins) + tid;
  u32x2 sum = {0, 0};
  own = before = u32x2{0, 0};
  for (int x0 = 0; x0 < chunks; x0 += 8) {        // (eight loads on their way at a time)
    u32x2 n[8];
#pragma unroll
    for (int x = 0; x < 8; x++) n[x] = hist[(size_t)min(x0 + x, chunks - 1) * (kBins / 2)];
#pragma unroll
    for (int x = 0; x < 8; x++) {
      if (x0 + x < chunks) sum += n[x];
      if (x0 + x < chunk) before += n[x];
      if (x0 + x == chunk) own = n[x];
    }
  }
  const Choice c = choose(sum[0], sum[1], need, tid, shared);
  prefix |= c.digit << kShift[pass];
  need = c.need;
  if (chunk == 0 && tid == 0) {
    s.border[2 * pass] = prefix;
    s.border[2 * pass + 1] = need;
  }
}

template <int PASS>
__global__ __launch_bounds__(kSelect) void kv_digit_kernel(SelectArgs a, uint32_t *ws) {
  const int chunk = blockIdx.x, chunks = gridDim.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int length = kv_length(a.lengths, b, a.capacity);
  const uint32_t need0 = (uint32_t)(a.keep - a.n_global - a.n_recent);
  if (length <= a.keep || need0 == 0) return;
  const int64_t row = (int64_t)b * a.heads_kv + h;
  const Scratch s = scratch_of(ws, row, chunks);
  const float *w = a.weights + row * a.capacity;
  __shared__ __attribute__((aligned(8))) uint32_t hist[kBins];
  __shared__ uint32_t shared[2 * kWaves + 3];
  const int first = a.n_global, last = length - a.n_recent, lo = chunk * a.pieces * kPiece, hi = min(lo + a.pieces * kPiece, length);
  uint32_t key[kChunkKeys];
  load_keys(w, lo, length, wave, lane, key);
  *reinterpret_cast<u32x2 *>(&hist[2 * tid]) = u32x2{0, 0};
  uint32_t prefix = 0;
  if (PASS > 0) {
    uint32_t need;
    u32x2 own, before;
    border_after(s, PASS - 1, chunks, chunk, need0, tid, shared, prefix, need, own, before);
    const uint32_t digit = digit_of(prefix, PASS - 1), d0 = 2u * (uint32_t)tid;
    const u32x2 mine = group_sum(u32x2{(d0 > digit ? own[0] : 0u) + (d0 + 1 > digit ? own[1] : 0u), 0u}, tid, shared);
    if (tid == 0) s.above[(PASS - 1) * chunks + chunk] = mine[0];
  }
  __syncthreads();
  const uint32_t mask = PASS == 0 ? 0u : ~0u << kShift[PASS > 0 ? PASS - 1 : 0];
  for (int base = lo; base < hi; base += kPiece) {
    if (base > lo) load_keys(w, base, length, wave, lane, key);
    const int n0 = base + wave * 64 * kChunkKeys + lane;
#pragma unroll
    for (int i = 0; i < kChunkKeys; i++)
      if (n0 + 64 * i >= first && n0 + 64 * i < last && (key[i] & mask) == prefix) atomicAdd(&hist[digit_of(key[i], PASS)], 1u);
  }
  __syncthreads();
  *reinterpret_cast<u32x2 *>(s.hist + ((size_t)PASS * chunks + chunk) * kBins + 2 * tid) = *reinterpret_cast<const u32x2 *>(&hist[2 * tid]);
}

__global__ __launch_bounds__(kSelect) void kv_place_kernel(SelectArgs a, uint32_t *ws) {
  const int chunk = blockIdx.x, chunks = gridDim.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int length = kv_length(a.lengths, b, a.capacity);
  const int64_t row = (int64_t)b * a.heads_kv + h;
  if (h == 0 && chunk == 0 && tid == 0) a.lengths_out[b] = min(length, a.keep);
  if (all_stay(a, row, length, chunk, chunks, tid)) return;
  const float *w = a.weights + row * a.capacity;
  const uint32_t need0 = (uint32_t)(a.keep - a.n_global - a.n_recent);
  const bool ranked = need0 > 0;
  __shared__ uint32_t shared[2 * kWaves + 3];
  const int first = a.n_global, last = length - a.n_recent, lo = chunk * a.pieces * kPiece, hi = min(lo + a.pieces * kPiece, length);
  if (lo >= hi) return;
  uint32_t prefix = 0, need = 0, placed = 0, equal = 0;
  uint32_t key[kChunkKeys];
  load_keys(w, lo, length, wave, lane, key);
  if (ranked) {
    const Scratch s = scratch_of(ws, row, chunks);
    u32x2 own, before;
    border_after(s, 2, chunks, chunk, need0, tid, shared, prefix, need, own, before);
    // in the chunks before: keys above the border, and equal to it
    const uint32_t digit = digit_of(prefix, 2), d0 = 2u * (uint32_t)tid;
    placed = (d0 > digit ? before[0] : 0u) + (d0 + 1 > digit ? before[1] : 0u);
    equal = (d0 == digit ? before[0] : 0u) + (d0 + 1 == digit ? before[1] : 0u);
    for (int x = tid; x < chunk; x += kSelect) placed += s.above[x] + s.above[chunks + x];
    const u32x2 sums = group_sum(u32x2{placed, equal}, tid, shared);
    placed = sums[0];
    equal = sums[1];
  }
  placed += (uint32_t)(min(lo, first) + max(0, min(lo, length) - max(last, 0)));      // and those that stay in any case
  // (place() counts tokens with the border's key from `equal` on; those of them before that stay are the first `need`)
  for (int base = lo; base < hi; base += kPiece) {
    if (base > lo) {
      __syncthreads();
      load_keys(w, base, length, wave, lane, key);
    }
    place<kChunkKeys>(a, row, w, key, base, length, prefix, need, ranked, placed, equal, base + kPiece < hi, tid, shared);
  }
}

// ---- the move

// One workgroup per block of the new cache, head, and keys or values; a thread has up to PIECES times 16 codes.
template <int CODE, int PIECES, int THREADS>
__global__ __launch_bounds__(THREADS) void kv_move_kernel(ns_kv_cache from, ns_kv_cache to, const int32_t *lengths, const int32_t *kept, int keep, int first) {
  const int b = blockIdx.z, h = blockIdx.y >> 1, value = blockIdx.y & 1, tid = threadIdx.x, block = first + (int)blockIdx.x;
  const int lo = block * to.block, here = min(to.block, min(kv_length(lengths, b, from.capacity), keep) - lo);
  if (here <= 0) return;
  const int64_t row = (int64_t)b * to.heads_kv + h;
  const int pieces = to.head_dim / 16, token = tid / pieces, step = THREADS / pieces;      // pieces of a token; tokens between a thread's
  const int d = tid % pieces * 16, lblock = 31 - __clz(from.block);
  const uint8_t *src = static_cast<const uint8_t *>(value ? from.v : from.k) + b * from.stride_b + h * from.stride_h + d;
  const float *src_scale = (value ? from.v_scale : from.k_scale) + row * (from.capacity / from.block);
  uint8_t *dst = static_cast<uint8_t *>(value ? to.v : to.k) + b * to.stride_b + h * to.stride_h + d;
  kept += row * keep + lo;
  u32x4 codes[PIECES];
  float scale[PIECES], most = 0.f;
#pragma unroll
  for (int i = 0; i < PIECES; i++) {
    const int t = token + i * step;
    codes[i] = u32x4{0, 0, 0, 0};
    scale[i] = 0.f;
    if (t < here) {
      const int n = kept[t];
      codes[i] = *reinterpret_cast<const u32x4 *>(src + n * from.stride_t);
      scale[i] = src_scale[n >> lblock];
    }
  }
  bool nan = false;
#pragma unroll
  for (int i = 0; i < PIECES; i++) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const f32x4 c = kv_decode4<CODE>(codes[i][j]);
      top = fmaxf(fmaxf(top, fmaxf(__builtin_fabsf(c[0]), __builtin_fabsf(c[1]))), fmaxf(__builtin_fabsf(c[2]), __builtin_fabsf(c[3])));
    }
    nan |= kv_is_nan(scale[i]);
    const float x = top * scale[i], off = __builtin_fmaf(top, scale[i], -x);
    most = fmaxf(most, off > 0.f ? __uint_as_float(__float_as_uint(x) + 1) : x);     // (rounded up: not to the limit of a scale below)
  }
  __shared__ float largest[THREADS / 64];
  if (nan) most = INFINITY;
  most = wave_max(most);
  if (tid % 64 == 0) largest[tid / 64] = most;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < THREADS / 64; x++) most = fmaxf(most, largest[x]);
  const float s = kv_scale_for<CODE>(__float_as_uint(most));
#pragma unroll
  for (int i = 0; i < PIECES; i++) {
    const int t = token + i * step;
    if (t >= to.block) continue;
    u32x4 w = codes[i];
    // (most tokens come from blocks of the same scale: their codes stay as they are)
    if (scale[i] != s && t < here) {
      const float ratio = scale[i] / s;               // (exact: s is a power of two)
#pragma unroll
      for (int j = 0; j < 4; j++) w[j] = kv_is_nan(s) ? 0u : kv_recode4<CODE>(w[j], ratio);
    }
    *reinterpret_cast<u32x4 *>(dst + (int64_t)(lo + t) * to.stride_t) = w;
  }
  if (tid == 0) (value ? to.v_scale : to.k_scale)[row * (to.capacity / to.block) + block] = s;
}

int pieces_of(int capacity) { return ((capacity + kPiece - 1) / kPiece + kMostChunks - 1) / kMostChunks; }
int chunks_of(int capacity) { return ((capacity + kPiece - 1) / kPiece + pieces_of(capacity) - 1) / pieces_of(capacity); }

template <int CODE> void move(hipStream_t s, const ns_kv_cache &from, const ns_kv_cache &to, const int32_t *lengths, const int32_t *kept, int keep) {
  constexpr int kMost = 1 << 22;                      // blocks of one launch: a grid's threads along an axis are counted in 32 bits
  auto go = [&](auto kernel, int threads) {
    for (int first = 0, blocks = (keep + to.block - 1) / to.block; first < blocks; first += kMost)
      hipLaunchKernelGGL(kernel, dim3((unsigned)min(blocks - first, kMost), (unsigned)to.heads_kv * 2, (unsigned)to.batch), dim3(threads), 0, s, from, to, lengths,
                         kept, keep, first);
  };
  switch (to.block * to.head_dim / 4096) {
    case 0: case 1: return go(kv_move_kernel<CODE, 1, 256>, 256);
    case 2: return go(kv_move_kernel<CODE, 2, 256>, 256);
    case 4: return go(kv_move_kernel<CODE, 4, 256>, 256);
    default: return go(kv_move_kernel<CODE, 4, 512>, 512);
  }
}

}  // namespace

size_t kv_evict_workspace_bytes(const ns_kv_cache &from, int) {
  return from.capacity <= kHeld ? 0 : align_up((size_t)from.batch * from.heads_kv * scratch_words(chunks_of(from.capacity)) * 4, 256);
}

ns_status launch_kv_evict(const ns_kv_cache &from, const ns_kv_cache &to, const float *weights, const int32_t *lengths, int keep,
                          int n_global, int n_recent, int32_t *kept, float *w_out, int32_t *lengths_out, void *ws, hipStream_t s) {
  const SelectArgs a{weights, lengths, from.capacity, keep, n_global, n_recent, from.heads_kv, to.capacity, pieces_of(from.capacity), kept, w_out, lengths_out};
  ns_status st;
  if (from.capacity <= kHeld) {
    const dim3 grid((unsigned)from.heads_kv, (unsigned)from.batch);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kSelect), 0, s, a); };
    from.capacity <= 2 * kSelect ? go(kv_select_kernel<2>) : from.capacity <= 8 * kSelect ? go(kv_select_kernel<8>) : go(kv_select_kernel<16>);
    st = check_launch("kv_select_kernel");
  } else {
    const dim3 grid((unsigned)chunks_of(from.capacity), (unsigned)from.heads_kv, (unsigned)from.batch);
    uint32_t *p = static_cast<uint32_t *>(ws);
    hipLaunchKernelGGL(kv_digit_kernel<0>, grid, dim3(kSelect), 0, s, a, p);
    hipLaunchKernelGGL(kv_digit_kernel<1>, grid, dim3(kSelect), 0, s, a, p);
    hipLaunchKernelGGL(kv_digit_kernel<2>, grid, dim3(kSelect), 0, s, a, p);
    hipLaunchKernelGGL(kv_place_kernel, grid, dim3(kSelect), 0, s, a, p);
    st = check_launch("kv_digit_kernel / kv_place_kernel");
  }
  if (st != NS_OK) return st;
  to.code == NS_CODE_I8 ? move<NS_CODE_I8>(s, from, to, lengths, kept, keep) : move<NS_CODE_E4M3>(s, from, to, lengths, kept, keep);
  return check_launch("kv_move_kernel");
}

}  // namespace ns
