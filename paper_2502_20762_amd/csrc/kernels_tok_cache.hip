// The upkeep of a paged cache: new tokens into its pages, and eviction by
// accumulated attention weight.
#include <algorithm>

#include "tokens.hpp"

namespace nc {
namespace {

__device__ __forceinline__ void copy_row(uint16_t* to, const uint16_t* from, int n, int lane) {
  for (int d = lane; d < n; d += 64) to[d] = from[d];
}

// One wave a row.
__global__ __launch_bounds__(256) void k_tok_append(AppendArgs a, int64_t items) {
  const ncodec_cache_shape& c = a.c;
  const ncodec_append_shape& s = a.s;
  const int lane = threadIdx.x & 63, shift = __ffs(c.page_size) - 1;
  const int64_t cap = s.columns * c.page_size;
  for (int64_t it = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); it < items; it += (int64_t)gridDim.x * 4) {
    const int h = (int)(it % c.kv_heads);
    const int64_t row = it / c.kv_heads, b = row / s.tokens, i = row % s.tokens;
    const int64_t count = a.counts ? min(max((int64_t)a.counts[b], (int64_t)0), s.tokens) : s.tokens;
    const int64_t j = a.starts[b] + i;
    if (i >= count || j < 0 || j >= cap) continue;
    const int32_t page = a.table[b * s.table_stride + (j >> shift)];
    if (page < 0 || page >= c.pages) continue;
    const int64_t r = j & (c.page_size - 1);
    copy_row((uint16_t*)a.k_cache + page * c.k_page_stride + r * c.k_token_stride + h * c.k_head_stride,
             (const uint16_t*)a.k + b * s.k_batch_stride + i * s.k_token_stride + h * s.k_head_stride, c.head_dim, lane);
    copy_row((uint16_t*)a.v_cache + page * c.v_page_stride + r * c.v_token_stride + h * c.v_head_stride,
             (const uint16_t*)a.v + b * s.v_batch_stride + i * s.v_token_stride + h * s.v_head_stride, c.value_dim, lane);
    if (a.mass && lane == 0) a.mass[(b * c.kv_heads + h) * cap + j] = 0.f;
  }
}

// A key whose order is that of the weights, -0 as 0 and a NaN above all.
__device__ __forceinline__ uint32_t weight_key(float f) {
  if (f != f) return 0xffffffffu;
  const uint32_t u = __float_as_uint(f + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One thread for a sequence and head finds the smallest key that is kept, bit by
// bit, and then the list.
__global__ __launch_bounds__(64) void k_tok_evict_pick(EvictArgs a) {
  const ncodec_cache_shape& c = a.c;
  const ncodec_evict_shape& s = a.s;
  const int64_t cap = s.columns * c.page_size, new_cap = s.new_columns * c.page_size;
  const int64_t b = blockIdx.x / c.kv_heads;
  const int lane = threadIdx.x;
  const int n = (int)min(max((int64_t)a.lengths[b], (int64_t)0), cap);
  const float* mass = a.mass + blockIdx.x * cap;
  float* new_mass = a.new_mass + blockIdx.x * new_cap;
  int32_t* kept = a.kept + blockIdx.x * s.keep;
  const int m = (int)min((int64_t)n, s.keep);
  const int lo = (int)min(s.sinks, (int64_t)n), hi = (int)max((int64_t)lo, n - s.recent);
  const int want = m - lo - (n - hi);  // of the positions lo .. hi - 1
  uint32_t key = 0;                    // the want-th largest
  for (int bit = 31; bit >= 0; --bit) {
    int count = 0;
    for (int j = lo + lane; j < hi; j += 64) count += weight_key(mass[j]) >= (key | 1u << bit);
    for (int w = 32; w; w >>= 1) count += __shfl_xor(count, w, 64);
    if (count >= want) key |= 1u << bit;
  }
  int above = 0;
  for (int j = lo + lane; j < hi; j += 64) above += weight_key(mass[j]) > key;
  for (int w = 32; w; w >>= 1) above += __shfl_xor(above, w, 64);
  int equal = want - above, at = 0;  // so many of the equals, the earliest
  for (int j0 = 0; j0 < n; j0 += 64) {
    const int j = j0 + lane;
    const uint32_t u = j < n ? weight_key(mass[j]) : 0;
    const bool mid = j >= lo && j < hi;
    const uint64_t ties = __ballot(mid && u == key);
    const int before = (int)__popcll(ties & ((1ull << lane) - 1));
    const bool keep = j < n && (!mid || u > key || (u == key && before < equal));
    const uint64_t all = __ballot(keep);
    if (keep) {
      const int to = at + (int)__popcll(all & ((1ull << lane) - 1));
      kept[to] = j;
      new_mass[to] = mass[j];
    }
    equal = max(0, equal - (int)__popcll(ties));
    at += (int)__popcll(all);
  }
  for (int64_t x = m + lane; x < s.keep; x += 64) kept[x] = -1;
  for (int64_t x = m + lane; x < new_cap; x += 64) new_mass[x] = 0.f;
  if (lane == 0 && blockIdx.x % c.kv_heads == 0) a.new_lengths[b] = m;
}

__global__ __launch_bounds__(256) void k_tok_evict_move(EvictArgs a, int64_t items) {
  const ncodec_cache_shape& c = a.c;
  const ncodec_evict_shape& s = a.s;
  const int lane = threadIdx.x & 63, shift = __ffs(c.page_size) - 1;
  for (int64_t it = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); it < items; it += (int64_t)gridDim.x * 4) {
    const int64_t bh = it / s.keep, b = bh / c.kv_heads, x = it % s.keep;
    const int h = (int)(bh % c.kv_heads);
    const int32_t j = a.kept[it];
    if (j < 0) continue;
    const int32_t from = a.table[b * s.table_stride + (j >> shift)], to = a.new_table[b * s.new_table_stride + (x >> shift)];
    if (from < 0 || from >= c.pages || to < 0 || to >= c.pages) continue;
    const int64_t r = j & (c.page_size - 1), t = x & (c.page_size - 1);
    uint16_t *k = (uint16_t*)a.k_cache + h * c.k_head_stride, *v = (uint16_t*)a.v_cache + h * c.v_head_stride;
    copy_row(k + to * c.k_page_stride + t * c.k_token_stride, k + from * c.k_page_stride + r * c.k_token_stride, c.head_dim, lane);
    copy_row(v + to * c.v_page_stride + t * c.v_token_stride, v + from * c.v_page_stride + r * c.v_token_stride, c.value_dim, lane);
  }
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t st) {
  const int64_t items = a.s.batch * a.s.tokens * a.c.kv_heads;
  launch(k_tok_append, dim3((unsigned)std::min<int64_t>((items + 3) / 4, 1 << 20)), dim3(256), st, a, items);
  return hipGetLastError();
}

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t st) {
  const int64_t items = a.s.batch * a.c.kv_heads * a.s.keep;
  launch(k_tok_evict_pick, dim3((unsigned)(a.s.batch * a.c.kv_heads)), dim3(64), st, a);
  launch(k_tok_evict_move, dim3((unsigned)std::min<int64_t>((items + 3) / 4, 1 << 20)), dim3(256), st, a, items);
  return hipGetLastError();
}

}  // namespace nc
