// Softmax attention of one new token of each sequence over a paged cache.
#include <algorithm>

#include "tok_attend.hpp"

namespace nc {
namespace {

// One wave for a sequence and head; its scores go to the workspace where weights are summed.
template <class E>
__global__ __launch_bounds__(64) void k_tok_paged(PagedArgs a) {
  typedef typename E::T T;
  const ncodec_cache_shape& c = a.c;
  const ncodec_paged_shape& s = a.s;
  const int lane = threadIdx.x, D = c.head_dim, V = c.value_dim;
  const int h = (int)(blockIdx.x % s.heads), hk = h / (s.heads / c.kv_heads);
  const int64_t b = blockIdx.x / s.heads, cap = s.columns * c.page_size;
  const int n = (int)min(max((int64_t)a.lengths[b], (int64_t)0), cap), shift = __ffs(c.page_size) - 1;
  const int32_t* table = a.table + b * s.table_stride;
  const T* q = (const T*)a.q + b * s.q_batch_stride + h * s.q_head_stride;
  T* o = (T*)a.o + b * s.o_batch_stride + h * s.o_head_stride;
  float* z_of = a.mass ? (float*)a.ws + 2 * s.batch * s.heads + blockIdx.x * cap : nullptr;
  float m = -__builtin_huge_valf(), l = 0.f, acc[2] = {};
  bool any = false;
  const Seen seen = seen_by(n - 1, s.window, s.sinks);
  for (int x0 = 0; x0 < seen.count; x0 += 64) {
    const int j = seen.at(min(x0 + lane, seen.count - 1));
    const int32_t page = table[j >> shift];
    const bool in = x0 + lane < seen.count && page >= 0 && page < c.pages;
    const int64_t krow = (in ? page * c.k_page_stride + (j & (c.page_size - 1)) * c.k_token_stride : 0) + hk * c.k_head_stride;
    const int64_t vrow = (in ? page * c.v_page_stride + (j & (c.page_size - 1)) * c.v_token_stride : 0) + hk * c.v_head_stride;
    float z = 0.f;
    if (in)
      for (int d = 0; d < D; ++d) z = fmaf((float)q[d], (float)((const T*)a.k)[krow + d], z);
    z = in ? z * s.scale * 1.44269504088896341f : -__builtin_huge_valf();
    if (z_of && x0 + lane < seen.count) z_of[j] = z;
    float top = z;
    for (int w = 32; w; w >>= 1) top = __builtin_elementwise_maximum(top, __shfl_xor(top, w, 64));
    const float m1 = __builtin_elementwise_maximum(m, top);
    const float base = m1 == -__builtin_huge_valf() ? 0.f : m1;
    const float fade = exp2f(m - base), p = exp2f(z - base - kBelow);
    float sum = p;
    for (int w = 32; w; w >>= 1) sum += __shfl_xor(sum, w, 64);
    l = l * fade + sum;
    m = m1;
    acc[0] *= fade;
    acc[1] *= fade;
    any |= __any(in);
    for (int x = 0; x < 64; ++x) {
      if (!__shfl((int)in, x, 64)) continue;
      const float px = __shfl(p, x, 64);
      const T* vr = (const T*)a.v + __shfl(vrow, x, 64);
      for (int y = 0; y < 2; ++y)
        if (lane + 64 * y < V) acc[y] = fmaf(px, (float)vr[lane + 64 * y], acc[y]);
    }
  }
  for (int y = 0; y < 2; ++y)
    if (lane + 64 * y < V) o[lane + 64 * y] = (T)(any ? acc[y] / l : 0.f);
  if (z_of && lane == 0) {
    ((float*)a.ws)[2 * blockIdx.x] = m;
    ((float*)a.ws)[2 * blockIdx.x + 1] = l;
  }
}

// mass += the weights of a key head's query heads
__global__ __launch_bounds__(256) void k_tok_paged_mass(PagedArgs a) {
  const ncodec_cache_shape& c = a.c;
  const ncodec_paged_shape& s = a.s;
  const int64_t cap = s.columns * c.page_size, b = blockIdx.x / c.kv_heads;
  const int hk = (int)(blockIdx.x % c.kv_heads), group = s.heads / c.kv_heads, shift = __ffs(c.page_size) - 1;
  const int n = (int)min(max((int64_t)a.lengths[b], (int64_t)0), cap);
  const Seen seen = seen_by(n - 1, s.window, s.sinks);
  for (int x = threadIdx.x; x < seen.count; x += 256) {
    const int j = seen.at(x);
    const int32_t page = a.table[b * s.table_stride + (j >> shift)];
    if (page < 0 || page >= c.pages) continue;
    float w = 0.f;
    for (int g = 0; g < group; ++g) {
      const int64_t bh = b * s.heads + hk * group + g;
      const float m = ((const float*)a.ws)[2 * bh], l = ((const float*)a.ws)[2 * bh + 1];
      w += exp2f(((const float*)a.ws)[2 * s.batch * s.heads + bh * cap + j] - m - kBelow) / l;
    }
    a.mass[blockIdx.x * cap + j] += w;
  }
}

}  // namespace

size_t paged_workspace_bytes(const ncodec_cache_shape& c, const ncodec_paged_shape& s, bool mass) {
  return mass ? (size_t)(s.batch * s.heads) * (2 + s.columns * c.page_size) * 4 : 0;
}

hipError_t launch_paged_attention(const PagedArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.s.batch * a.s.heads));
  if (a.c.dtype == NCODEC_DTYPE_FP16)
    launch(k_tok_paged<F16>, grid, dim3(64), st, a);
  else
    launch(k_tok_paged<BF16>, grid, dim3(64), st, a);
  if (a.mass) launch(k_tok_paged_mass, dim3((unsigned)(a.s.batch * a.c.kv_heads)), dim3(256), st, a);
  return hipGetLastError();
}

}  // namespace nc
