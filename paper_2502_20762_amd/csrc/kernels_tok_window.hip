// Softmax attention with a sliding window and sinks over whole sequences:
//   o_i = sum_j p_ij v_j over the tokens j that token i sees, p = softmax(scale q_i . k_j).
#include <algorithm>

#include "tok_attend.hpp"

namespace nc {
namespace {

// One wave for a token and head: a lane scores a key at a time, a running maximum
// and sum join the rounds of 64, then each lane sums two columns of v.
template <class E>
__global__ __launch_bounds__(256) void k_tok_window(WindowArgs a, int64_t items) {
  typedef typename E::T T;
  const ncodec_window_shape& s = a.s;
  const int lane = threadIdx.x & 63;
  const int D = s.head_dim, V = s.value_dim;
  for (int64_t it = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); it < items; it += (int64_t)gridDim.x * 4) {
    const int h = (int)(it % s.heads);
    const int64_t row = it / s.heads, b = row / s.tokens, i = row % s.tokens;
    const int hk = h / (s.heads / s.kv_heads);
    const int64_t len = a.lengths ? min(max((int64_t)a.lengths[b], (int64_t)0), s.tokens) : s.tokens;
    const T* q = (const T*)a.q + b * s.q_batch_stride + i * s.q_token_stride + h * s.q_head_stride;
    const T* k = (const T*)a.k + b * s.k_batch_stride + hk * s.k_head_stride;
    const T* v = (const T*)a.v + b * s.v_batch_stride + hk * s.v_head_stride;
    T* o = (T*)a.o + b * s.o_batch_stride + i * s.o_token_stride + h * s.o_head_stride;
    float m = -__builtin_huge_valf(), l = 0.f, acc[2] = {};
    if (i < len) {
      const Seen seen = seen_by((int)i, s.window, s.sinks);
      for (int x0 = 0; x0 < seen.count; x0 += 64) {
        const bool in = x0 + lane < seen.count;
        const int64_t j = in ? seen.at(x0 + lane) : 0;
        float z = 0.f;
        for (int d = 0; d < D; ++d) z = fmaf((float)q[d], (float)k[j * s.k_token_stride + d], z);
        z = in ? z * s.scale * 1.44269504088896341f : -__builtin_huge_valf();
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
        for (int x = 0; x < min(64, seen.count - x0); ++x) {
          const float px = __shfl(p, x, 64);
          const T* vr = v + (int64_t)seen.at(x0 + x) * s.v_token_stride;
          for (int y = 0; y < 2; ++y)
            if (lane + 64 * y < V) acc[y] = fmaf(px, (float)vr[lane + 64 * y], acc[y]);
        }
      }
    }
    for (int y = 0; y < 2; ++y)
      if (lane + 64 * y < V) o[lane + 64 * y] = (T)(i < len ? acc[y] / l : 0.f);
  }
}

}  // namespace

hipError_t launch_window_attention(const WindowArgs& a, hipStream_t st) {
  const int64_t items = a.s.batch * a.s.tokens * a.s.heads;
  const dim3 grid((unsigned)std::min<int64_t>((items + 3) / 4, 1 << 20));
  if (a.s.dtype == NCODEC_DTYPE_FP16)
    launch(k_tok_window<F16>, grid, dim3(256), st, a, items);
  else
    launch(k_tok_window<BF16>, grid, dim3(256), st, a, items);
  return hipGetLastError();
}

}  // namespace nc
