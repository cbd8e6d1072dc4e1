// RMS norm of every query and key head and the rotation by the token's
// position, in one pass over q and k.
#include "tokens.hpp"

namespace nc {
namespace {

constexpr int kMaxPairs = 128;

// cos and sin of pos * freq radians.  The angle is counted in turns in 64
// bits, where a 31-bit position times a 24-bit frequency is exact up to the
// factor 1 / (2 pi), and only its fraction goes to 32 bits (v_sin_f32 and
// v_cos_f32 take turns), so a late token is turned as exactly as the first.
__device__ __forceinline__ float2 turn(int pos, float freq) {
  const double t = (double)pos * ((double)freq * 0.15915494309189533577);
  const float f = (float)(t - __builtin_floor(t));
  return make_float2(__builtin_amdgcn_cosf(f), __builtin_amdgcn_sinf(f));
}

__device__ __forceinline__ float wave_sum_f(float v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// One workgroup per token, one wave per head.
template <class E>
__global__ __launch_bounds__(256) void k_tok_rope(QkArgs a) {
  typedef typename E::T T;
  __shared__ float2 cs[kMaxPairs];
  const ncodec_qk_shape& s = a.s;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int P = s.section[0] + s.section[1] + s.section[2], D = s.head_dim;
  const int64_t t = blockIdx.x;
  for (int p = threadIdx.x; p < P; p += 256) {
    const int axis = p < s.section[0] ? 0 : p < s.section[0] + s.section[1] ? 1 : 2;
    cs[p] = turn(a.pos[t * s.axes + axis], a.freq[p]);
  }
  __syncthreads();
  for (int h = wave; h < s.q_heads + s.k_heads; h += 4) {
    const bool is_q = h < s.q_heads;
    const int hh = is_q ? h : h - s.q_heads;
    const T* x = is_q ? (const T*)a.q + t * s.q_token_stride + hh * s.q_head_stride
                      : (const T*)a.k + t * s.k_token_stride + hh * s.k_head_stride;
    T* y = is_q ? (T*)a.qo + t * s.qo_token_stride + hh * s.qo_head_stride
                : (T*)a.ko + t * s.ko_token_stride + hh * s.ko_head_stride;
    const T* w = (const T*)(is_q ? a.wq : a.wk);
    float v[4], o[4], sq = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = lane + 64 * i;
      v[i] = d < D ? (float)x[d] : 0.f;
      sq = fmaf(v[i], v[i], sq);
    }
    float inv = 1.f;
    if (s.norm) inv = 1.f / sqrtf(wave_sum_f(sq) / D + s.eps);
    // each pair's other half, read before anything is written
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = lane + 64 * i;
      if (d >= D) continue;
      float e = v[i] * inv * (s.norm && w ? (float)w[d] : 1.f);
      if (d < 2 * P) {
        const int p = s.interleaved ? d >> 1 : d < P ? d : d - P;
        const bool second = s.interleaved ? d & 1 : d >= P;
        const int od = s.interleaved ? d ^ 1 : second ? d - P : d + P;
        const float other = (float)x[od] * inv * (s.norm && w ? (float)w[od] : 1.f);
        const float2 c = cs[p];
        e = second ? fmaf(other, c.y, e * c.x) : fmaf(-other, c.y, e * c.x);
      }
      o[i] = e;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < D) y[lane + 64 * i] = (T)o[i];
  }
}

}  // namespace

hipError_t launch_qk_norm_rope(const QkArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.s.tokens);
  if (a.s.dtype == NCODEC_DTYPE_FP16)
    launch(k_tok_rope<F16>, grid, dim3(256), st, a);
  else
    launch(k_tok_rope<BF16>, grid, dim3(256), st, a);
  return hipGetLastError();
}

}  // namespace nc
