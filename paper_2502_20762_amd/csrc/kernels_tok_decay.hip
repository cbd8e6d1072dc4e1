// Linear attention with a decay for each head:
//   S_t = lambda S_{t-1} + k_t v_t^T,  o_t = scale q_t S_t.
#include "tokens.hpp"

namespace nc {
namespace {

// lambda^n = exp2(n * this).  Positive decays count as 0, -inf becomes a
// number so that lambda^0 is 1 (0 * -inf is not a number).
__device__ __forceinline__ float log2_decay(float log_decay) {
  return fmaxf(fminf(log_decay, 0.f), -1e30f) * 1.44269504088896341f;
}

// The recurrence itself, token by token.  A workgroup holds 64 columns of one
// sequence's and head's state in registers: thread (g, c) the rows g + 16 r and
// the columns 4 c .. 4 c + 3.
template <class E, int R>
__global__ __launch_bounds__(256) void k_tok_decay_recur(DecayArgs a) {
  typedef typename E::T T;
  __shared__ float qs[16 * R], ks[16 * R], part[4][64];
  const ncodec_decay_shape& s = a.s;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = lane & 15, g = wave * 4 + (lane >> 4);
  const int64_t b = blockIdx.x / s.heads, h = blockIdx.x % s.heads, hk = h / (s.heads / s.kv_heads);
  const int D = s.head_dim, V = s.value_dim, v0 = blockIdx.y * 64 + 4 * c;
  const float lam = exp2f(log2_decay(a.log_decay[h]));
  const int64_t len = a.lengths ? min(max((int64_t)a.lengths[b], (int64_t)0), s.tokens) : s.tokens;
  const T* q = (const T*)a.q + b * s.q_batch_stride + h * s.q_head_stride;
  const T* k = (const T*)a.k + b * s.k_batch_stride + hk * s.k_head_stride;
  const T* v = (const T*)a.v + b * s.v_batch_stride + hk * s.v_head_stride;
  T* o = (T*)a.o + b * s.o_batch_stride + h * s.o_head_stride;
  const int64_t sbase = (b * s.heads + h) * (int64_t)D * V;
  float S[R][4];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = g + 16 * r;
      S[r][j] = a.state_in && d < D && v0 + j < V ? a.state_in[sbase + d * V + v0 + j] : 0.f;
    }
  for (int64_t t = 0; t < len; ++t) {
    __syncthreads();
    if (threadIdx.x < 16 * R) {
      const int d = threadIdx.x;
      qs[d] = d < D ? (float)q[t * s.q_token_stride + d] * s.scale : 0.f;
      ks[d] = d < D ? (float)k[t * s.k_token_stride + d] : 0.f;
    }
    float vv[4], ov[4] = {};
#pragma unroll
    for (int j = 0; j < 4; ++j) vv[j] = v0 + j < V ? (float)v[t * s.v_token_stride + v0 + j] : 0.f;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float kd = ks[g + 16 * r], qd = qs[g + 16 * r];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        S[r][j] = fmaf(kd, vv[j], lam * S[r][j]);
        ov[j] = fmaf(qd, S[r][j], ov[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      ov[j] += __shfl_xor(ov[j], 16, 64);
      ov[j] += __shfl_xor(ov[j], 32, 64);
      if (lane < 16) part[wave][4 * c + j] = ov[j];
    }
    __syncthreads();
    const int col = blockIdx.y * 64 + threadIdx.x;
    if (threadIdx.x < 64 && col < V) {
      const int i = threadIdx.x;
      o[t * s.o_token_stride + col] = (T)(part[0][i] + part[1][i] + part[2][i] + part[3][i]);
    }
  }
  // outputs past the sequence's end
  for (int64_t i = threadIdx.x; i < (s.tokens - len) * 64; i += 256) {
    const int col = blockIdx.y * 64 + (int)(i % 64);
    if (col < V) o[(len + i / 64) * s.o_token_stride + col] = (T)0.f;
  }
  if (a.state_out) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = g + 16 * r;
        if (d < D && v0 + j < V) a.state_out[sbase + d * V + v0 + j] = S[r][j];
      }
  }
}

template <class E>
hipError_t recur(const DecayArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.s.batch * a.s.heads), (unsigned)((a.s.value_dim + 63) / 64));
  if (a.s.head_dim <= 32)
    launch(k_tok_decay_recur<E, 2>, grid, dim3(256), st, a);
  else if (a.s.head_dim <= 64)
    launch(k_tok_decay_recur<E, 4>, grid, dim3(256), st, a);
  else
    launch(k_tok_decay_recur<E, 8>, grid, dim3(256), st, a);
  return hipGetLastError();
}

}  // namespace

size_t decay_workspace_bytes(const ncodec_decay_shape&) { return 0; }

hipError_t launch_decay_attention(const DecayArgs& a, hipStream_t st) {
  return a.s.dtype == NCODEC_DTYPE_FP16 ? recur<F16>(a, st) : recur<BF16>(a, st);
}

}  // namespace nc
