// Matrix product with bias, activation, gate and residual in its epilogue:
//   y = act(x W^T + b) [* (x W2^T + b2)] + r.
// Computed transposed like the codec's pointwise kernels: the weight rows are
// the MFMA A operand, the tokens are the columns, and a lane of the
// accumulator holds one token and four consecutive features at a time.
#include "tokens.hpp"

namespace nc {
namespace {

// Activations in fp32.  The logistic is 1 / (1 + exp(-v)) with the hardware
// exponential and reciprocal (relative error below 2^-21, far below the
// rounding of y); v Phi(v) goes through erfc, whose fit is relative, so the
// tail keeps its digits.
template <int ACT>
__device__ __forceinline__ float activate(float v) {
  if (ACT == NCODEC_ACT_LRELU) return v >= 0.f ? v : 0.1f * v;
  if (ACT == NCODEC_ACT_WSILU) return v * __builtin_amdgcn_rcpf(1.f + __expf(-4.f * v));
  if (ACT == NCODEC_ACT_SILU) return v * __builtin_amdgcn_rcpf(1.f + __expf(-v));
  if (ACT == NCODEC_ACT_GELU) {
    const float e = 0.5f * erfc_pos(0.70710678118654752f * fabsf(v));
    return v * (v >= 0.f ? 1.f - e : e);
  }
  return v;
}

constexpr int kTile = 64, kStep = 64, kPitch = kStep + 8;

// 64 tokens x 64 features a workgroup, four waves of 32 x 32.
template <class E, int ACT, bool GATED>
__global__ __launch_bounds__(256) void k_tok_linear(LinearArgs a) {
  typedef typename E::T T;
  typedef typename E::V8 V8;
  __shared__ __align__(16) T xs[kTile * kPitch];
  __shared__ __align__(16) T wsm[(GATED ? 2 : 1) * kTile * kPitch];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tm = (wave & 1) * 32, tn = (wave >> 1) * 32;
  const int64_t nt = (a.s.n + kTile - 1) / kTile;
  const int64_t m0 = (int64_t)(blockIdx.x / nt) * kTile, n0 = (int64_t)(blockIdx.x % nt) * kTile;
  const T* x = (const T*)a.x;
  const T* w = (const T*)a.w;
  floatx16 acc[GATED ? 2 : 1] = {};
  for (int64_t k0 = 0; k0 < a.s.k; k0 += kStep) {
    for (int i = threadIdx.x; i < kTile * kStep; i += 256) {
      const int row = i / kStep, kk = i % kStep;
      const bool in = k0 + kk < a.s.k;
      xs[row * kPitch + kk] = in && m0 + row < a.s.m ? x[(m0 + row) * a.s.ldx + k0 + kk] : (T)0.f;
#pragma unroll
      for (int g = 0; g < (GATED ? 2 : 1); ++g)
        wsm[(g * kTile + row) * kPitch + kk] =
            in && n0 + row < a.s.n ? w[(g * a.s.n + n0 + row) * a.s.ldw + k0 + kk] : (T)0.f;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kStep; s += 16) {
      const int kk = s + 8 * (lane >> 5);
      const V8 b = *(const V8*)&xs[(tm + (lane & 31)) * kPitch + kk];
#pragma unroll
      for (int g = 0; g < (GATED ? 2 : 1); ++g)
        acc[g] = E::mfma(*(const V8*)&wsm[(g * kTile + tn + (lane & 31)) * kPitch + kk], b, acc[g]);
    }
    __syncthreads();
  }
  const int64_t m = m0 + tm + (lane & 31);
  if (m >= a.s.m) return;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int64_t n = n0 + tn + drow(r, lane >> 5);
    if (n >= a.s.n) continue;
    float v = acc[0][r] + (a.b ? (float)((const T*)a.b)[n] : 0.f);
    v = activate<ACT>(v);
    if (GATED) v *= acc[1][r] + (a.b ? (float)((const T*)a.b)[a.s.n + n] : 0.f);
    if (a.r) v += (float)((const T*)a.r)[m * a.s.ldr + n];
    ((T*)a.y)[m * a.s.ldy + n] = (T)v;
  }
}

template <class E, int ACT, bool GATED>
hipError_t go(const LinearArgs& a, hipStream_t st) {
  const int64_t grid = ((a.s.m + kTile - 1) / kTile) * ((a.s.n + kTile - 1) / kTile);
  if (grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  launch(k_tok_linear<E, ACT, GATED>, dim3((unsigned)grid), dim3(256), st, a);
  return hipGetLastError();
}

template <class E, bool GATED>
hipError_t by_act(const LinearArgs& a, hipStream_t st) {
  switch (a.s.act) {
    case NCODEC_ACT_LRELU: return go<E, NCODEC_ACT_LRELU, GATED>(a, st);
    case NCODEC_ACT_WSILU: return go<E, NCODEC_ACT_WSILU, GATED>(a, st);
    case NCODEC_ACT_SILU: return go<E, NCODEC_ACT_SILU, GATED>(a, st);
    case NCODEC_ACT_GELU: return go<E, NCODEC_ACT_GELU, GATED>(a, st);
    default: return go<E, NCODEC_ACT_NONE, GATED>(a, st);
  }
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, hipStream_t st) {
  if (a.s.dtype == NCODEC_DTYPE_FP16) return a.s.gated ? by_act<F16, true>(a, st) : by_act<F16, false>(a, st);
  return a.s.gated ? by_act<BF16, true>(a, st) : by_act<BF16, false>(a, st);
}

}  // namespace nc
