// Shared by the token operators (matrix product with epilogue, head norms with
// rotation, attention with a decay): element types and the launch interface.
#pragma once
#include "common.hpp"
#include "internal.hpp"

typedef __bf16 bf16;
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bhalf4 __attribute__((ext_vector_type(4)));
typedef __bf16 bhalf2 __attribute__((ext_vector_type(2)));

namespace nc {

// The two element types behind one interface; mfma: 32x32x16, fp32 accumulate,
// lane l holds row (A) or column (B) l % 32 and k = 8 (l / 32) + e.
struct F16 {
  typedef f16 T;
  typedef half8 V8;
  typedef half4 V4;
  typedef half2 V2;
  static __device__ __forceinline__ floatx16 mfma(V8 a, V8 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};
struct BF16 {
  typedef bf16 T;
  typedef bhalf8 V8;
  typedef bhalf4 V4;
  typedef bhalf2 V2;
  static __device__ __forceinline__ floatx16 mfma(V8 a, V8 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};

struct LinearArgs {
  ncodec_linear_shape s;
  const void* x;
  const void* w;
  const void* b;
  const void* r;
  void* y;
};
hipError_t launch_linear(const LinearArgs& a, hipStream_t st);

struct QkArgs {
  ncodec_qk_shape s;
  const void* q;
  const void* k;
  const void* wq;
  const void* wk;
  const int32_t* pos;
  const float* freq;
  void* qo;
  void* ko;
};
hipError_t launch_qk_norm_rope(const QkArgs& a, hipStream_t st);

struct DecayArgs {
  ncodec_decay_shape s;
  const void* q;
  const void* k;
  const void* v;
  const float* log_decay;
  const int32_t* lengths;
  const float* state_in;
  float* state_out;
  void* o;
  void* ws;
};
size_t decay_workspace_bytes(const ncodec_decay_shape& s);
hipError_t launch_decay_attention(const DecayArgs& a, hipStream_t st);

}  // namespace nc
