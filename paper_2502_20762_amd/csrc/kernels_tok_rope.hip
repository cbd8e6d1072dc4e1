// RMS norm of every query and key head and the rotation by the token's
// position, in one pass over q and k: each element is read once and written
// once, so the bytes are the bound: 130,560 tokens of 10 + 10 heads of 128, 1.34 GB, take
// 235 us (5.7 TB/s; a large copy reaches 5.0 and one inside the last-level cache 6.6),
// 8,160 tokens of 8 + 8 heads of 64, 33 MB, 8.4 us (4.0 TB/s).  A few tokens take the 2.5 to
// 3 us of a launch.
#include <algorithm>

#include "tokens.hpp"

namespace nc {
namespace {

constexpr int kTable = 1024;  // pairs of a workgroup's tokens: 8 tokens of the largest head

// cos and sin of pos * freq radians.  The angle is counted in turns in 64
// bits, where a 31-bit position times a 24-bit frequency is exact up to the
// factor 1 / (2 pi), and only its fraction goes to 32 bits (v_sin_f32 and
// v_cos_f32 take turns), so a late token is turned as exactly as the first.
__device__ __forceinline__ float2 turn(int pos, float freq) {
  const double t = (double)pos * ((double)freq * 0.15915494309189533577);
  const float f = (float)(t - __builtin_floor(t));
  return make_float2(__builtin_amdgcn_cosf(f), __builtin_amdgcn_sinf(f));
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, false));
}
// Sum over the 2^log2g neighbouring lanes of a group, in every lane of it.
__device__ __forceinline__ float group_sum(float v, int log2g) {
  if (log2g > 0) v += dpp<0xB1>(v);   // lanes i ^ 1
  if (log2g > 1) v += dpp<0x4E>(v);   // i ^ 2
  if (log2g > 2) v += dpp<0x141>(v);  // mirrored in 8: the other four, which are all alike
  if (log2g > 3) v += dpp<0x140>(v);  // mirrored in 16
  if (log2g > 4) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  if (log2g > 5) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  return v;
}

struct RopeArgs {
  QkArgs a;
  int tokens;      // of a workgroup
  int log2g;       // lanes of a head
  uint32_t magic;  // ceil(2^32 / heads): row / heads = row * magic >> 32 for the rows of a workgroup (heads > 1)
};

// A lane holds VEC pairs of a head (two runs of VEC elements), a group of lanes
// the head, a workgroup all heads of a few tokens.  The sines and cosines of
// those tokens are formed once, in LDS, for all their heads.  UPL: units a
// lane holds (2 only where a head has more than 64 units).
template <class E, int VEC, int UPL>
__global__ __launch_bounds__(256) void k_tok_rope(RopeArgs ra) {
  typedef typename E::T T;
  typedef T TV __attribute__((ext_vector_type(VEC)));
  __shared__ __align__(16) float2 cs[kTable];
  const ncodec_qk_shape& s = ra.a.s;
  const int P = s.section[0] + s.section[1] + s.section[2], D = s.head_dim, H = s.q_heads + s.k_heads;
  const int64_t tk0 = (int64_t)blockIdx.x * ra.tokens;
  const int nt = (int)min((int64_t)ra.tokens, s.tokens - tk0);
  const int G = 1 << ra.log2g, gl = threadIdx.x & (G - 1);

  // this lane's units: rotated ones first, then the dimensions that pass
  const int RU = (P + VEC - 1) / VEC;
  int offa[UPL], offb[UPL];
  bool rot[UPL];
  TV wq[UPL][2], wk[UPL][2];
#pragma unroll
  for (int x = 0; x < UPL; ++x) {
    const int u = gl + x * G;
    rot[x] = u < RU;
    offa[x] = !rot[x] ? 2 * P + 2 * VEC * (u - RU) : s.interleaved ? 2 * VEC * u : VEC * u;
    offb[x] = rot[x] && !s.interleaved ? P + VEC * u : offa[x] + VEC;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int off = y ? offb[x] : offa[x];
#pragma unroll
      for (int e = 0; e < VEC; ++e) wq[x][y][e] = wk[x][y][e] = (T)1.f;
      if (s.norm && off < D) {
        if (ra.a.wq) __builtin_memcpy(&wq[x][y], (const T*)ra.a.wq + off, sizeof(TV));
        if (ra.a.wk) __builtin_memcpy(&wk[x][y], (const T*)ra.a.wk + off, sizeof(TV));
      }
    }
  }
  for (int i = threadIdx.x; i < nt * P; i += 256) {
    const int t = i / P, p = i - t * P;
    const int axis = p < s.section[0] ? 0 : p < s.section[0] + s.section[1] ? 1 : 2;
    cs[t * P + p] = turn(ra.a.pos[(tk0 + t) * s.axes + axis], ra.a.freq[p]);
  }
  __syncthreads();

  const float inv_d = 1.f / (float)D;
  for (int row = threadIdx.x >> ra.log2g; row < nt * H; row += 256 >> ra.log2g) {
    const int t = H == 1 ? row : (int)__umulhi((uint32_t)row, ra.magic), hh = row - t * H;
    const bool is_q = hh < s.q_heads;
    const int64_t tok = tk0 + t, hd = is_q ? hh : hh - s.q_heads;
    const T* x = is_q ? (const T*)ra.a.q + tok * s.q_token_stride + hd * s.q_head_stride
                      : (const T*)ra.a.k + tok * s.k_token_stride + hd * s.k_head_stride;
    T* y = is_q ? (T*)ra.a.qo + tok * s.qo_token_stride + hd * s.qo_head_stride
                : (T*)ra.a.ko + tok * s.ko_token_stride + hd * s.ko_head_stride;
    float v[UPL][2][VEC];
#pragma unroll
    for (int i = 0; i < UPL; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int off = j ? offb[i] : offa[i];
        TV r = {};
        if (off < D) __builtin_memcpy(&r, x + off, sizeof(TV));
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i][j][e] = (float)r[e];
      }
    if (s.norm) {
      float sq = 0.f;
#pragma unroll
      for (int i = 0; i < UPL; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < VEC; ++e) sq = fmaf(v[i][j][e], v[i][j][e], sq);
      const float inv = __builtin_amdgcn_rsqf(fmaf(group_sum(sq, ra.log2g), inv_d, s.eps));
#pragma unroll
      for (int i = 0; i < UPL; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < VEC; ++e) v[i][j][e] *= inv * (float)(is_q ? wq[i][j][e] : wk[i][j][e]);
    }
#pragma unroll
    for (int i = 0; i < UPL; ++i) {
      if (rot[i]) {
        const float2* c = cs + t * P + VEC * (gl + i * G);
        float2 tab[VEC];
        __builtin_memcpy(tab, __builtin_assume_aligned(c, VEC == 1 ? 8 : 16), sizeof(tab));
        if (s.interleaved && VEC > 1) {
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < VEC / 2; ++e) {
              const float2 w = tab[j * (VEC / 2) + e];
              const float a = v[i][j][2 * e], b = v[i][j][2 * e + 1];
              v[i][j][2 * e] = fmaf(-b, w.y, a * w.x);
              v[i][j][2 * e + 1] = fmaf(b, w.x, a * w.y);
            }
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float a = v[i][0][e], b = v[i][1][e];
            v[i][0][e] = fmaf(-b, tab[e].y, a * tab[e].x);
            v[i][1][e] = fmaf(b, tab[e].x, a * tab[e].y);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int off = j ? offb[i] : offa[i];
        TV r;
#pragma unroll
        for (int e = 0; e < VEC; ++e) r[e] = (T)v[i][j][e];
        if (off < D) __builtin_memcpy(y + off, &r, sizeof(TV));
      }
    }
  }
}

template <class E, int VEC, int UPL>
hipError_t go(const QkArgs& a, int units, hipStream_t st) {
  const ncodec_qk_shape& s = a.s;
  RopeArgs ra{a, 1, 0, 0};
  while (ra.log2g < 6 && (1 << ra.log2g) * UPL < units) ++ra.log2g;
  const int64_t H = s.q_heads + s.k_heads;
  // Tokens of a workgroup: 16 KiB of values (two rounds of its lanes), so that the sines
  // and the start are spread over enough of them (130,560 tokens, 8 + 8 heads of 64: 8 tokens
  // 95 us, one 179; 1 + 1 heads: 32 tokens 17 us, 8 tokens 24) and one round's loads run
  // beside the other's stores (16 + 16 heads of 128: 2 tokens 354 us, 1 or 8 390 to 399), and
  // no more than leaves three workgroups a CU (2,048 tokens of 8 + 8 heads of 64: 2 tokens 3.9
  // us, one 4.7, eight 4.4; 256 tokens 2.9 with one, 3.9 with eight).
  const int64_t bytes = 2 * H * s.head_dim, pairs = std::max(1, s.section[0] + s.section[1] + s.section[2]);
  ra.tokens = (int)std::max<int64_t>(1, std::min({kTable / pairs, 16384 / bytes, s.tokens / 768}));
  ra.magic = (uint32_t)((((uint64_t)1 << 32) + H - 1) / H);
  // a launch counts its threads in 32 bits: tokens past 2^22 workgroups go in further ones
  const int64_t most = ((int64_t)1 << 22) * ra.tokens;
  for (int64_t t0 = 0; t0 < s.tokens; t0 += most) {
    ra.a.s.tokens = std::min(most, s.tokens - t0);
    ra.a.q = (const char*)a.q + 2 * t0 * s.q_token_stride;
    ra.a.k = (const char*)a.k + 2 * t0 * s.k_token_stride;
    ra.a.qo = (char*)a.qo + 2 * t0 * s.qo_token_stride;
    ra.a.ko = (char*)a.ko + 2 * t0 * s.ko_token_stride;
    if (a.pos) ra.a.pos = a.pos + t0 * s.axes;
    launch(k_tok_rope<E, VEC, UPL>, dim3((unsigned)((ra.a.s.tokens + ra.tokens - 1) / ra.tokens)), dim3(256), st, ra);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Runs of eight or four elements where head_dim and the pairs are made of them
// (16- and 8-byte accesses), single elements otherwise: 130,560 tokens of 16 + 16 heads of
// 128 take 356, 403 and 656 us so.
template <class E>
hipError_t pick(const QkArgs& a, hipStream_t st) {
  const int P = a.s.section[0] + a.s.section[1] + a.s.section[2], D = a.s.head_dim;
  if (D % 16 == 0 && P % 8 == 0) return go<E, 8, 1>(a, D / 16, st);
  if (D % 8 == 0 && P % 4 == 0) return go<E, 4, 1>(a, D / 8, st);
  if (D <= 128) return go<E, 1, 1>(a, (D + 1) / 2, st);
  return go<E, 1, 2>(a, (D + 1) / 2, st);
}

}  // namespace

hipError_t launch_qk_norm_rope(const QkArgs& a, hipStream_t st) {
  return a.s.dtype == NCODEC_DTYPE_FP16 ? pick<F16>(a, st) : pick<BF16>(a, st);
}

}  // namespace nc
