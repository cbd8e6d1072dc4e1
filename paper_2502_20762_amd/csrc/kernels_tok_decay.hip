// Linear attention with a decay for each head:
//   S_t = lambda S_{t-1} + k_t v_t^T,  o_t = scale q_t S_t.
//
// Two forms.  A few tokens run the recurrence itself.  Longer ones go in chunks
// of 64 tokens, whose outputs are two products, one with the state before the
// chunk and one inside the chunk,
//   o_i = scale (lambda^(i+1) q_i S + sum_{j<=i} lambda^(i-j) (q_i . k_j) v_j),
//   S' = lambda^n S + sum_j lambda^(n-1-j) k_j v_j^T,
// all of them MFMA work.  Where there are too few heads to fill the chip a
// sequence is cut into segments: their contributions to the state first (one
// pass over k and v), then a scan over the segments, then the outputs.
#include <algorithm>

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

// ---- chunks -------------------------------------------------------------------
constexpr int kChunk = 64;

template <class E, int DP_, int NV_>
struct Chunk {
  static constexpr int DP = DP_, NV = NV_, VP = 32 * NV_;  // padded head and value width; a wave per 32 values
  static constexpr int DT = DP / 32;
  static constexpr int QB = kChunk * DP * 2, VB = kChunk * VP * 2;
  static constexpr int STAGE = 2 * QB + VB;  // q, k, v of a chunk
  static constexpr uint32_t INF = __is_same(E, F16) ? 0x7c00 : 0x7f80;
  static constexpr int OPITCH = 80;          // a token's 32 outputs of a wave, padded
  static constexpr int LDS = 2 * STAGE + NV * 32 * OPITCH;
};

// Slot of 16-byte unit u of a row of W elements: 16 consecutive rows of one
// unit, and four consecutive rows of four units (a transposed read), each
// touch every LDS bank once.
template <int W>
__device__ __forceinline__ int unit_slot(int row, int u) {
  if (W == 128) return u ^ (((row & 3) << 2) | ((row >> 2) & 3));
  if (W == 64) return u ^ ((((row >> 1) & 1) << 2) | ((row >> 2) & 3));
  return u ^ ((row >> 2) & 3);
}

__device__ __align__(16) uint32_t decay_zero16[4];

// Stage a chunk of a tensor into LDS: rows pad .. 63 from base (the address of
// row 0), d valid elements of W, zeros elsewhere.  DMA: direct global->LDS loads,
// which the caller waits for; rows are then 16-byte aligned and their stride is
// below 2^26.
template <class E, int W, int NW, bool DMA>
__device__ __forceinline__ void stage_rows(char* lds, const typename E::T* base, int64_t stride, int pad, int d, int wave,
                                           int lane) {
  typedef typename E::V8 V8;
  constexpr int U = W / 8, R = 64 / U, LOADS = kChunk / R;
  static_assert(LOADS % NW == 0, "every wave loads as much");
  const int r0 = lane / U, u0 = unit_slot<W>(r0, lane % U);
  const char* rows = (const char*)(base + (int64_t)(R * wave) * stride);
  const int64_t step = (int64_t)(R * NW) * stride * 2;
  if (DMA && pad == 0 && d == W) {
    const uint32_t voff = (uint32_t)r0 * (uint32_t)stride * 2u;
#pragma unroll
    for (int i0 = 0; i0 < LOADS / NW; ++i0) {
      const int i = wave + NW * i0;
      dma16s(rows, voff + 16 * (u0 ^ unit_slot<W>(R * i, 0)), lds + 1024 * i);
      rows += step;
    }
  } else {
#pragma unroll
    for (int i0 = 0; i0 < LOADS / NW; ++i0) {
      const int i = wave + NW * i0, u = u0 ^ unit_slot<W>(R * i, 0);
      const char* p = rows + r0 * stride * 2 + 16 * u;
      const bool in = R * i + r0 >= pad && 8 * u < d;
      if (DMA) {
        dma16(in ? (const void*)p : (const void*)decay_zero16, lds + 1024 * i);
      } else {
        V8 v = {};
        if (in) {
          if (8 * u + 8 <= d)
            __builtin_memcpy(&v, p, 16);
          else
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (8 * u + e < d) v[e] = ((const typename E::T*)p)[e];
        }
        *(V8*)(lds + 1024 * i + 16 * lane) = v;
      }
      rows += step;
    }
  }
}

// Byte offset, in an LDS tile of W wide rows, of unit h of row l32; unit
// 2 x + h of row l32 + 32 t lies at (this ^ 32 x) + 64 W t.
template <int W>
__device__ __forceinline__ int row_offset(int lane) {
  return (lane & 31) * (2 * W) + 16 * unit_slot<W>(lane & 31, lane >> 5);
}

// Transposed read of four rows x 16 columns per 16 lanes: lane i of the 16
// passes the address of element (i / 4, 4 (i % 4)) and receives column i of the
// four rows.
__device__ __forceinline__ half4 read_tr(const char* p, F16) {
  typedef __fp16 H4 __attribute__((vector_size(8)));
  typedef H4 __attribute__((address_space(3))) L;
  return __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((L*)p));
}
__device__ __forceinline__ bhalf4 read_tr(const char* p, BF16) {
  typedef bhalf4 __attribute__((address_space(3))) L;
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((L*)p);
}
// MFMA fragment of 32 columns of an LDS tile as rows, contraction over the
// tile's rows ("tokens") in the order of an accumulator: lane half h, element e
// holds token 16 s + 8 (e / 4) + 4 h + e % 4.  Two transposed reads, p = 0 and 1,
// at col_offset(p); columns 32 d.. lie at (that ^ 64 d), tokens 16 s.. at that +
// 32 W s.  With PI the columns of each 16 are taken as 0-3, 8-11, 4-7, 12-15, so
// that a lane of the resulting accumulator holds eight consecutive columns in
// eight registers.
template <int W, bool PI>
__device__ __forceinline__ int col_offset(int lane, int p) {
  const int h = lane >> 5, c = (lane >> 4) & 1, i = lane & 15, k = i & 3;
  const int col = 16 * c + 4 * (PI ? ((k & 1) << 1 | k >> 1) : k), row = 8 * p + 4 * h + (i >> 2);
  return row * (2 * W) + 16 * unit_slot<W>(row, col >> 3) + 2 * (col & 7);
}
template <class E>
__device__ __forceinline__ typename E::V8 read_cols(const char* p0, const char* p1) {
  const auto x = read_tr(p0, E{}), y = read_tr(p1, E{});
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}

// max over all lanes
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(b[0], b[1]);
#define NC_ROR(N) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xf, 0xf, false));
  NC_ROR(8) NC_ROR(4) NC_ROR(2) NC_ROR(1)
#undef NC_ROR
  return __builtin_amdgcn_readfirstlane(v);
}
// of a value >= 0 that is no NaN: its bits order it
__device__ __forceinline__ float wave_max(float v) { return __uint_as_float(wave_max(__float_as_uint(v))); }
template <class V8>
__device__ __forceinline__ uint32_t max_bits(V8 v) {  // of eight 16-bit magnitudes
  typedef unsigned short US8 __attribute__((ext_vector_type(8)));
  typedef unsigned short US2 __attribute__((ext_vector_type(2)));
  const US8 u = __builtin_bit_cast(US8, v) & (unsigned short)0x7fff;
  US2 m = __builtin_elementwise_max(__builtin_elementwise_max(u.s01, u.s23), __builtin_elementwise_max(u.s45, u.s67));
  return max((uint32_t)m.x, (uint32_t)m.y);
}
// max(m, |a|, |b|), NaN ignored
__device__ __forceinline__ float max3_abs(float m, float a, float b) {
  asm("v_max3_f32 %0, %0, |%1|, |%2|" : "+v"(m) : "v"(a), "v"(b));
  return m;
}
__device__ __forceinline__ float max_abs(float m, const floatx16& v) {
#pragma unroll
  for (int r = 0; r < 16; r += 2) m = max3_abs(m, v[r], v[r + 1]);
  return m;
}
__device__ __forceinline__ float half_max(float v) {  // over the two lanes l, l + 32
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// Power of two that takes a largest magnitude m into [2^14, 2^15), and its
// inverse: fp16 operands are brought there, so that no sum of magnitudes and no
// small scale leaves the range in which fp16 has its 11 bits.
__device__ __forceinline__ float scale_up(float m, float* inverse) {
  const uint32_t e = max((__float_as_uint(m) >> 23) & 255u, 15u);
  *inverse = __uint_as_float((e - 14) << 23);
  return __uint_as_float((268 - e) << 23);
}

struct Decay64 {  // lambda^n in two floats, so that long products of it lose nothing
  float hi, lo;
};
__device__ __forceinline__ Decay64 decay_pow(float log_decay, int64_t n) {
  const double l = fmax(fmin((double)log_decay, 0.0), -1e30);
  const double f = exp((double)n * l);
  const float hi = (float)f;
  return {hi, (float)(f - (double)hi)};
}

struct SegArgs {
  DecayArgs a;
  int seg_chunks;  // chunks of a segment
  int nseg;
};

// One segment of one sequence and head.  OUT: the outputs, from the state before
// the segment (and the sequence's last state); otherwise only what the segment
// adds to the state, into the workspace.  Wave w holds the state's columns
// 32 w .. 32 w + 31 in its accumulators: register r of tile a and lane (h, c) is
// row 32 a + 16 (r / 8) + 8 h + r % 8, column 32 w + c.
template <class E, int DP, int NV, bool OUT, bool DMA>
__global__ __launch_bounds__(64 * NV, DP <= 64 ? 2 : 1) void k_tok_decay_chunk(SegArgs sa) {
  typedef Chunk<E, DP, NV> C;
  typedef typename E::T T;
  typedef typename E::V8 V8;
  typedef typename E::V4 V4;
  constexpr bool F = __is_same(E, F16);
  constexpr int DT = C::DT, VP = C::VP, NT = F ? 2 : 3;  // NT: 16-bit terms of a weighted value
  constexpr int STAGE = OUT ? C::STAGE : C::QB + C::VB;
  __shared__ __align__(1024) char lds[OUT ? C::LDS : 2 * STAGE];
  const DecayArgs& a = sa.a;
  const ncodec_decay_shape& s = a.s;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, l32 = lane & 31;
  const int nsg = OUT ? sa.nseg : sa.nseg - 1;
  const int64_t bh = blockIdx.x / nsg;
  const int seg = blockIdx.x % nsg;
  const int64_t b = bh / s.heads, hd = bh % s.heads, hk = hd / (s.heads / s.kv_heads);
  const int D = s.head_dim, V = s.value_dim;
  const int64_t len = a.lengths ? min(max((int64_t)a.lengths[b], (int64_t)0), s.tokens) : s.tokens;
  const int64_t SL = (int64_t)sa.seg_chunks * kChunk, t0 = seg * SL;
  const int64_t tend = min(t0 + SL, len);  // tokens [t0, tend) are computed
  const T* q = (const T*)a.q + b * s.q_batch_stride + hd * s.q_head_stride;
  const T* k = (const T*)a.k + b * s.k_batch_stride + hk * s.k_head_stride;
  const T* v = (const T*)a.v + b * s.v_batch_stride + hk * s.v_head_stride;
  T* o = (T*)a.o + b * s.o_batch_stride + hd * s.o_head_stride;
  const int64_t sdv = (int64_t)D * V;
  const int col = 32 * wave + l32;

  if (!OUT && t0 + SL >= len) return;  // no later segment reads it
  if (OUT) {
    // outputs past the sequence's end
    const int64_t z0 = max(t0, len), z1 = min(t0 + SL, s.tokens);
    for (int64_t t = z0 + (threadIdx.x / VP); t < z1; t += 64 * NV / VP)
      if ((int)(threadIdx.x % VP) < V) o[t * s.o_token_stride + threadIdx.x % VP] = (T)0.f;
    if (t0 >= len && seg > 0) return;
  }

  const int nch = tend > t0 ? (int)((tend - t0 + kChunk - 1) / kChunk) : 0;
  // A last chunk of n < 64 tokens sits at the end of its tile, behind 64 - n rows of
  // zeros: the ages and lags of its rows are then those of a full chunk.
  auto stage = [&](int c) {
    const int64_t te = min(t0 + (int64_t)(c + 1) * kChunk, tend), t = te - kChunk;  // of row 0
    const int pad = kChunk - (int)(te - (t0 + (int64_t)c * kChunk));
    char* base = lds + (c & 1) * STAGE;
    stage_rows<E, DP, NV, DMA>(base, k + t * s.k_token_stride, s.k_token_stride, pad, D, wave, lane);
    stage_rows<E, VP, NV, DMA>(base + C::QB, v + t * s.v_token_stride, s.v_token_stride, pad, V, wave, lane);
    if (OUT)
      stage_rows<E, DP, NV, DMA>(base + C::QB + C::VB, q + t * s.q_token_stride, s.q_token_stride, pad, D, wave, lane);
  };
  if (nch) stage(0);

  const float log_decay = a.log_decay[hd];
  const float l2 = log2_decay(log_decay);
  floatx16 S[DT];
  const float* sin = !OUT ? nullptr : seg == 0 ? a.state_in : (const float*)a.ws + (bh * (sa.nseg - 1) + seg - 1) * sdv;
  if (seg == 0 && sin) sin += bh * sdv;
#pragma unroll
  for (int x = 0; x < DT; ++x)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int d = 32 * x + 16 * (r >> 3) + 8 * h + (r & 7);
      S[x][r] = sin && d < D && col < V ? sin[(int64_t)d * V + col] : 0.f;
    }
  float* sout = !OUT ? (float*)a.ws + (bh * (sa.nseg - 1) + seg) * sdv
                : a.state_out && t0 + SL >= len ? a.state_out + bh * sdv : nullptr;

  // Decays.  Inside a diagonal 32 x 32 tile lambda^(i - j) for j <= i (i this lane's
  // token, j the register's), one tile below it lambda^(32 + i - j).  At the end
  // of a chunk token 16 x + j counts lambda^(15 - j) lambda^(48 - 16 x).
  float mdiag[OUT ? 16 : 1], mlow[OUT ? 16 : 1], wage[8], wstep[4];
  if (OUT) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int lag = l32 - drow(r, h);
      mdiag[r] = __builtin_amdgcn_exp2f(max(lag, 0) * l2);
      mlow[r] = __builtin_amdgcn_exp2f((32 + lag) * l2);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) wage[e] = __builtin_amdgcn_exp2f((15 - (8 * (e >> 2) + 4 * h + (e & 3))) * l2);
#pragma unroll
  for (int x = 0; x < 4; ++x) wstep[x] = __builtin_amdgcn_exp2f((48 - 16 * x) * l2);
  Decay64 keep = decay_pow(log_decay, kChunk);
  const int ro = row_offset<DP>(lane);
  const int ck0 = col_offset<DP, true>(lane, 0), ck1 = col_offset<DP, true>(lane, 1);
  const int cv0 = C::QB + (col_offset<VP, false>(lane, 0) ^ (64 * wave)),
            cv1 = C::QB + (col_offset<VP, false>(lane, 1) ^ (64 * wave));
  char* mine = lds + 2 * STAGE + wave * 32 * C::OPITCH;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  for (int c = 0; c < nch; ++c) {
    // every wave's loads of chunk c have landed (each waited for its own), and
    // every wave is done with the other buffer
    lds_barrier();
    if (c + 1 < nch) stage(c + 1);
    const int buf = (c & 1) * STAGE;
    const int64_t t = t0 + (int64_t)c * kChunk;
    const int n = (int)min(tend - t, (int64_t)kChunk), pad = kChunk - n;

    V8 vf[4];
    {
      const char *p0 = lds + (cv0 + buf), *p1 = lds + (cv1 + buf);
#pragma unroll
      for (int x = 0; x < 4; ++x) vf[x] = read_cols<E>(p0 + 32 * VP * x, p1 + 32 * VP * x);
    }
    // largest magnitude, by its bits, which order finite values, infinities and NaN
    uint32_t mb = max(max(max_bits(vf[0]), max_bits(vf[1])), max(max_bits(vf[2]), max_bits(vf[3])));
    mb = wave_max(mb);
    int bad = kChunk;  // first row of this lane's column that is not finite
    const bool any_bad = mb >= C::INF;
    if (any_bad) {
      // a product would carry it to earlier tokens too (0 times NaN): it is taken
      // out here and put into the outputs and the state that it reaches
      mb = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t u = (uint32_t)__builtin_bit_cast(uint16_t, (T)vf[x][e]) & 0x7fffu;
          if (u >= C::INF) {
            bad = min(bad, 16 * x + 8 * (e >> 2) + 4 * h + (e & 3));
            vf[x][e] = (T)0.f;
          } else {
            mb = max(mb, u);
          }
        }
      mb = wave_max(mb);
      bad = min(bad, __shfl_xor(bad, 32, 64));
    }
    float vinv = 1.f;
    if (F) {  // a power of two, exact in fp16: what is lost lies 2^-24 below 2^14
      const float m = fmaxf((float)__builtin_bit_cast(f16, (uint16_t)mb), 0.5f);
      const float up = scale_up(m, &vinv);
#pragma unroll
      for (int x = 0; x < 4; ++x) vf[x] = vf[x] * (T)up;
    }

    if (OUT) {
      float sinv = 1.f, sup = 1.f;
      if (F) {
        float m = 0.f;
#pragma unroll
        for (int x = 0; x < DT; ++x) m = max_abs(m, S[x]);
        m = wave_max(m);
        if (m == __builtin_huge_valf()) {  // the finite ones keep their scale
          m = 0.f;
#pragma unroll
          for (int x = 0; x < DT; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (fabsf(S[x][r]) < __builtin_huge_valf()) m = fmaxf(m, fabsf(S[x][r]));
          m = wave_max(m);
        }
        sup = scale_up(m, &sinv);
      }
#pragma unroll
      for (int it = 0; it < 2; ++it) {  // 32 queries
        __builtin_amdgcn_sched_barrier(0);
        floatx16 p[2] = {}, inter = {};
        const int rb = ro + buf;
#pragma unroll
        for (int x = 0; x < 2 * DT; ++x) {
          const char* r = lds + (rb ^ (32 * x));
          const V8 qf = *(const V8*)(r + (C::QB + C::VB + 64 * DP * it));
#pragma unroll
          for (int jt = 0; jt <= it; ++jt) p[jt] = E::mfma(*(const V8*)(r + 64 * DP * jt), qf, p[jt]);
          V8 sf;
#pragma unroll
          for (int e = 0; e < 8; ++e) sf[e] = (T)(F ? S[x >> 1][8 * (x & 1) + e] * sup : S[x >> 1][8 * (x & 1) + e]);
          inter = E::mfma(sf, qf, inter);
        }
        __builtin_amdgcn_sched_barrier(0);
        // pairs above the diagonal count nothing, whatever their product is
        int tok = l32;
        asm volatile("" : "+v"(tok));  // compared here and not before the loop, where 16 masks would have to be kept
#pragma unroll
        for (int r = 0; r < 16; ++r) p[it][r] = drow(r, h) > tok ? 0.f : p[it][r];
        float pinv = 1.f, pup = 1.f;
        if (F) {
          float m = max_abs(0.f, p[0]);
          if (it) m = max_abs(m, p[1]);
          pup = scale_up(half_max(m), &pinv);
        }
        floatx16 intra = {};
#pragma unroll
        for (int jt = 0; jt <= it; ++jt) {
          V8 pf[2];
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float w = jt == it ? mdiag[r] : mlow[r];
            pf[r >> 3][r & 7] = (T)(F ? p[jt][r] * pup * w : p[jt][r] * w);
          }
          intra = E::mfma(vf[2 * jt], pf[0], intra);
          intra = E::mfma(vf[2 * jt + 1], pf[1], intra);
        }
        // row i is token i - pad of the chunk; rows of the padding are not stored
        const float di = __builtin_amdgcn_exp2f(max(32 * it + l32 + 1 - pad, 0) * l2);
        const float ci = s.scale * di * sinv, cp = s.scale * pinv * vinv;
#pragma unroll
        for (int r = 0; r < 16; ++r) inter[r] = fmaf(inter[r], ci, intra[r] * cp);
        if (any_bad) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (32 * it + l32 >= __shfl(bad, drow(r, h), 64)) inter[r] = __builtin_nanf("");
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          V4 x;
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = (T)inter[4 * g + j];
          *(V4*)(mine + l32 * C::OPITCH + 16 * g + 8 * h) = x;
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int row = 16 * y + (lane >> 2), u = lane & 3;
          const V8 x = *(const V8*)(mine + row * C::OPITCH + 16 * u);
          const int left = V - (32 * wave + 8 * u);
          if (32 * it + row >= pad && left > 0) {
            T* p = o + (t + 32 * it + row - pad) * s.o_token_stride + 32 * wave + 8 * u;
            if (left >= 8)
              __builtin_memcpy(p, &x, 16);
            else
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (e < left) p[e] = x[e];
          }
        }
        __builtin_amdgcn_wave_barrier();
      }
    }

    if (!OUT || c + 1 < nch || sout) {
      __builtin_amdgcn_sched_barrier(0);
      // the state: v weighted by its age, as a sum of 16-bit terms that holds 22 (fp16)
      // or 24 (bf16) bits, because the state is an fp32 output
      V8 term[4][NT];
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float w = (float)vf[x][e] * (wage[e] * wstep[x]);
          // one value of the product for all terms: formed anew for a term (fused,
          // rounded once instead of twice) it could differ from the one subtracted
          asm("" : "+v"(w));
#pragma unroll
          for (int y = 0; y < NT; ++y) {
            term[x][y][e] = (T)w;
            w -= (float)term[x][y][e];
          }
        }
      __builtin_amdgcn_sched_barrier(0);
      if (pad) keep = decay_pow(log_decay, n);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const char *p0 = lds + ((ck0 + buf) ^ (64 * d)), *p1 = lds + ((ck1 + buf) ^ (64 * d));
        floatx16 add = {};
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const V8 kf = read_cols<E>(p0 + 32 * DP * x, p1 + 32 * DP * x);
#pragma unroll
          for (int y = NT - 1; y >= 0; --y) add = E::mfma(kf, term[x][y], add);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) S[d][r] = fmaf(S[d][r], keep.hi, fmaf(S[d][r], keep.lo, F ? add[r] * vinv : add[r]));
      }
      if (any_bad && bad < kChunk) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) S[d][r] = __builtin_nanf("");
      }
    }
    // this wave's part of the next chunk has landed (and its stores, long sent)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }

  if (sout) {
#pragma unroll
    for (int x = 0; x < DT; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int d = 32 * x + 16 * (r >> 3) + 8 * h + (r & 7);
        if (d < D && col < V) sout[(int64_t)d * V + col] = S[x][r];
      }
  }
}

// Over the segments of a sequence and head: what each adds becomes the state
// after it (slot g: the state before segment g + 1).
__global__ __launch_bounds__(256) void k_tok_decay_scan(SegArgs sa) {
  const DecayArgs& a = sa.a;
  const ncodec_decay_shape& s = a.s;
  const int64_t sdv = (int64_t)s.head_dim * s.value_dim;
  const int blocks = (int)((sdv + 255) / 256);
  const int64_t bh = blockIdx.x / blocks, e = (int64_t)(blockIdx.x % blocks) * 256 + threadIdx.x;
  if (e >= sdv) return;
  const int64_t b = bh / s.heads;
  const int64_t len = a.lengths ? min(max((int64_t)a.lengths[b], (int64_t)0), s.tokens) : s.tokens;
  const int64_t SL = (int64_t)sa.seg_chunks * kChunk;
  const Decay64 keep = decay_pow(a.log_decay[bh % s.heads], SL);
  const int last = (int)min((len + SL - 1) / SL, (int64_t)sa.nseg) - 1;  // segment 0 .. last have tokens
  float* ws = (float*)a.ws + bh * (sa.nseg - 1) * sdv + e;
  float S = a.state_in ? a.state_in[bh * sdv + e] : 0.f;
  // the loads do not depend on each other: sixteen in flight
  constexpr int N = 16;
  for (int g0 = 0; g0 < last; g0 += N) {
    float add[N];
#pragma unroll
    for (int i = 0; i < N; ++i) add[i] = g0 + i < last ? ws[(g0 + i) * sdv] : 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (g0 + i >= last) break;
      S = fmaf(S, keep.hi, fmaf(S, keep.lo, add[i]));
      ws[(g0 + i) * sdv] = S;
    }
  }
}

// Sequences shorter than this run the recurrence (few workgroups, no chunk to fill).
constexpr int64_t kRecurTokens = 8;

struct Plan {
  bool chunked;
  int seg_chunks, nseg;
};

// Segments so that about kTargetWGs workgroups share the work.
Plan plan_of(const ncodec_decay_shape& s) {
  Plan p{s.tokens >= kRecurTokens, 0, 1};
  const int64_t chunks = (s.tokens + kChunk - 1) / kChunk, bh = s.batch * s.heads;
  if (!p.chunked || bh == 0) return p;
  const int64_t target = s.head_dim > 64 || s.value_dim > 64 ? 256 : 512;
  int64_t nseg = std::max<int64_t>(1, std::min(chunks, target / bh));
  const int64_t per = (chunks + nseg - 1) / nseg;
  p.seg_chunks = (int)per;
  p.nseg = (int)((chunks + per - 1) / per);
  return p;
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

template <class E, int DP, int NV, bool DMA>
hipError_t chunked(const SegArgs& sa, hipStream_t st) {
  const ncodec_decay_shape& s = sa.a.s;
  const int64_t bh = s.batch * s.heads;
  if (sa.nseg > 1) {
    launch(k_tok_decay_chunk<E, DP, NV, false, DMA>, dim3((unsigned)(bh * (sa.nseg - 1))), dim3(64 * NV), st, sa);
    const int64_t sdv = (int64_t)s.head_dim * s.value_dim;
    launch(k_tok_decay_scan, dim3((unsigned)(bh * ((sdv + 255) / 256))), dim3(256), st, sa);
  }
  launch(k_tok_decay_chunk<E, DP, NV, true, DMA>, dim3((unsigned)(bh * sa.nseg)), dim3(64 * NV), st, sa);
  return hipGetLastError();
}

template <class E, int DP, bool DMA>
hipError_t by_value(const SegArgs& sa, hipStream_t st) {
  if (sa.a.s.value_dim <= 32) return chunked<E, DP, 1, DMA>(sa, st);
  if (sa.a.s.value_dim <= 64) return chunked<E, DP, 2, DMA>(sa, st);
  return chunked<E, DP, 4, DMA>(sa, st);
}

template <class E, bool DMA>
hipError_t by_dim(const SegArgs& sa, hipStream_t st) {
  if (sa.a.s.head_dim <= 64) return by_value<E, 64, DMA>(sa, st);
  return by_value<E, 128, DMA>(sa, st);
}

template <class E>
hipError_t run(const DecayArgs& a, hipStream_t st) {
  const ncodec_decay_shape& s = a.s;
  const Plan p = plan_of(s);
  if (!p.chunked) return recur<E>(a, st);
  const auto direct = [](const void* x, int64_t batch, int64_t token, int64_t head) {
    return (uintptr_t)x % 16 == 0 && batch % 8 == 0 && token % 8 == 0 && head % 8 == 0 && token < (1 << 26);
  };
  const bool dma = s.head_dim % 8 == 0 && s.value_dim % 8 == 0 &&
                   direct(a.q, s.q_batch_stride, s.q_token_stride, s.q_head_stride) &&
                   direct(a.k, s.k_batch_stride, s.k_token_stride, s.k_head_stride) &&
                   direct(a.v, s.v_batch_stride, s.v_token_stride, s.v_head_stride);
  const SegArgs sa{a, p.seg_chunks, p.nseg};
  return dma ? by_dim<E, true>(sa, st) : by_dim<E, false>(sa, st);
}

}  // namespace

size_t decay_workspace_bytes(const ncodec_decay_shape& s) {
  const Plan p = plan_of(s);
  return (size_t)(s.batch * s.heads) * (size_t)(p.nseg - 1) * (size_t)(s.head_dim * s.value_dim) * 4;
}

hipError_t launch_decay_attention(const DecayArgs& a, hipStream_t st) {
  return a.s.dtype == NCODEC_DTYPE_FP16 ? run<F16>(a, st) : run<BF16>(a, st);
}

}  // namespace nc
