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
//
// The bytes of q, k, v and o are the floor.  What bounds the chunks is not them but
// the work between two of them: a wave goes through scores, outputs and state one
// after the other, MFMAs and the arithmetic on their results taking turns.  130,560
// tokens of 16 heads of 128 x 128, fp16, 2.1 GB: 832 us (2.6 TB/s; 219 + 14 + 591 at best, in
// the last VALU issuing 64 % of the CUs' busy time, MFMAs 42 %); 64 sequences of 512 tokens, 8 heads of 64 x
// 64, 134 MB: 43 us (3.1 TB/s); 8,160 tokens of 8 heads of 64 x 64, 33 MB: 32 us, three launches
// of 9, 6 and 17.
#include <algorithm>

#include "token_rules.hpp"
#include "tokens.hpp"

namespace nc {
namespace {

// lambda^n = exp2(n * this).  Positive decays count as 0, -inf becomes a
// number so that lambda^0 is 1 (0 * -inf is not a number).  A NaN stays one: these
// minima and maxima keep it.
__device__ __forceinline__ float log2_decay(float log_decay) {
  return __builtin_elementwise_maximum(__builtin_elementwise_minimum(log_decay, 0.f), -1e30f) * 1.44269504088896341f;
}

struct Decay64 {  // lambda^n in two floats, so that long products of it lose nothing
  float hi, lo;
};
__device__ __forceinline__ Decay64 decay_pow(float log_decay, int64_t n) {
  const double l = __builtin_elementwise_maximum(__builtin_elementwise_minimum((double)log_decay, 0.0), -1e30);
  const double f = exp((double)n * l);
  const float hi = (float)f;
  return {hi, (float)(f - (double)hi)};
}

// The recurrence itself, token by token.  A workgroup holds 64 columns of one
// sequence's and head's state in registers: thread (g, c) the rows g + 16 r and
// the columns 4 c .. 4 c + 3.  For one token it reads and writes the state once and is
// bound by that: 512 heads of 64 x 64, 17 MB, 5.2 us (3.2 TB/s), of 128 x 128, 67 MB, 13.2
// (5.1 TB/s).  VEC, where value_dim is a multiple of 4 and the states are 16-byte aligned:
// 8.3 and 22.2 us in single elements.
template <class E, int R, bool VEC>
__global__ __launch_bounds__(256) void k_tok_decay_recur(DecayArgs a) {
  typedef typename E::T T;
  __shared__ float qs[16 * R], ks[16 * R], part[4][64];
  const ncodec_decay_shape& s = a.s;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = lane & 15, g = wave * 4 + (lane >> 4);
  const uint32_t b = blockIdx.x / (uint32_t)s.heads, h = blockIdx.x - b * s.heads,
                 hk = h / ((uint32_t)s.heads / (uint32_t)s.kv_heads);
  const int D = s.head_dim, V = s.value_dim, v0 = blockIdx.y * 64 + 4 * c;
  const int64_t len = a.lengths ? min(max((int64_t)a.lengths[b], (int64_t)0), s.tokens) : s.tokens;
  const T* q = (const T*)a.q + b * s.q_batch_stride + h * s.q_head_stride;
  const T* k = (const T*)a.k + b * s.k_batch_stride + hk * s.k_head_stride;
  const T* v = (const T*)a.v + b * s.v_batch_stride + hk * s.v_head_stride;
  T* o = (T*)a.o + b * s.o_batch_stride + h * s.o_head_stride;
  const int64_t sbase = (int64_t)blockIdx.x * D * V;
  float S[R][4];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int d = g + 16 * r;
    const float* p = a.state_in + sbase + d * V + v0;
    if (VEC && a.state_in && d < D && v0 < V) {
      const floatx4 f = *(const floatx4*)p;
#pragma unroll
      for (int j = 0; j < 4; ++j) S[r][j] = f[j];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) S[r][j] = !VEC && a.state_in && d < D && v0 + j < V ? p[j] : 0.f;
    }
  }
  // lambda in two floats: it multiplies the state once a token, call after call
  const Decay64 lam = decay_pow(a.log_decay[h], 1);
  for (int64_t t = 0; t < len; ++t) {
    if (t) __syncthreads();
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
        S[r][j] = fmaf(S[r][j], lam.hi, fmaf(S[r][j], lam.lo, kd * vv[j]));
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
    for (int r = 0; r < R; ++r) {
      const int d = g + 16 * r;
      float* p = a.state_out + sbase + d * V + v0;
      if (VEC) {
        if (d < D && v0 < V) *(floatx4*)p = floatx4{S[r][0], S[r][1], S[r][2], S[r][3]};
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (d < D && v0 + j < V) p[j] = S[r][j];
      }
    }
  }
}

// ---- chunks -------------------------------------------------------------------
// LDS: two buffers of k (and q), one of v, which goes to registers first thing.
template <class E, int DP_, int NV_, bool OUT>
struct Chunk {
  static constexpr int DP = DP_, NV = NV_, VP = 32 * NV_;  // padded head and value width; a wave per 32 values
  static constexpr int DT = DP / 32;
  static constexpr int KB = kChunk * DP * 2, VB = kChunk * VP * 2;
  static constexpr int STAGE = (OUT ? 2 : 1) * KB;  // k, then q
  static constexpr int VOFF = 2 * STAGE, LDS = 2 * STAGE + VB;
  static constexpr uint32_t INF = __is_same(E, F16) ? 0x7c00 : 0x7f80;
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
  } else if (DMA) {
    int ln = lane;
    asm volatile("" : "+v"(ln));  // seldom taken: nothing of it is kept in registers from chunk to chunk
    const int r1 = ln / U, u1 = unit_slot<W>(r1, ln % U);
#pragma unroll
    for (int i0 = 0; i0 < LOADS / NW; ++i0) {
      const int i = wave + NW * i0, u = u1 ^ unit_slot<W>(R * i, 0);
      const char* p = rows + r1 * stride * 2 + 16 * u;
      const bool in = R * i + r1 >= pad && 8 * u < d;
      dma16(in ? (const void*)p : (const void*)decay_zero16, lds + 1024 * i);
      rows += step;
    }
  } else {
    // through registers: the loads of whole units hang on no condition (what has
    // none reads zeros), so that four are on their way at a time
    constexpr int N = LOADS / NW < 4 ? LOADS / NW : 4;
#pragma unroll
    for (int j = 0; j < LOADS / NW; j += N) {
      V8 v[N];
      const char* p[N];
      bool in[N];
#pragma unroll
      for (int x = 0; x < N; ++x) {
        const int i = wave + NW * (j + x), u = u0 ^ unit_slot<W>(R * i, 0);
        p[x] = rows + r0 * stride * 2 + 16 * u;
        in[x] = R * i + r0 >= pad && 8 * u < d;
        const void* from = in[x] && 8 * u + 8 <= d ? (const void*)p[x] : (const void*)decay_zero16;
        __builtin_memcpy(&v[x], from, 16);
        rows += step;
      }
      if (d & 7) {  // the last unit of a row, element by element
#pragma unroll
        for (int x = 0; x < N; ++x) {
          const int i = wave + NW * (j + x), u = u0 ^ unit_slot<W>(R * i, 0);
          const bool part = in[x] && 8 * u + 8 > d;
          const uint16_t* from = (const uint16_t*)(part ? (const void*)p[x] : (const void*)decay_zero16);
          const int top = part ? d - 8 * u - 1 : 0;
          uint32_t el[7];
#pragma unroll
          for (int e = 0; e < 7; ++e) el[e] = from[min(e, top)];
#pragma unroll
          for (int e = 0; e < 7; ++e) {
            asm volatile("" : "+v"(el[e]));  // or the load would move behind the condition
            if (part && e <= top) v[x][e] = __builtin_bit_cast(typename E::T, (uint16_t)el[e]);
          }
        }
      }
#pragma unroll
      for (int x = 0; x < N; ++x) *(V8*)(lds + 1024 * (wave + NW * (j + x)) + 16 * lane) = v[x];
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

// max over a lane and the other of its column, l ^ 32, of a value >= 0 that is no NaN (its bits order it)
__device__ __forceinline__ float half_max(float f) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(f), __float_as_uint(f), false, false);
  return __uint_as_float(max(a[0], a[1]));
}
// max over all lanes
__device__ __forceinline__ float wave_max(float f) {
  uint32_t v = __float_as_uint(f);
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(b[0], b[1]);
#define NC_ROR(N) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xf, 0xf, false));
  NC_ROR(8) NC_ROR(4) NC_ROR(2) NC_ROR(1)
#undef NC_ROR
  return __uint_as_float(__builtin_amdgcn_readfirstlane(v));
}
template <class V8>
__device__ __forceinline__ uint32_t max_bits(const V8 (&v)[4]) {  // of 16-bit magnitudes
  typedef unsigned short US8 __attribute__((ext_vector_type(8)));
  typedef unsigned short US2 __attribute__((ext_vector_type(2)));
  US8 u[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) u[x] = __builtin_bit_cast(US8, v[x]) & (unsigned short)0x7fff;
  const US8 w = __builtin_elementwise_max(__builtin_elementwise_max(u[0], u[1]), __builtin_elementwise_max(u[2], u[3]));
  const US2 m = __builtin_elementwise_max(__builtin_elementwise_max(w.s01, w.s23), __builtin_elementwise_max(w.s45, w.s67));
  return max((uint32_t)m.x, (uint32_t)m.y);
}
// max(m, |a|, |b|), NaN ignored
__device__ __forceinline__ float max3_abs(float m, float a, float b) {
  asm("v_max3_f32 %0, %0, |%1|, |%2|" : "+v"(m) : "v"(a), "v"(b));
  return m;
}
__device__ __forceinline__ float max_abs(const floatx16& v) {
  float m[4];  // four chains
#pragma unroll
  for (int r = 0; r < 4; ++r) m[r] = max3_abs(fabsf(v[4 * r]), v[4 * r + 1], v[4 * r + 2]);
  m[0] = max3_abs(m[0], v[3], v[7]);
  m[1] = max3_abs(m[1], v[11], v[15]);
  return max3_abs(max3_abs(m[0], m[1], m[2]), m[3], 0.f);
}
__device__ __forceinline__ float max_finite(float m, const floatx16& v) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
    if (fabsf(v[r]) < __builtin_huge_valf()) m = fmaxf(m, fabsf(v[r]));
  return m;
}

// Operands.  Scores, the state and weighted values are fp32; MFMA operands have 16
// bits.  They go in as sums of 16-bit terms, each the rest of the one before: two
// hold 22 bits in fp16 and 16 in bf16, where an output keeps 11 and 8, so that the
// outputs' own rounding is the only one that counts.  With one term, as many bits as
// the output, the outputs err 1.4 times as much as their rounding, for 0.88 to 1.1 times
// the time (130,560 tokens of 16 heads of 128 x 128: 536 us for the last pass, 591 with two).
template <class E>
__device__ __forceinline__ void two_terms(const float (&x)[8], float u, typename E::V8& hi, typename E::V8& lo) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const float a = x[i] * u, b = x[i + 1] * u;  // u a power of two: exact, however often it is formed
    typename E::V2 h;
    if (__is_same(E, F16))
      h = {(typename E::T)a, (typename E::T)b};
    else  // bf16 has no unit: the upper halves, which no value close to the end of fp32 rounds up to infinity
      h = __builtin_bit_cast(typename E::V2, __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u));
    asm("" : "+v"(h));  // or each half would be formed anew for its rest
    const typename E::V2 l = {(typename E::T)(a - (float)h.x), (typename E::T)(b - (float)h.y)};
    hi[i] = h.x;
    hi[i + 1] = h.y;
    lo[i] = l.x;
    lo[i + 1] = l.y;
  }
}

// Units.  What becomes an fp16 operand is held in a power-of-two unit, so that
// neither large nor small magnitudes leave the range in which its terms have
// their bits.
// The unit in which m >= 0 is in [2^14, 2^15), and its inverse; m below 2^-112, zero
// too, counts as 2^-112.
struct Fresh {
  float u, inv;
};
__device__ __forceinline__ Fresh fresh_unit(float m) {
  const uint32_t e = max(__float_as_uint(m) >> 23, 15u);  // m >= 0: 15 .. 255
  return {__uint_as_float((268u - e) << 23), __uint_as_float((e - 14u) << 23)};
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
__global__ __launch_bounds__(64 * NV) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_tok_decay_chunk(SegArgs sa) {
  typedef Chunk<E, DP, NV, OUT> C;
  typedef typename E::T T;
  typedef typename E::V8 V8;
  typedef typename E::V4 V4;
  constexpr bool F = __is_same(E, F16);
  constexpr int DT = C::DT, VP = C::VP, NT = F ? 2 : 3;  // NT: 16-bit terms of a weighted value
  __shared__ __align__(1024) char lds[C::LDS];
  const DecayArgs& a = sa.a;
  const ncodec_decay_shape& s = a.s;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, l32 = lane & 31;
  const int nsg = OUT ? sa.nseg : sa.nseg - 1;
  const int64_t bh = blockIdx.x / nsg;
  const int seg = blockIdx.x % nsg;
  const uint32_t b = (uint32_t)bh / (uint32_t)s.heads, hd = (uint32_t)bh - b * s.heads,
                 hk = hd / ((uint32_t)s.heads / (uint32_t)s.kv_heads);  // batch * heads < 2^24
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

  // A last chunk of n < 64 tokens sits at the end of its tile, behind 64 - n rows of
  // zeros: the ages and lags of its rows are then those of a full chunk.
  const int nch = tend > t0 ? (int)((tend - t0 + kChunk - 1) / kChunk) : 0;
  const int last_pad = (int)((int64_t)nch * kChunk - (tend - t0));  // of the last chunk
  const int64_t ks = s.k_token_stride, qs = s.q_token_stride, vs = s.v_token_stride;
  const T *kp = k + t0 * ks, *qp = q + t0 * qs, *vp = v + t0 * vs;  // of the chunk to be staged next
  auto stage_kq = [&](int c) {
    const int pad = c + 1 == nch ? last_pad : 0;
    char* base = lds + (c & 1) * C::STAGE;
    stage_rows<E, DP, NV, DMA>(base, kp - pad * ks, ks, pad, D, wave, lane);
    kp += kChunk * ks;
    if (OUT) {
      stage_rows<E, DP, NV, DMA>(base + C::KB, qp - pad * qs, qs, pad, D, wave, lane);
      qp += kChunk * qs;
    }
  };
  auto stage_v = [&](int c) {
    const int pad = c + 1 == nch ? last_pad : 0;
    stage_rows<E, VP, NV, DMA>(lds + C::VOFF, vp - pad * vs, vs, pad, V, wave, lane);
    vp += kChunk * vs;
  };
  // The state's loads before the tiles': behind those they would stand in the queue.
  const float log_decay = a.log_decay[hd];
  const float l2 = log2_decay(log_decay);
  floatx16 S[DT];
  // With segments the scan has put the state before each into the workspace, the
  // caller's too: state_out, which may be the same memory, is written while other
  // segments still begin.
  const float* sin = !OUT ? nullptr
                     : sa.nseg > 1 ? (const float*)a.ws + (bh * sa.nseg + seg) * sdv
                     : a.state_in  ? a.state_in + bh * sdv
                                   : nullptr;
#pragma unroll
  for (int x = 0; x < DT; ++x)
#pragma unroll
    for (int r = 0; r < 16; ++r) S[x][r] = 0.f;
  if (sin) {  // from inside the state whatever the padding, so that no load hangs on a condition
    const float* from = sin + min(col, V - 1);
#pragma unroll
    for (int x = 0; x < DT; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int d = 32 * x + 16 * (r >> 3) + 8 * h + (r & 7);
        S[x][r] = from[min(d, D - 1) * V];
      }
  }
  if (nch) {
    stage_v(0);
    stage_kq(0);
  }

  float* sout = !OUT ? (float*)a.ws + (bh * sa.nseg + seg + 1) * sdv
                : a.state_out && t0 + SL >= len ? a.state_out + bh * sdv : nullptr;

  // Decays.  Inside a diagonal 32 x 32 tile lambda^(i - j) for j <= i (i this lane's
  // token, j the register's).  At the end of a chunk token 16 x + j counts
  // lambda^(15 - j) lambda^(48 - 16 x).  One tile below the diagonal lambda^(32 + i - j)
  // is lambda^(i + 1) lambda^(31 - j), whose second factor is that age again.
  float mdiag[OUT ? 16 : 1], wage[8], wstep[4];
  uint32_t below = 0;  // bit r: j <= i
  if (OUT) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int lag = l32 - drow(r, h);
      below |= lag >= 0 ? 1u << r : 0u;
      mdiag[r] = __builtin_amdgcn_exp2f(max(lag, 0) * l2);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) wage[e] = __builtin_amdgcn_exp2f((15 - (8 * (e >> 2) + 4 * h + (e & 3))) * l2);
#pragma unroll
  for (int x = 0; x < 4; ++x) wstep[x] = __builtin_amdgcn_exp2f((48 - 16 * x) * l2);
  const float di0 = __builtin_amdgcn_exp2f((l32 + 1) * l2), di16 = __builtin_amdgcn_exp2f((l32 + 17) * l2),
              d32 = __builtin_amdgcn_exp2f(32 * l2);
  Decay64 keep = decay_pow(log_decay, kChunk), keep_last = keep;
  if (last_pad) keep_last = decay_pow(log_decay, kChunk - last_pad);
  T* op = o + (t0 + l32) * s.o_token_stride + 32 * wave + 8 * h;  // this lane's first output row
  const int64_t ostep = 32 * s.o_token_stride;
  const int ro = row_offset<DP>(lane);
  const int ck0 = col_offset<DP, true>(lane, 0), ck1 = col_offset<DP, true>(lane, 1);
  const char *pv0 = lds + C::VOFF + (col_offset<VP, false>(lane, 0) ^ (64 * wave)),
             *pv1 = lds + C::VOFF + (col_offset<VP, false>(lane, 1) ^ (64 * wave));
  // what rounding lambda^n to its hi part leaves out of a state, relative to it
  const float rest = keep.hi > 0.f ? keep.lo / keep.hi : 0.f;
  const float rest_last = keep_last.hi > 0.f ? keep_last.lo / keep_last.hi : 0.f;
  float owed = 0.f;
  auto settle = [&]() {
#pragma unroll
    for (int x = 0; x < DT; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) S[x][r] = fmaf(S[x][r], owed, S[x][r]);
    owed = 0.f;
  };
  if (sin) {
    const bool whole = D == DP && V == VP;
#pragma unroll
    for (int x = 0; x < DT; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        asm volatile("" : "+v"(S[x][r]));  // or the load would move behind the condition
        const int d = 32 * x + 16 * (r >> 3) + 8 * h + (r & 7);
        S[x][r] = whole || (d < D && col < V) ? S[x][r] : 0.f;  // zeros in the padding
      }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  for (int c = 0; c < nch; ++c) {
    // every wave's loads of chunk c have landed (each waited for its own), and
    // every wave is done with the other buffer
    lds_barrier();
    if (c + 1 < nch) stage_kq(c + 1);
    const int buf = (c & 1) * C::STAGE;
    const int pad = c + 1 == nch ? last_pad : 0;
    if (pad) {
      keep = keep_last;
      op -= pad * s.o_token_stride;
    }

    V8 vf[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) vf[x] = read_cols<E>(pv0 + 32 * VP * x, pv1 + 32 * VP * x);
    lds_barrier();  // v is in registers: its buffer takes the next chunk's
    if (c + 1 < nch) stage_v(c + 1);

    int bad = kChunk;  // first row of this lane's column that is not finite
    const bool any_bad = __any(max_bits(vf) >= C::INF);  // bits order finite values, infinities and NaN
    if (any_bad) {
      // a product would carry it to earlier tokens too (0 times NaN): it is taken
      // out here and put into the outputs and the state that it reaches
      int h4 = 4 * h;
      asm volatile("" : "+v"(h4));  // nothing of this rare path is computed, and kept, before the loop
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t u = (uint32_t)__builtin_bit_cast(uint16_t, (T)vf[x][e]) & 0x7fffu;
          if (u >= C::INF) {
            bad = min(bad, 16 * x + 8 * (e >> 2) + h4 + (e & 3));
            vf[x][e] = (T)0.f;
          }
        }
      bad = min(bad, __shfl_xor(bad, 32, 64));
    }

    if (OUT) {
      // The state's operand has one unit for the wave's columns, whose largest magnitude
      // it follows: an element keeps 22 bits, or those above 2^-39 of that magnitude.
      Fresh us = {1.f, 1.f};
      if (F) {
        float m = max_abs(S[0]);
#pragma unroll
        for (int x = 1; x < DT; ++x) m = fmaxf(m, max_abs(S[x]));
        if (__any(m == __builtin_huge_valf())) {  // the finite ones keep their unit
          m = 0.f;
#pragma unroll
          for (int x = 0; x < DT; ++x) m = max_finite(m, S[x]);
        }
        us = fresh_unit(wave_max(m));
      }
      // Products of the 64 queries with the state, and the scores: keys against queries
      // in the tiles (0, 0), (0, 1) and (1, 1), p holds k_j . q_i.
      floatx16 inter2[2] = {}, p[3] = {};
#pragma unroll
      for (int x = 0; x < 2 * DT; ++x) {
        const char* r = lds + ((ro + buf) ^ (32 * x));
        const V8 k0 = *(const V8*)r, k1 = *(const V8*)(r + 64 * DP);
        const V8 q0 = *(const V8*)(r + C::KB), q1 = *(const V8*)(r + (C::KB + 64 * DP));
        p[0] = E::mfma(k0, q0, p[0]);
        p[1] = E::mfma(k0, q1, p[1]);
        p[2] = E::mfma(k1, q1, p[2]);
        V8 sh, sl;
        float part[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) part[e] = S[x >> 1][8 * (x & 1) + e];
        two_terms<E>(part, us.u, sh, sl);
        inter2[0] = E::mfma(sh, q0, inter2[0]);
        inter2[1] = E::mfma(sh, q1, inter2[1]);
        inter2[0] = E::mfma(sl, q0, inter2[0]);
        inter2[1] = E::mfma(sl, q1, inter2[1]);
      }
#pragma unroll
      for (int it = 0; it < 2; ++it) {  // 32 queries
        floatx16 &inter = inter2[it], intra = {}, &diag = p[2 * it], &below0 = p[1];
        // weighted scores: pairs above the diagonal count nothing, whatever their product is
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          diag[r] = __int_as_float(__float_as_int(diag[r]) & ((int)(below << (31 - r)) >> 31)) * mdiag[r];
          if (it) below0[r] *= wage[r & 7] * (r < 8 ? di16 : di0);
        }
        Fresh up = {1.f, 1.f};  // of this lane's query
        if (F) {
          float m = max_abs(diag);
          if (it) m = fmaxf(m, max_abs(below0));
          up = fresh_unit(half_max(m));
        }
        const auto add_values = [&](const floatx16& w, int x) {  // values 16 x .. 16 x + 31
          V8 wh[2], wl[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float part[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) part[e] = w[8 * y + e];
            two_terms<E>(part, up.u, wh[y], wl[y]);
          }
          intra = E::mfma(vf[x], wl[0], intra);
          intra = E::mfma(vf[x + 1], wl[1], intra);
          intra = E::mfma(vf[x], wh[0], intra);
          intra = E::mfma(vf[x + 1], wh[1], intra);
        };
        if (it) add_values(below0, 0);
        add_values(diag, 2 * it);
        // row i is token i - pad of the chunk; rows of the padding are not stored
        float di = it ? di0 * d32 : di0;
        if (pad) di = __builtin_amdgcn_exp2f(max(32 * it + l32 + 1 - pad, 0) * l2);
        const float ci = s.scale * di * us.inv, cp = s.scale * up.inv;
#pragma unroll
        for (int r = 0; r < 16; ++r) inter[r] = fmaf(inter[r], ci, intra[r] * cp);
        if (any_bad) {
          int h2 = h;
          asm volatile("" : "+v"(h2));
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (32 * it + l32 >= __shfl(bad, drow(r, h2), 64)) inter[r] = __builtin_nanf("");
        }
        // a lane has four consecutive values eight times, its neighbour l ^ 32 the
        // four after them: exchanged, each has eight, a 16-byte unit of the row
        const bool row_in = 32 * it + l32 >= pad;
        T* row = op;
        op += ostep;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          V4 lo, hi;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            lo[j] = (T)inter[8 * g + j];
            hi[j] = (T)inter[8 * g + 4 + j];
          }
          typedef uint32_t U2 __attribute__((ext_vector_type(2)));
          typedef uint32_t U4 __attribute__((ext_vector_type(4)));
          const U2 x = __builtin_bit_cast(U2, lo), y = __builtin_bit_cast(U2, hi);
          const auto w0 = __builtin_amdgcn_permlane32_swap(x.x, y.x, false, false);
          const auto w1 = __builtin_amdgcn_permlane32_swap(x.y, y.y, false, false);
          const U4 w = {w0[0], w1[0], w0[1], w1[1]};
          const int left = V - (32 * wave + 16 * g + 8 * h);
          if (row_in && left > 0) {
            if (left >= 8) {
              __builtin_memcpy(row + 16 * g, &w, 16);
            } else {
              const V8 z = __builtin_bit_cast(V8, w);
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (e < left) row[16 * g + e] = z[e];
            }
          }
        }
      }
    }

    if (!OUT || c + 1 < nch || sout) {
      // the state: v weighted by its age, as a sum of 16-bit terms that holds 22 (fp16)
      // or 24 (bf16) bits, because the state is an fp32 output.  fp16 terms are in a unit
      // of this lane's column, from its largest weighted value: a quiet column keeps its
      // bits beside a loud one, and a late value behind a loud one that has decayed.
      float w[4][8];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        float ws = wstep[x];
        asm volatile("" : "+v"(ws));  // or the 32 weights would be formed, and kept, before the loop
#pragma unroll
        for (int e = 0; e < 8; ++e) w[x][e] = fmaf((float)vf[x][e], wage[e] * ws, 0.f);
      }
      Fresh uv = {1.f, 1.f};
      if (F) {
        float m[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          m[x] = max3_abs(fabsf(w[x][0]), w[x][1], w[x][2]);
          m[x] = max3_abs(max3_abs(m[x], w[x][3], w[x][4]), w[x][5], w[x][6]);
        }
        m[0] = max3_abs(max3_abs(m[0], w[0][7], w[1][7]), w[2][7], w[3][7]);
        m[0] = fmaxf(max3_abs(m[0], m[1], m[2]), m[3]);
        uv = fresh_unit(half_max(m[0]));
      }
      V8 term[4][NT];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        two_terms<E>(w[x], uv.u, term[x][0], term[x][1]);
        if (!F) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            term[x][NT - 1][e] = (T)(w[x][e] - (float)term[x][0][e] - (float)term[x][1][e]);
        }
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const char *p0 = lds + ((ck0 + buf) ^ (64 * d)), *p1 = lds + ((ck1 + buf) ^ (64 * d));
        floatx16 add = {};
        V8 kf[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) kf[x] = read_cols<E>(p0 + 32 * DP * x, p1 + 32 * DP * x);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int y = NT - 1; y >= 0; --y) add = E::mfma(kf[x], term[x][y], add);
#pragma unroll
        for (int r = 0; r < 16; ++r) S[d][r] = F ? fmaf(add[r], uv.inv, S[d][r] * keep.hi) : fmaf(S[d][r], keep.hi, add[r]);
      }
      // made up for every sixteenth chunk
      owed += pad ? rest_last : rest;
      if ((c & 15) == 15) settle();
      if (any_bad) {
        asm volatile("");  // a branch, not a select for each register
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) S[d][r] = bad < kChunk ? __builtin_nanf("") : S[d][r];
      }
    }
    // this wave's part of the next chunk has landed (and its stores, long sent)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }

  if (sout) {
    if (nch) settle();  // without tokens the state stands still, an infinity in it too
    sout += col;
    if (D == DP && V == VP) {
#pragma unroll
      for (int x = 0; x < DT; ++x)
#pragma unroll
        for (int r = 0; r < 16; ++r) sout[(32 * x + 16 * (r >> 3) + 8 * h + (r & 7)) * VP] = S[x][r];
    } else if (col < V) {
#pragma unroll
      for (int x = 0; x < DT; ++x)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int d = 32 * x + 16 * (r >> 3) + 8 * h + (r & 7);
          if (d < D) sout[d * V] = S[x][r];
        }
    }
  }
}

// Over the segments of a sequence and head: slot g + 1, what segment g adds, becomes
// the state before segment g + 1; slot 0 the state before the first.  A workgroup
// has 64 VEC elements of the state and a wave for every M segments (eight at
// most): wave j takes segments j M .. j M + M - 1, all its loads in flight, first alone,
// then from the state that the waves before it give.  VEC: 4 where the state is a
// multiple of 4, which also forms the decays (64-bit exponentials) for four elements
// at a time.  16 heads of 128 x 128 in 32 segments, 67 MB read and written: 13.8 us (4.9
// TB/s), 16.3 in single elements.
constexpr int kScanM = 8;
template <int VEC>
__global__ __launch_bounds__(512) void k_tok_decay_scan(SegArgs sa) {
  typedef float FV __attribute__((ext_vector_type(VEC)));
  __shared__ FV part[8][64];
  const DecayArgs& a = sa.a;
  const ncodec_decay_shape& s = a.s;
  const int64_t sdv = (int64_t)s.head_dim * s.value_dim;
  const int blocks = (int)((sdv + 64 * VEC - 1) / (64 * VEC));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const uint32_t bh = blockIdx.x / blocks, b = bh / (uint32_t)s.heads;
  const int64_t e = ((int64_t)(blockIdx.x % blocks) * 64 + lane) * VEC;
  const bool in = e < sdv;
  const int64_t len = a.lengths ? min(max((int64_t)a.lengths[b], (int64_t)0), s.tokens) : s.tokens;
  const int64_t SL = (int64_t)sa.seg_chunks * kChunk;
  const int last = (int)min((len + SL - 1) / SL, (int64_t)sa.nseg) - 1;  // segments 0 .. last have tokens
  float* ws = (float*)a.ws + (int64_t)bh * sa.nseg * sdv + (in ? e : 0);
  FV S = {};
  if (in && a.state_in) __builtin_memcpy(&S, a.state_in + bh * sdv + e, sizeof(FV));
  if (in && wave == 0) *(FV*)ws = S;
  const float ld = a.log_decay[bh % (uint32_t)s.heads];
  const Decay64 keep = decay_pow(ld, SL), all = decay_pow(ld, kScanM * SL);
  const auto step = [](FV x, const Decay64& f, FV add) { return x * f.hi + (x * f.lo + add); };
  for (int g0 = 0; g0 < last; g0 += waves * kScanM) {
    const int first = g0 + wave * kScanM;
    FV add[kScanM], mine = {};
#pragma unroll
    for (int i = 0; i < kScanM; ++i) add[i] = first + i < last ? *(const FV*)(ws + (first + i + 1) * sdv) : FV{};
#pragma unroll
    for (int i = 0; i < kScanM; ++i) mine = step(mine, keep, add[i]);
    part[wave][lane] = mine;
    __syncthreads();
    FV P = S;
    for (int j = 0; j < waves; ++j) {
      if (j == wave) P = S;
      S = step(S, all, part[j][lane]);
    }
#pragma unroll
    for (int i = 0; i < kScanM; ++i) {
      P = step(P, keep, add[i]);
      if (in && first + i < last) *(FV*)(ws + (first + i + 1) * sdv) = P;
    }
    __syncthreads();
  }
}

DecayPlan plan_of(const ncodec_decay_shape& s) { return decay_rule(s.batch * s.heads, s.tokens, s.value_dim); }

template <class E, bool VEC>
hipError_t recur(const DecayArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.s.batch * a.s.heads), (unsigned)((a.s.value_dim + 63) / 64));
  if (a.s.head_dim <= 32)
    launch(k_tok_decay_recur<E, 2, VEC>, grid, dim3(256), st, a);
  else if (a.s.head_dim <= 64)
    launch(k_tok_decay_recur<E, 4, VEC>, grid, dim3(256), st, a);
  else
    launch(k_tok_decay_recur<E, 8, VEC>, grid, dim3(256), st, a);
  return hipGetLastError();
}

template <class E, int DP, int NV, bool DMA>
hipError_t chunked(const SegArgs& sa, hipStream_t st) {
  const ncodec_decay_shape& s = sa.a.s;
  const int64_t bh = s.batch * s.heads;
  if (sa.nseg > 1) {
    launch(k_tok_decay_chunk<E, DP, NV, false, DMA>, dim3((unsigned)(bh * (sa.nseg - 1))), dim3(64 * NV), st, sa);
    const int64_t sdv = (int64_t)s.head_dim * s.value_dim;
    const unsigned waves = (unsigned)std::min(8, (sa.nseg - 2) / kScanM + 1);
    if (sdv % 4 == 0)
      launch(k_tok_decay_scan<4>, dim3((unsigned)(bh * ((sdv + 255) / 256))), dim3(64 * waves), st, sa);
    else
      launch(k_tok_decay_scan<1>, dim3((unsigned)(bh * ((sdv + 63) / 64))), dim3(64 * waves), st, sa);
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
  const DecayPlan p = plan_of(s);
  if (!p.chunked) {
    const bool vec = s.value_dim % 4 == 0 && (uintptr_t)a.state_in % 16 == 0 && (uintptr_t)a.state_out % 16 == 0;
    return vec ? recur<E, true>(a, st) : recur<E, false>(a, st);
  }
  const auto direct = [](const void* x, int64_t batch, int64_t token, int64_t head) {
    return (uintptr_t)x % 16 == 0 && batch % 8 == 0 && token % 8 == 0 && head % 8 == 0 && token < (1 << 26);
  };
  // Straight to LDS where rows are whole 16-byte units, through registers otherwise (8,160
  // tokens of 8 heads of 64 x 64 33.1 us, 35.8 through registers; 130,560 of 16 heads of 128 x
  // 128, one head's tokens next to each other, 832 and 935).
  const bool dma = s.head_dim % 8 == 0 && s.value_dim % 8 == 0 &&
                   direct(a.q, s.q_batch_stride, s.q_token_stride, s.q_head_stride) &&
                   direct(a.k, s.k_batch_stride, s.k_token_stride, s.k_head_stride) &&
                   direct(a.v, s.v_batch_stride, s.v_token_stride, s.v_head_stride);
  const SegArgs sa{a, p.seg_chunks, p.nseg};
  return dma ? by_dim<E, true>(sa, st) : by_dim<E, false>(sa, st);
}

}  // namespace

size_t decay_workspace_bytes(const ncodec_decay_shape& s) {
  const DecayPlan p = plan_of(s);
  if (p.nseg == 1) return 0;
  return (size_t)(s.batch * s.heads) * (size_t)p.nseg * (size_t)(s.head_dim * s.value_dim) * 4;
}

hipError_t launch_decay_attention(const DecayArgs& a, hipStream_t st) {
  return a.s.dtype == NCODEC_DTYPE_FP16 ? run<F16>(a, st) : run<BF16>(a, st);
}

}  // namespace nc
