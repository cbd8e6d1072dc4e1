// Softmax attention with a sliding window and sinks over whole sequences:
//   o_i = sum_j p_ij v_j over the tokens j that token i sees, p = softmax(scale q_i . k_j).
//
// One pass over the keys with a running maximum and sum.  Both products are MFMAs,
// transposed: scores^T = K q^T with keys as rows and queries as columns, so that a lane
// holds half of one query's scores and its maximum, sum and rescaling are the lane's own;
// and outputs^T = V^T p^T, whose operand p the accumulators of the scores already are, in
// the order of keys that a transposed read of V from LDS gives.  Weights enter that product
// as two 16-bit terms each (22 bits in fp16, 17 in bf16): with one, as many bits as the output,
// the outputs err 1.4 times as much as their rounding, for 0.74 to 0.85 of the time.
//
// A workgroup's four waves share tiles of 64 keys and values in LDS, 32 queries a wave: of
// four heads of a group, or of one.  What bounds it is a wave's own sequence of scores,
// weights and outputs, of which the other wave of the SIMD hides a part: 32,640 tokens of 16
// heads over 4 of 128 x 128, 8,160 in sight, bf16, 2.0 TFLOP: 2.4 to 2.7 ms (0.8 PFLOP/s, 1.2
// with the second terms, which is what the library's large product reaches; MFMAs run 64 % of the
// CUs' busy time, VALU issues 56 %); 8,160 tokens of 8 heads of 64 x 64, 4,080 in sight, fp16: 107 to
// 119 us (MFMAs 36 %, VALU 54 %); 8 ragged sequences of up to 1,560, 8 heads over 2 of 64 x 96: 35 to 37 us
// (39 as a kernel by itself; MFMAs 23 %, VALU 45 %).
// Tried and no faster there: the next tile's scores beside the weights of this one, weights and
// products of 16 keys in turn, 64 queries a wave, three waves a SIMD, two or eight waves a workgroup.
#include <algorithm>

#include "tok_attend.hpp"
#include "tok_tiles.hpp"
#include "token_rules.hpp"

namespace nc {
namespace {

constexpr int kTile = 64;     // keys
constexpr int kQueries = 32;  // of a wave
constexpr int kWaves = 4;

struct WindowRun {
  WindowArgs a;
  int64_t first;     // block of this launch's first workgroup
  int head_waves;    // waves of a workgroup on different heads of a group; the others on further queries
  int head_tiles;    // workgroups for a group's heads
  int query_blocks;  // of a sequence
  bool q_runs;       // queries are whole 16-byte runs
};

__device__ __align__(16) uint32_t window_zero16[4];

// Stage kTile rows of d elements from `base` into an LDS tile of W wide rows; rows from
// `rows` on and elements past d are zero.  DMA: direct loads, which the caller waits for;
// rows are then 16-byte aligned and their stride is below 2^26.
template <class E, int W, bool DMA>
__device__ __forceinline__ void stage_tile(char* lds, const typename E::T* base, int64_t stride, int rows, int d, int wave,
                                           int lane) {
  typedef typename E::V8 V8;
  constexpr int U = W / 8, R = 64 / U, LOADS = kTile / R / kWaves;
  const int r0 = lane / U, u0 = unit_slot<W>(r0, lane % U);
  const char* from = (const char*)(base + (int64_t)(R * wave) * stride);
  const int64_t step = (int64_t)(R * kWaves) * stride * 2;
  if (DMA && rows >= kTile && d == W) {
    const uint32_t voff = (uint32_t)r0 * (uint32_t)stride * 2u;
#pragma unroll
    for (int x = 0; x < LOADS; ++x) {
      const int i = wave + kWaves * x;
      dma16s(from, voff + 16 * (u0 ^ unit_slot<W>(R * i, 0)), lds + 1024 * i);
      from += step;
    }
  } else {
#pragma unroll
    for (int x = 0; x < LOADS; ++x) {
      const int i = wave + kWaves * x, u = u0 ^ unit_slot<W>(R * i, 0);
      const char* p = from + r0 * stride * 2 + 16 * u;
      const bool in = R * i + r0 < rows && 8 * u < d;
      if (DMA) {
        dma16(in ? (const void*)p : (const void*)window_zero16, lds + 1024 * i);
      } else {
        V8 v = {};
        if (in) {
          const int left = d - 8 * u;
          const typename E::T* e = (const typename E::T*)p;
          if (left >= 8)
            __builtin_memcpy(&v, e, 16);
          else
#pragma unroll
            for (int y = 0; y < 8; ++y)
              if (y < left) v[y] = e[y];
        }
        *(V8*)(lds + 1024 * i + 16 * lane) = v;
      }
      from += step;
    }
  }
}

// Eight weights as two 16-bit terms (as two_terms(), in fewer steps: the rest of an fp16 term
// is formed and rounded in one instruction, a multiply-add of mixed types).
__device__ __forceinline__ void weight_terms(const float (&w)[8], half8& hi, half8& lo) {
  float minus = -1.f;
  asm("" : "+s"(minus));  // or the multiply-add would become a conversion and a subtraction
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    half2 x = {(f16)w[i], (f16)w[i + 1]};
    asm("" : "+v"(x));  // or each half would be formed anew for its rest
    hi[i] = x.x;
    hi[i + 1] = x.y;
    lo[i] = (f16)__builtin_fmaf((float)x.x, minus, w[i]);
    lo[i + 1] = (f16)__builtin_fmaf((float)x.y, minus, w[i + 1]);
  }
}
__device__ __forceinline__ void weight_terms(const float (&w)[8], bhalf8& hi, bhalf8& lo) { two_terms<BF16, true>(w, 1.f, hi, lo); }

template <class V8>
__device__ __forceinline__ bool any_not_finite(const V8 (&v)[4], uint32_t inf) {
  typedef unsigned short US8 __attribute__((ext_vector_type(8)));
  US8 m = __builtin_bit_cast(US8, v[0]) & (unsigned short)0x7fff;
#pragma unroll
  for (int x = 1; x < 4; ++x) m = __builtin_elementwise_max(m, __builtin_bit_cast(US8, v[x]) & (unsigned short)0x7fff);
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, (uint32_t)m[e]);
  return __any(top >= inf);
}

// DP: padded head width, NV: 32-column tiles of the values.  KS: tiles of a round, each for
// waves of its own, which join at the end.
template <class E, int DP, int NV, bool DMA, int KS>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2))) void k_tok_window(WindowRun run) {
  typedef typename E::T T;
  typedef typename E::V8 V8;
  typedef typename E::V4 V4;
  constexpr bool F = __is_same(E, F16);
  constexpr int VW = NV == 1 ? 32 : NV == 4 ? 128 : 64;  // LDS row of values; of 96 the last 32 in a tile of their own
  constexpr int KB = kTile * DP * 2, VB = kTile * VW * 2, STAGE = KB + kTile * NV * 64;
  constexpr uint32_t INF = F ? 0x7c00 : 0x7f80;
  // Weights are held at 2^off of the largest, which is let grow to 2^lag of that before the
  // outputs are rescaled.  fp16 terms stay below 2^15 and keep the bits above 2^-32 of the largest weight.  In
  // bf16 the values have fp32's range: weights add up to less than a half, 64 of 2^-8 at most to an eighth, and
  // beyond that all are taken down by 2^8, so that no sum leaves fp32 where the mean does not; and where one token
  // has all the weight, its value of 2^-126 ends above fp32's last bit.
  constexpr float off = F ? 7.f : -14.f, lag = F ? 8.f : 6.f, kFull = 0x1p-4f;
  // Scores whose product with c this large a number is would, rounded once for the base and not
  // at all in the weights, leave that room: they are multiplied first, and the largest is taken from them, which
  // then weighs 2^far_off.  In fp16 that is lower than off: one that is 2^15 larger by the unrounded product, up to
  // which no rise is looked for, may be 2^17 larger by the rounded one.
  constexpr float kLarge = 0x1p22f, kNothing = -0x1.fffffep127f, far_off = F ? -2.f : off;
  __shared__ __align__(1024) char lds[2 * KS * STAGE];
  const WindowArgs& a = run.a;
  const ncodec_window_shape& s = a.s;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, l32 = lane & 31;
  const int group = s.heads / s.kv_heads, D = s.head_dim, V = s.value_dim;
  // the last queries of all heads first: they see most
  const int64_t block = run.first + blockIdx.x, per = s.batch * s.kv_heads * run.head_tiles;
  const int qb = run.query_blocks - 1 - (int)(block / per);
  // Workgroups go to the eight XCDs in turn, and inside of one to its shader engines, in order: a
  // long sequence among short ones would sit on the same few for all of its queries, so its place
  // moves on by one XCD and one engine with each block of them (sixteen sequences of up to 1560, 8
  // heads over 2 of 64 x 96: 87 -> 47 us, 64 x 64: 72 -> 37).
  uint32_t at = (uint32_t)((block + (a.lengths ? 9 * (int64_t)qb : 0)) % per);
  const int ht = at % (uint32_t)run.head_tiles;
  at /= (uint32_t)run.head_tiles;
  const int hk = at % (uint32_t)s.kv_heads;
  const int64_t b = at / (uint32_t)s.kv_heads;
  const int ks = wave / (kWaves / KS), qwave = wave % (kWaves / KS);
  const int qw = kWaves / KS / run.head_waves;  // waves along the queries
  const int hd = hk * group + ht * run.head_waves + qwave % run.head_waves;
  const int64_t len = a.lengths ? min(max((int64_t)a.lengths[b], (int64_t)0), s.tokens) : s.tokens;
  const int i0 = qb * qw * kQueries;                                     // the workgroup's first query
  const int wi0 = i0 + qwave / run.head_waves * kQueries, i = wi0 + l32;  // the wave's, the lane's
  const int iend = (int)min((int64_t)i0 + qw * kQueries, len);           // behind its last one
  const int wend = (int)min((int64_t)wi0 + kQueries, len);

  T* o = (T*)a.o + b * s.o_batch_stride + (int64_t)i * s.o_token_stride + hd * s.o_head_stride;
  floatx16 out[NV];
#pragma unroll
  for (int x = 0; x < NV; ++x)
#pragma unroll
    for (int r = 0; r < 16; ++r) out[x][r] = 0.f;
  float sum = 0.f;

  if (i0 < iend) {
    const T* k = (const T*)a.k + b * s.k_batch_stride + hk * s.k_head_stride;
    const T* v = (const T*)a.v + b * s.v_batch_stride + hk * s.v_head_stride;
    const int window = s.window ? (int)s.window : 0x7fffffff, sinks = (int)s.sinks;
    const WindowTiles all_tiles = window_tiles(i0, qw * kQueries, len, (int)s.window, sinks);
    const int whole = all_tiles.whole, tiles = all_tiles.count;
    const auto key0 = [&](int t) { return all_tiles.key0(t); };
    const auto stage = [&](int t) {
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        if (t + x >= tiles) break;
        char* to = lds + ((t / KS & 1) * KS + x) * STAGE;
        const int j0 = key0(t + x), rows = (int)min((int64_t)kTile, len - j0);
        stage_tile<E, DP, DMA>(to, k + (int64_t)j0 * s.k_token_stride, s.k_token_stride, rows, D, wave, lane);
        stage_tile<E, VW, DMA>(to + KB, v + (int64_t)j0 * s.v_token_stride, s.v_token_stride, rows, min(V, VW), wave, lane);
        if (NV == 3)
          stage_tile<E, 32, DMA>(to + KB + VB, v + (int64_t)j0 * s.v_token_stride + 64, s.v_token_stride, rows, V - 64, wave, lane);
      }
    };
    stage(0);

    // the scale's sign goes into the queries, so that the largest product is the largest score
    const float c = s.scale == 0.f ? 1.f : fabsf(s.scale) * 1.44269504088896341f;
    V8 qf[DP / 16];
    {
      const T* q = (const T*)a.q + b * s.q_batch_stride + (int64_t)min(i, (int)len - 1) * s.q_token_stride + hd * s.q_head_stride;
#pragma unroll
      for (int x = 0; x < DP / 16; ++x) {
        const int d = 16 * x + 8 * h;
        V8 w = {};
        if (run.q_runs) {
          if (d < D) w = *(const V8*)(q + d);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (d + e < D) w[e] = q[d + e];
        }
        qf[x] = w;
      }
      if (s.scale <= 0.f) {
#pragma unroll
        for (int x = 0; x < DP / 16; ++x)
#pragma unroll
          for (int e = 0; e < 8; ++e) qf[x][e] = s.scale == 0.f ? (T)((float)qf[x][e] * 0.f) : (T)-qf[x][e];
      }
    }
    const int ro = row_offset<DP>(lane);
    const int pv0 = col_offset<VW, false>(lane, 0), pv1 = col_offset<VW, false>(lane, 1);
    const int pw0 = VB + col_offset<32, false>(lane, 0), pw1 = VB + col_offset<32, false>(lane, 1);
    // columns 32 y .. of values 16 x .. of a tile
    const auto columns = [&](const char* vt, int y, int x) {
      return NV == 3 && y == 2 ? read_cols<E>(vt + pw0 + 32 * 32 * x, vt + pw1 + 32 * 32 * x)
                               : read_cols<E>(vt + (pv0 ^ (64 * y)) + 32 * VW * x, vt + (pv1 ^ (64 * y)) + 32 * VW * x);
    };
    // a weight is 2^(score * c - base), of a lane whose query has large scores 2^((score * c - base) + far_off)
    float base = kNothing;
    bool far = false, large = false;  // has the lane's query, has any of the wave's large scores?
    float cl = c, less = 0.f;         // what follow() leaves: a weight is 2^(score * cl - less)

    // does any of the wave's queries see any of the tile's keys?
    const auto some = [&](int j0) { return j0 < wend && (j0 < sinks || wi0 - (j0 + kTile - 1) < window); };
    const auto scores = [&](const char* kt, floatx16(&p)[2]) {
      p[0] = p[1] = floatx16{};
      constexpr int N = DP / 16, A = 3;  // reads that many steps ahead
      V8 kf[N][2];
      const auto keys = [&](int x) {
        const char* r = kt + (ro ^ (32 * x));
        kf[x][0] = *(const V8*)r;
        kf[x][1] = *(const V8*)(r + 64 * DP);
      };
#pragma unroll
      for (int x = 0; x < A; ++x) keys(x);
#pragma unroll
      for (int x = 0; x < N; ++x) {
        if (x + A < N) keys(x + A);
        __builtin_amdgcn_sched_barrier(0);
        p[0] = E::mfma(kf[x][0], qf[x], p[0]);
        p[1] = E::mfma(kf[x][1], qf[x], p[1]);
      }
    };
    const auto rounded = [&](float f) {  // f c
      f *= c;
      asm("" : "+v"(f));  // no multiply-add
      return f;
    };
    // log2 of the weight of score f
    const auto power = [&](float f) { return far ? (rounded(f) - base) + far_off : fmaf(f, c, -base); };
    const auto follow = [&](floatx16(&p)[2]) {  // the base after the maximum
      float top = fmaxf(p[0][0], p[1][0]);
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(fmaxf(top, p[0][r]), p[1][r]);
      if (__any(fmaf(top, c, -base) > off + lag || (!F && sum > kFull))) {  // of large scores: at least where power() is
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        // each query by its own scores, whatever the wave's others are
        const bool rises = power(top) > off + lag, now = rises && !far && fabsf(top * c) >= kLarge;
        far = far || now;
        large = large || __any(now);
        float base1 = far ? rounded(top) : fmaf(top, c, -off);
        bool moves = rises;
        if (!F) {
          const auto su = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
          base1 = rises ? base1 : base + 8.f;
          moves = rises || __uint_as_float(su[0]) + __uint_as_float(su[1]) > kFull;
        }
        const float fade = moves ? __builtin_amdgcn_exp2f((base - base1) + (now ? far_off : 0.f)) : 1.f;
        base = moves ? base1 : base;
        sum *= fade;
#pragma unroll
        for (int x = 0; x < NV; ++x)
#pragma unroll
          for (int r = 0; r < 16; ++r) out[x][r] *= fade;
      }
      less = base;
      if (large) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          p[0][r] = power(p[0][r]);
          p[1][r] = power(p[1][r]);
        }
        cl = 1.f;
        less = 0.f;
      }
    };
    // weights of keys 16 x .. of a tile
    const auto weights = [&](const floatx16(&p)[2], int x, V8& hi, V8& lo) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = __builtin_amdgcn_exp2f(fmaf(p[x >> 1][8 * (x & 1) + e], cl, -less));
        sum += w[e];
      }
      weight_terms(w, hi, lo);
    };

#pragma unroll
    for (int x = 0; x < DP / 16; ++x) asm volatile("" : "+v"(qf[x]));  // here, not in the loop, are the queries waited for
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

    int t = 0;
    for (; t + KS <= whole; t += KS) {
      // every wave's loads of this round have landed (each waited for its own), and every
      // wave is done with the other buffer
      lds_barrier();
      if (t + KS < tiles) stage(t + KS);
      const char* kt = lds + ((t / KS & 1) * KS + ks) * STAGE;
      const char* vt = kt + KB;
      floatx16 cur[2];
      __builtin_amdgcn_s_setprio(1);
      scores(kt, cur);
      __builtin_amdgcn_s_setprio(0);
      follow(cur);
      V8 hi[4], lo[4], vf[2][4];
      const auto values = [&](int y) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
          vf[y & 1][x] = columns(vt, y, x);
      };
      values(0);
#pragma unroll
      for (int x = 0; x < 4; ++x) weights(cur, x, hi[x], lo[x]);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int y = 0; y < NV; ++y) {
        if (y + 1 < NV) values(y + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          out[y] = E::mfma(vf[y & 1][x], lo[x], out[y]);
          out[y] = E::mfma(vf[y & 1][x], hi[x], out[y]);
        }
      }
      __builtin_amdgcn_s_setprio(0);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    for (; t < tiles; t += KS) {
      lds_barrier();
      if (t + KS < tiles) stage(t + KS);
      const char* kt = lds + ((t / KS & 1) * KS + ks) * STAGE;
      const char* vt = kt + KB;
      const int j0 = key0(min(t + ks, tiles - 1));
      if (t + ks < tiles && some(j0)) {
        const bool all = j0 + kTile - 1 <= wi0 && (wi0 + kQueries - 1 - j0 < window || j0 + kTile <= sinks);
        floatx16 cur[2];
        __builtin_amdgcn_s_setprio(1);
        scores(kt, cur);
        __builtin_amdgcn_s_setprio(0);
        uint32_t seen[2] = {0xffffu, 0xffffu};
        if (!all) {
          int h0 = h, il = i;
          asm volatile("" : "+v"(h0), "+v"(il));  // nothing of this is computed, and kept, before the loop
          seen[0] = seen[1] = 0;
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int j = j0 + 32 * y + drow(r, h0), d = il - j;
              const bool in = (uint32_t)d < (uint32_t)window || (d >= 0 && j < sinks);
              seen[y] |= in ? 1u << r : 0u;
              cur[y][r] = in ? cur[y][r] : -__builtin_huge_valf();
            }
        }
        follow(cur);
        V8 hi[4], lo[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) weights(cur, x, hi[x], lo[x]);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int y = 0; y < NV; ++y) {
          V8 vf[4];
#pragma unroll
          for (int x = 0; x < 4; ++x)
            vf[x] = columns(vt, y, x);
          if (!all && any_not_finite(vf, INF)) {
            // a product would carry it to queries that do not see it too (0 times NaN): it is
            // taken out, and counted for those that do
            floatx16 hit = {};
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              V8 bad = {}, sees = {};
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const uint32_t u = (uint32_t)__builtin_bit_cast(uint16_t, (T)vf[x][e]) & 0x7fffu;
                bad[e] = u >= INF ? (T)1.f : (T)0.f;
                vf[x][e] = u >= INF ? (T)0.f : vf[x][e];
                sees[e] = seen[x >> 1] >> (8 * (x & 1) + e) & 1 ? (T)1.f : (T)0.f;
              }
              hit = E::mfma(bad, sees, hit);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) out[y][r] = hit[r] > 0.f ? __builtin_nanf("") : out[y][r];
          }
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            out[y] = E::mfma(vf[x], lo[x], out[y]);
            out[y] = E::mfma(vf[x], hi[x], out[y]);
          }
        }
      }
      __builtin_amdgcn_s_setprio(0);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    if (KS > 1) {
      // the second half's maximum, sum and outputs, lane by lane
      float* mine = (float*)lds + (qwave * 64 + lane) * 4;  // and 16 outputs at a time, 16 bytes a lane
      constexpr int STEP = kWaves / KS * 64 * 4;
      lds_barrier();
      if (ks) {
        *(floatx4*)mine = floatx4{base, sum, far ? 1.f : 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 4 * NV; ++x)
          *(floatx4*)(mine + (x + 1) * STEP) =
              floatx4{out[x / 4][x % 4 * 4], out[x / 4][x % 4 * 4 + 1], out[x / 4][x % 4 * 4 + 2], out[x / 4][x % 4 * 4 + 3]};
      }
      lds_barrier();
      if (ks) return;
      const floatx4 other = *(const floatx4*)mine;
      // by which power of two a weight of this half counts less than one of the other
      const float d = (other[0] - base) + far_off * ((far ? 1.f : 0.f) - other[2]);
      const float f0 = __builtin_amdgcn_exp2f(fminf(-d, 0.f)), f1 = __builtin_amdgcn_exp2f(fminf(d, 0.f));
      sum = sum * f0 + other[1] * f1;
#pragma unroll
      for (int x = 0; x < 4 * NV; ++x) {
        const floatx4 w = *(const floatx4*)(mine + (x + 1) * STEP);
#pragma unroll
        for (int e = 0; e < 4; ++e) out[x / 4][x % 4 * 4 + e] = out[x / 4][x % 4 * 4 + e] * f0 + w[e] * f1;
      }
    }
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
    sum = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    // a token sees itself: without any weight its scores are all -inf, and no weight is a number
    sum = sum == 0.f ? __builtin_nanf("") : 1.f / sum;
  }
  if (KS > 1 && ks) return;
  if (i >= s.tokens) return;
  const bool live = i < len;
  // A lane has four consecutive values four times for each 32, its neighbour l ^ 32 the
  // four after them: exchanged, each has eight, a 16-byte run of the row.
#pragma unroll
  for (int y = 0; y < NV; ++y)
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      V4 x0, x1;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x0[e] = (T)(live ? out[y][8 * g + e] * sum : 0.f);
        x1[e] = (T)(live ? out[y][8 * g + 4 + e] * sum : 0.f);
      }
      typedef uint32_t U2 __attribute__((ext_vector_type(2)));
      typedef uint32_t U4 __attribute__((ext_vector_type(4)));
      const U2 u0 = __builtin_bit_cast(U2, x0), u1 = __builtin_bit_cast(U2, x1);
      const auto w0 = __builtin_amdgcn_permlane32_swap(u0.x, u1.x, false, false);
      const auto w1 = __builtin_amdgcn_permlane32_swap(u0.y, u1.y, false, false);
      const U4 w = {w0[0], w1[0], w0[1], w1[1]};
      const int d = 32 * y + 16 * g + 8 * h, left = V - d;
      if (left >= 8) {
        __builtin_memcpy(o + d, &w, 16);
      } else if (left > 0) {
        const V8 z = __builtin_bit_cast(V8, w);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < left) o[d + e] = z[e];
      }
    }
}

template <class E, int DP, int NV, bool DMA, int KS>
hipError_t go(WindowRun run, hipStream_t st) {
  const ncodec_window_shape& s = run.a.s;
  const int group = s.heads / s.kv_heads, waves = kWaves / KS;
  run.head_waves = group % waves == 0 ? waves : group % 2 == 0 ? 2 : 1;
  run.head_tiles = group / run.head_waves;
  const int64_t queries = kQueries * (waves / run.head_waves);
  run.query_blocks = (int)((s.tokens + queries - 1) / queries);
  const int64_t blocks = s.batch * s.kv_heads * run.head_tiles * run.query_blocks;
  // a launch counts its threads in 32 bits
  for (; run.first < blocks; run.first += 1 << 23) {
    launch(k_tok_window<E, DP, NV, DMA, KS>, dim3((unsigned)std::min<int64_t>(blocks - run.first, 1 << 23)), dim3(64 * kWaves), st, run);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <class E, int DP, int NV, bool DMA>
hipError_t by_blocks(const WindowRun& run, hipStream_t st) {
  const ncodec_window_shape& s = run.a.s;
  return window_halves(s.batch * s.heads, s.tokens, s.head_dim, s.value_dim, s.window, s.sinks, run.a.lengths)
             ? go<E, DP, NV, DMA, 2>(run, st)
             : go<E, DP, NV, DMA, 1>(run, st);
}
template <class E, int DP, bool DMA>
hipError_t by_value(const WindowRun& run, hipStream_t st) {
  const int V = run.a.s.value_dim;
  if (V <= 32) return by_blocks<E, DP, 1, DMA>(run, st);
  if (V <= 64) return by_blocks<E, DP, 2, DMA>(run, st);
  if (V <= 96) return by_blocks<E, DP, 3, DMA>(run, st);
  return by_blocks<E, DP, 4, DMA>(run, st);
}
template <class E>
hipError_t run_window(const WindowArgs& a, hipStream_t st) {
  const ncodec_window_shape& s = a.s;
  const auto runs = [](const void* x, int64_t batch, int64_t token, int64_t head) {
    return (uintptr_t)x % 16 == 0 && batch % 8 == 0 && token % 8 == 0 && head % 8 == 0;
  };
  const WindowRun run{a, 0, 0, 0, 0,
                      s.head_dim % 8 == 0 && runs(a.q, s.q_batch_stride, s.q_token_stride, s.q_head_stride)};
  const bool dma = s.head_dim % 8 == 0 && s.value_dim % 8 == 0 && runs(a.k, s.k_batch_stride, s.k_token_stride, s.k_head_stride) &&
                   runs(a.v, s.v_batch_stride, s.v_token_stride, s.v_head_stride) && s.k_token_stride < (1 << 26) &&
                   s.v_token_stride < (1 << 26);
  if (s.head_dim <= 64) return dma ? by_value<E, 64, true>(run, st) : by_value<E, 64, false>(run, st);
  return dma ? by_value<E, 128, true>(run, st) : by_value<E, 128, false>(run, st);
}

}  // namespace

hipError_t launch_window_attention(const WindowArgs& a, hipStream_t st) {
  return a.s.dtype == NCODEC_DTYPE_FP16 ? run_window<F16>(a, st) : run_window<BF16>(a, st);
}

}  // namespace nc
