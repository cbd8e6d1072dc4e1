// Matrix product with bias, activation, gate and residual in its epilogue:
//   y = act(x W^T + b) [* (x W2^T + b2)] + r.
// Computed transposed like the codec's pointwise kernels: the weight rows are
// the MFMA A operand, the tokens are the columns, and a lane of the
// accumulator holds one token and four consecutive features at a time.
// Operands are read as they lie in memory: nothing is packed beforehand.
#include <algorithm>

#include "token_rules.hpp"
#include "tokens.hpp"

namespace nc {
namespace {

// Activations in fp32.  The logistic is 1 / (1 + exp(-v)) with the hardware
// exponential and reciprocal.  Rounding the exponential's argument makes a relative
// error of 2^-24 times it and a little, 2^-21 at 8 and 2^-17 at 88 where the result ends, far
// below the rounding of y.  v Phi(v) = max(v, 0) - |v| Phi(-|v|), and Phi(-a) =
// exp(-a^2 / 2) M(a) with M fitted on [0, 14] as t times a polynomial of degree 6
// in t = 1 / (1 + 0.36 a) by iteratively reweighted least squares of the relative
// error, which stays below 9e-7, so the tail keeps its digits.
template <int ACT>
__device__ __forceinline__ float act1(float v) {
  if (ACT == NCODEC_ACT_LRELU) return v >= 0.f ? v : 0.1f * v;
  if (ACT == NCODEC_ACT_WSILU) return v * __builtin_amdgcn_rcpf(1.f + __expf(-4.f * v));
  if (ACT == NCODEC_ACT_SILU) return v * __builtin_amdgcn_rcpf(1.f + __expf(-v));
  if (ACT == NCODEC_ACT_GELU) {
    // Phi(-64) is 0: an infinity times it would be no number.  This minimum keeps a NaN, the
    // maximum below need not.
    const float a = __builtin_elementwise_minimum(fabsf(v), 64.f);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.36f, a, 1.f));
    float p = 0.047059200f;
    p = fmaf(p, t, -0.179774719f);
    p = fmaf(p, t, 0.180967717f);
    p = fmaf(p, t, 0.0265398683f);
    p = fmaf(p, t, 0.139722717f);
    p = fmaf(p, t, 0.141771825f);
    p = fmaf(p, t, 0.143713090f);
    const float e = p * t * __builtin_amdgcn_exp2f(-0.72134752f * a * a);
    return fmaf(-a, e, fmaxf(v, 0.f));
  }
  return v;
}
// act is uniform over the launch, so the branch is a scalar one.
template <int N>
__device__ __forceinline__ void activate(float (&v)[N], int act) {
  switch (act) {
#define NC_CASE(A)                                      \
  case A:                                               \
    _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = act1<A>(v[i]); \
    break;
    NC_CASE(NCODEC_ACT_LRELU)
    NC_CASE(NCODEC_ACT_WSILU)
    NC_CASE(NCODEC_ACT_SILU)
    NC_CASE(NCODEC_ACT_GELU)
#undef NC_CASE
    default: break;
  }
}

template <class V>
__device__ __forceinline__ V load_any(const void* p) {  // any alignment
  V v;
  __builtin_memcpy(&v, p, sizeof(V));
  return v;
}
template <class V>
__device__ __forceinline__ void store_any(void* p, V v) {
  __builtin_memcpy(p, &v, sizeof(V));
}
// Eight elements of a row from k on, zeros past its end (rem = K - k).
template <class E>
__device__ __forceinline__ typename E::V8 load_row8(const typename E::T* p, int64_t rem) {
  if (rem >= 8) return load_any<typename E::V8>(p);
  typename E::V8 v = {};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < rem) v[i] = p[i];
  return v;
}

__device__ __align__(16) uint32_t zero16[4];  // what a load past the end of the contraction reads

// ---- tiles ------------------------------------------------------------------
// WN x WM waves of 64 weight rows x 32 TB tokens each.  K streams through LDS in
// stages of BK = 32 or 64 (unit u, 16 bytes, of row r lies at a slot such that 16
// consecutive rows of one unit touch every bank once).  DMA: rows 16-byte
// aligned and K a multiple of 8, staged by direct global->LDS loads ST - 1
// stages ahead; otherwise through registers.  With the gate each 64-row group
// holds 32 rows of W1 and the same 32 of W2, so that both halves of an output
// are in one lane.  A wave reads 2 + TB fragments from LDS for 2 TB MFMAs: with
// TB = 4 the LDS takes 1.5 KiB for every two MFMAs, which its 128 B a clock just
// carry, and the products set the pace (8192 x 4096 -> 4096 bf16 231 us, 1.19 PFLOP/s
// of the 1.49 that the library reaches on 8192^3; 32640 x 2048 -> 512 66 us, 70 with bias
// and residual, again and again on the same tensors; the library's bare product 54.5).
template <class E, bool GATED, bool DMA, int WN, int WM, int TB, int BK, int ST_>
struct Tile {
  static constexpr int NW = WN * WM, TN = 64 * WN, TM = 32 * TB * WM, ROWS = TN + TM;
  static constexpr int OF = GATED ? 32 : 64;       // output features of a wave
  static constexpr int ST = DMA ? ST_ : 2;
  static constexpr int STAGE = ROWS * BK * 2;      // bytes
  static constexpr int U = BK / 8, RPL = 64 / U;   // units of a row, rows of a 1 KiB load
  static constexpr int LOADS = ROWS / RPL / NW;    // 1 KiB loads of a wave and stage
  static __device__ __forceinline__ int slot(int row, int u) { return u ^ (BK == 32 ? (row >> 2) & 3 : (row >> 1) & 7); }
  static constexpr int PITCH = OF * 2 + 16;        // bytes of a token's row in the epilogue
  static constexpr int LDS = ST * STAGE > NW * 32 * PITCH ? ST * STAGE : NW * 32 * PITCH;
  static_assert(ST >= 2 && ST <= 4, "the waits in the loop count one to three stages in flight");
  static_assert(ROWS / RPL % NW == 0, "every wave stages the same number of rows");
};

template <class E, bool GATED, bool DMA, int WN, int WM, int TB, int BK, int ST_>
__global__ __launch_bounds__(64 * WN * WM, 2) void k_tok_linear(LinearArgs a) {
  typedef Tile<E, GATED, DMA, WN, WM, TB, BK, ST_> C;
  typedef typename E::T T;
  typedef typename E::V8 V8;
  typedef typename E::V4 V4;
  __shared__ __align__(1024) char lds[C::LDS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, l32 = lane & 31;
  const int wn = wave % WN, wm = wave / WN;
  const int K = (int)a.s.k;
  // token tiles of one XCD follow each other, all feature tiles of a token tile together
  const uint32_t nt = (uint32_t)((a.s.n + C::OF * WN - 1) / (C::OF * WN));
  const uint32_t tile = xcd_tile(blockIdx.x, gridDim.x);
  const int64_t m0 = (int64_t)(tile / nt) * C::TM, n0 = (int64_t)(tile % nt) * (C::OF * WN);
  if (m0 >= a.s.m) return;  // the grid is rounded up to the XCDs

  // this lane's source of each staged unit
  const T* src[C::LOADS];
  int kof[C::LOADS];
#pragma unroll
  for (int i = 0; i < C::LOADS; ++i) {
    const int row = C::RPL * (wave + C::NW * i) + lane / C::U;
    const int unit = C::slot(row, lane % C::U);
    if (row < C::TN) {
      int64_t n = GATED ? n0 + 32 * (row >> 6) + (row & 31) : n0 + row;
      n = min(n, a.s.n - 1);
      if (GATED && (row & 32)) n += a.s.n;
      src[i] = (const T*)a.w + n * a.s.ldw + 8 * unit;
    } else {
      const int64_t m = min(m0 + row - C::TN, a.s.m - 1);
      src[i] = (const T*)a.x + m * a.s.ldx + 8 * unit;
    }
    kof[i] = 8 * unit;
  }
  const int nk = (K + BK - 1) / BK;
  auto stage_dma = [&](int kt, int buf) {
    const bool tail = (kt + 1) * BK > K;
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) {
      const void* p = src[i] + (int64_t)kt * BK;
      if (tail && kt * BK + kof[i] >= K) p = zero16;
      dma16(p, lds + buf * C::STAGE + 1024 * (wave + C::NW * i));
    }
  };

  floatx16 acc[2][TB] = {};
  // The fragments of a step of 16 are read between the MFMAs of the step before, one
  // after each (8192 x 4096 -> 4096 bf16: 243 us with the reads right before their
  // use, 231 so).
  auto compute = [&](int buf) {
    const char* base = lds + buf * C::STAGE;
    constexpr int S = BK / 16;
    V8 fa[2][2], fb[2][TB];
    auto get = [&](int s) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = 64 * wn + 32 * i + l32;
        fa[s & 1][i] = *(const V8*)(base + row * (2 * BK) + 16 * C::slot(row, 2 * s + h));
      }
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        const int row = C::TN + 32 * (TB * wm + t) + l32;
        fb[s & 1][t] = *(const V8*)(base + row * (2 * BK) + 16 * C::slot(row, 2 * s + h));
      }
    };
    get(0);
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (s + 1 < S) get(s + 1);
#pragma unroll
      for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) acc[i][t] = E::mfma(fa[s & 1][i], fb[s & 1][t], acc[i][t]);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 2 + TB, 0);
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int x = 0; x < 2 + TB; ++x) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (s + 1 < S) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, TB - 2, 0);
    }
  };

  if (DMA) {
#pragma unroll
    for (int i = 0; i < C::ST - 1; ++i)
      if (i < nk) stage_dma(i, i);
    int buf = 0;
    for (int kt = 0; kt < nk; ++kt) {
      // this wave's loads of stage kt have landed (those of later stages may be in flight) ...
      if (C::ST > 3 && kt + 2 < nk)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * C::LOADS) : "memory");
      else if (C::ST > 2 && kt + 1 < nk)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(C::LOADS) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      // ... and everyone's, and everyone is done with the buffer that the next load goes to
      lds_barrier();
      if (kt + C::ST - 1 < nk) stage_dma(kt + C::ST - 1, buf == 0 ? C::ST - 1 : buf - 1);
      compute(buf);
      buf = buf == C::ST - 1 ? 0 : buf + 1;
    }
  } else {
    V8 reg[C::LOADS];
    auto fetch = [&](int kt) {
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i) reg[i] = load_row8<E>(src[i] + (int64_t)kt * BK, K - kt * BK - kof[i]);
    };
    auto put = [&](int buf) {
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i)
        *(V8*)(lds + buf * C::STAGE + 1024 * (wave + C::NW * i) + 16 * lane) = reg[i];
    };
    fetch(0);
    put(0);
    for (int kt = 0; kt < nk; ++kt) {
      if (kt + 1 < nk) fetch(kt + 1);
      __syncthreads();
      compute(kt & 1);
      if (kt + 1 < nk) put((kt + 1) & 1);
    }
  }
  lds_barrier();  // the stages are read; each wave's part of LDS is its own from here on

  // Epilogue, 32 tokens at a time: results (and the residual before them) go
  // through LDS so that global accesses are whole 16-byte units of a row.
  char* mine = lds + wave * 32 * C::PITCH;
  constexpr int UNITS = C::OF / 8;            // 16-byte units of a token's row
  constexpr int RPI = 64 / UNITS;             // tokens an instruction covers
  constexpr int ITER = 32 / RPI;
  const int eu = lane % UNITS, er = lane / UNITS;
  const int64_t nw0 = n0 + C::OF * wn, mw0 = m0 + 32 * TB * wm;
  const int64_t ne = nw0 + 8 * eu;            // first feature of this lane's unit
  const int nval = (int)min(max(a.s.n - ne, (int64_t)0), (int64_t)8);
  const T* bias = (const T*)a.b;
  const T* res = (const T*)a.r;
  T* y = (T*)a.y;
  V4 bq[2][4] = {};  // the lane's features: 32 i + 8 q + 4 h, with the gate i is the half
  if (bias) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t n = nw0 + (GATED ? 0 : 32 * i) + 8 * q + 4 * h;
        const T* p = bias + (GATED && i ? a.s.n : 0) + n;
        if (n + 4 <= a.s.n)
          bq[i][q] = load_any<V4>(p);
        else
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (n + j < a.s.n) bq[i][q][j] = p[j];
      }
  }
#pragma unroll
  for (int t = 0; t < TB; ++t) {
    const int64_t mt = mw0 + 32 * t;
    if (res) {
#pragma unroll
      for (int it = 0; it < ITER; ++it) {
        const int64_t m = mt + RPI * it + er;
        V8 v = {};
        if (m < a.s.m) v = load_row8<E>(res + m * a.s.ldr + ne, nval);
        *(V8*)(mine + (RPI * it + er) * C::PITCH + 16 * eu) = v;
      }
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int i = 0; i < (GATED ? 1 : 2); ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int f = 32 * i + 8 * q + 4 * h;  // first of the lane's four features
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = acc[i][t][4 * q + j] + (float)bq[i][q][j];
        activate(v, a.s.act);
        if (GATED) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] *= acc[1][t][4 * q + j] + (float)bq[1][q][j];
        }
        V4* slot = (V4*)(mine + l32 * C::PITCH + 2 * f);
        if (res) {
          const V4 r4 = *slot;
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] += (float)r4[j];
        }
        V4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = (T)v[j];
        *slot = o;
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int it = 0; it < ITER; ++it) {
      const int64_t m = mt + RPI * it + er;
      const V8 o = *(const V8*)(mine + (RPI * it + er) * C::PITCH + 16 * eu);
      if (m < a.s.m) {
        T* p = y + m * a.s.ldy + ne;
        if (nval == 8)
          store_any(p, o);
        else
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < nval) p[j] = o[j];
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- few rows -----------------------------------------------------------------
// 16 features x 16 TB tokens a workgroup; its eight waves take turns along K
// (32 at a time, both operands straight from memory) and their partial sums
// meet in LDS in wave order.  The weights are read once and the launch is wide
// enough to read them from every CU: 1 x 512 -> 2048 bf16, 2 MB, 3.3 us, most of it a
// launch and one pass through the memory's latency.
__device__ __forceinline__ floatx4 mfma16(half8 a, half8 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 mfma16(bhalf8 a, bhalf8 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

template <class E, bool GATED, int TB>
__global__ __launch_bounds__(512) void k_tok_linear_rows(LinearArgs a) {
  typedef typename E::T T;
  typedef typename E::V8 V8;
  constexpr int G = GATED ? 2 : 1;
  __shared__ float part[8][G][TB][16][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l16 = lane & 15, kl = 8 * (lane >> 4);
  const uint32_t nt = (uint32_t)((a.s.n + 15) / 16);
  const int64_t m0 = (int64_t)(blockIdx.x / nt) * (16 * TB), n0 = (int64_t)(blockIdx.x % nt) * 16;
  const int K = (int)a.s.k;
  const T* wp = (const T*)a.w + min(n0 + l16, a.s.n - 1) * a.s.ldw;
  const T* xp[TB];
#pragma unroll
  for (int t = 0; t < TB; ++t) xp[t] = (const T*)a.x + min(m0 + 16 * t + l16, a.s.m - 1) * a.s.ldx;
  floatx4 acc[G][TB] = {};
#pragma unroll 2
  for (int k0 = 32 * wave; k0 < K; k0 += 256) {
    const int k = k0 + kl;
    V8 fa[G], fb[TB];
#pragma unroll
    for (int g = 0; g < G; ++g) fa[g] = load_row8<E>(wp + g * a.s.n * a.s.ldw + k, K - k);
#pragma unroll
    for (int t = 0; t < TB; ++t) fb[t] = load_row8<E>(xp[t] + k, K - k);
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
      for (int g = 0; g < G; ++g) acc[g][t] = mfma16(fa[g], fb[t], acc[g][t]);
  }
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) part[wave][g][t][l16][4 * (lane >> 4) + r] = acc[g][t][r];
  __syncthreads();
  const T* bias = (const T*)a.b;
  for (int i = threadIdx.x; i < 256 * TB; i += 512) {
    const int f = i & 15, tok = i >> 4;
    const int64_t m = m0 + tok, n = n0 + f;
    if (m >= a.s.m || n >= a.s.n) continue;
    float s[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      s[g] = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) s[g] += part[w][g][tok >> 4][tok & 15][f];
      if (bias) s[g] += (float)bias[g * a.s.n + n];
    }
    float v[1] = {s[0]};
    activate(v, a.s.act);
    if (GATED) v[0] *= s[G - 1];
    if (a.r) v[0] += (float)((const T*)a.r)[m * a.s.ldr + n];
    ((T*)a.y)[m * a.s.ldy + n] = (T)v[0];
  }
}

template <class E, bool GATED, bool DMA, int WN, int WM, int TB, int BK, int ST_>
hipError_t go_tile(const LinearArgs& a, hipStream_t st) {
  typedef Tile<E, GATED, DMA, WN, WM, TB, BK, ST_> C;
  int64_t grid = ((a.s.m + C::TM - 1) / C::TM) * ((a.s.n + C::OF * WN - 1) / (C::OF * WN));
  grid = (grid + kNumXCD - 1) / kNumXCD * kNumXCD;
  launch(k_tok_linear<E, GATED, DMA, WN, WM, TB, BK, ST_>, dim3((unsigned)grid), dim3(64 * C::NW), st, a);
  return hipGetLastError();
}

template <class E, bool GATED, int TB>
hipError_t go_rows(const LinearArgs& a, hipStream_t st) {
  const int64_t grid = ((a.s.m + 16 * TB - 1) / (16 * TB)) * ((a.s.n + 15) / 16);
  launch(k_tok_linear_rows<E, GATED, TB>, dim3((unsigned)grid), dim3(512), st, a);
  return hipGetLastError();
}

template <class E, bool GATED>
hipError_t pick(const LinearArgs& a, hipStream_t st) {
  const ncodec_linear_shape& s = a.s;
  const bool direct =
      s.k % 8 == 0 && s.ldx % 8 == 0 && s.ldw % 8 == 0 && (uintptr_t)a.x % 16 == 0 && (uintptr_t)a.w % 16 == 0;
  switch (linear_rule(s.m, s.n * (GATED ? 2 : 1), s.k, direct)) {
    case LinearKernel::rows16: return go_rows<E, GATED, 1>(a, st);
    case LinearKernel::rows32: return go_rows<E, GATED, 2>(a, st);
    case LinearKernel::rows64: return go_rows<E, GATED, 4>(a, st);
    case LinearKernel::reg128x64: return go_tile<E, GATED, false, 2, 2, 1, 32, 2>(a, st);
    case LinearKernel::reg128x128: return go_tile<E, GATED, false, 2, 2, 2, 32, 2>(a, st);
    case LinearKernel::reg256x256: return go_tile<E, GATED, false, 4, 2, 4, 32, 2>(a, st);
    case LinearKernel::dma128x64: return go_tile<E, GATED, true, 2, 2, 1, 64, 2>(a, st);
    case LinearKernel::dma128x128: return go_tile<E, GATED, true, 2, 2, 2, 32, 3>(a, st);
    case LinearKernel::dma256x128k32: return go_tile<E, GATED, true, 4, 2, 2, 32, 3>(a, st);
    case LinearKernel::dma256x128k64: return go_tile<E, GATED, true, 4, 2, 2, 64, 2>(a, st);
    case LinearKernel::dma256x256: return go_tile<E, GATED, true, 4, 2, 4, 64, 2>(a, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace

// A launch counts its threads in 32 bits: rows past 2^22 of the smallest tiles go in further launches.
hipError_t launch_linear(const LinearArgs& a, hipStream_t st) {
  const int64_t nf = a.s.n * (a.s.gated ? 2 : 1), rows = (((int64_t)1 << 22) / ((nf + 127) / 128)) * 64;
  for (int64_t m0 = 0; m0 < a.s.m; m0 += rows) {
    LinearArgs p = a;
    p.s.m = std::min(rows, a.s.m - m0);
    p.x = (const char*)a.x + 2 * m0 * a.s.ldx;
    p.y = (char*)a.y + 2 * m0 * a.s.ldy;
    if (a.r) p.r = (const char*)a.r + 2 * m0 * a.s.ldr;
    const hipError_t e = a.s.dtype == NCODEC_DTYPE_FP16
                             ? (a.s.gated ? pick<F16, true>(p, st) : pick<F16, false>(p, st))
                             : (a.s.gated ? pick<BF16, true>(p, st) : pick<BF16, false>(p, st));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace nc
