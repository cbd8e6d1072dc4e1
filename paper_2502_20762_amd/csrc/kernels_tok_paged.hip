// Softmax attention of one new token of each sequence over a paged cache:
//   o = sum_j p_j v_j over the tokens j that the last one sees, p = softmax(scale q . k_j).
//
// Two operations for each pair of cached elements and query heads of a group: the
// bytes of the cache are the floor.  Positions go in steps of 32, as MFMA products of
// 16 query heads of one key head: scores^T = K q^T, outputs^T = V^T p^T, with both
// operands loaded from memory straight into their registers, the next step's keys behind this
// one's values; in the 16 x 16 accumulators a lane holds one head, so that maximum, sum and
// rescaling stay in the lane's column.  Fewer heads than 16 leave columns empty, which costs
// nothing that the bytes do not.  Weights enter the products as two 16-bit terms, which costs
// nothing either and leaves the output's rounding as the only one.
// A sequence is cut over workgroups, whose maxima, sums and outputs a second launch
// joins; where weights are summed it also turns the scores, which the first one keeps, into them.
//
// 64 sequences of up to 8,160 tokens, 4 key heads of 128 + 128, bf16, 557 MB: 119 + 5 us (4.7 TB/s,
// where a large copy reaches 4.9); one of 130,560, fp16, 267 MB: 54 + 5 (5.0 TB/s); 8 with 4,080 in
// sight, 8 key heads of 64 + 64, weights summed, 68 MB: 17 + 6, of which the start of the
// workgroups, three dependent loads (length, page number, row), takes about 5; one token of 200: 6.5 us,
// nearly all of it that start and the end.
#include <algorithm>

#include "tok_attend.hpp"
#include "tok_tiles.hpp"

namespace nc {
namespace {

constexpr int kStep = 32;    // positions of a wave's step
constexpr int kHeads = 16;   // query heads of a workgroup
constexpr int kWaves = 4;
constexpr int kMaxSplits = 256;
// In the place of a sum: tokens are seen, and all scores are -inf.  With another token's
// score that is not, they weigh nothing; alone, no weight is a number.
constexpr float kAllMinusInf = -1.f;

struct PagedRun {
  PagedArgs a;
  int splits, head_tiles;
  bool q_runs;      // queries are whole 16-byte runs
  int64_t zstride;  // scores of a head in the workspace; 0: they are not kept
  float2* ml;       // batch x heads x splits: maximum and sum
  float* o;         // batch x heads x splits x value_dim: means of the values
  float* z;         // batch x heads x zstride: scores
};

__device__ __forceinline__ floatx4 mfma16(half8 a, half8 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 mfma16(bhalf8 a, bhalf8 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// The steps of a sequence: those that hold first tokens, then those from the window on.
struct Steps {
  int lead, from, count;
  __device__ __forceinline__ int at(int x) const { return x < lead ? x : x - lead + from; }
};
__device__ __forceinline__ Steps steps_of(const Seen& s, int n) {
  Steps r;
  r.lead = (s.first + kStep - 1) / kStep;
  r.from = max(s.near / kStep, r.lead);
  r.count = n > 0 ? r.lead + max(0, (n + kStep - 1) / kStep - r.from) : 0;
  return r;
}

// Steps of a split: whole rounds of the workgroup's waves.
__device__ __forceinline__ int share_of(const Steps& s, int splits) {
  return ((s.count + splits - 1) / splits + kWaves - 1) / kWaves * kWaves;
}
// log2 of the largest weight as the sums hold it.  fp16: its terms keep 2^-38 of that.  bf16: a wave's
// weights sum up to 1 at most, so that no sum of weighted values leaves fp32 where their mean does not, and none is
// smaller than it has to be: up to 2^16 positions a wave, a value of 2^-126 that has all the weight keeps its bits
// above fp32's last, 2^-149.  The sums join as means.
template <class E>
__device__ __forceinline__ float top_power(int share) {
  if (__is_same(E, F16)) return 14.f;
  return (float)__clz(max(1, share / kWaves) * kStep - 1) - 32.f;
}

// N elements from p; those from `left` on, or all where !in, are zero.  VEC: whole
// runs only, aligned to them; otherwise whole runs lie where they may, and a row's last,
// shorter one goes element by element.
template <int N, bool VEC>
__device__ __forceinline__ void load_run(uint32_t (&r)[N / 2], const uint16_t* p, bool in, int left) {
  typedef uint32_t V __attribute__((ext_vector_type(N / 2)));
  typedef V Loose __attribute__((aligned(2)));
#pragma unroll
  for (int i = 0; i < N / 2; ++i) r[i] = 0;
  if (in && left >= N) {
    const V v = VEC ? *(const V*)p : *(const Loose*)p;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) r[i] = v[i];
  } else if (!VEC && in && left > 0) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < left) r[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
  }
}

// PAGE: 2 where a step lies in one page, 1 where in two, 0 where each row is looked up.
template <class E, int DC, int VW, int PAGE, bool VEC>
__global__ __launch_bounds__(64 * kWaves) void k_tok_paged(PagedRun run) {
  typedef typename E::T T;
  typedef typename E::V8 V8;
  typedef uint32_t U4 __attribute__((ext_vector_type(4)));
  constexpr int VP = 16 * VW;
  __shared__ float part[kWaves][kHeads][VP + 4], ml[kWaves][2][kHeads];
  const PagedArgs& a = run.a;
  const ncodec_cache_shape& c = a.c;
  const ncodec_paged_shape& s = a.s;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m16 = lane & 15, g4 = lane >> 4;
  const int group = s.heads / c.kv_heads, D = c.head_dim, V = c.value_dim;
  uint32_t at = blockIdx.x;
  const int split = at % (uint32_t)run.splits;
  at /= (uint32_t)run.splits;
  const int tile = at % (uint32_t)run.head_tiles;
  at /= (uint32_t)run.head_tiles;
  const int hk = at % (uint32_t)c.kv_heads;
  const int64_t b = at / (uint32_t)c.kv_heads;
  const int h0 = hk * group + tile * kHeads, nh = min(kHeads, group - tile * kHeads);
  const int64_t bh0 = b * s.heads + h0;

  const int64_t cap = c.pages ? s.columns * c.page_size : 0;
  const int n = (int)min(max((int64_t)a.lengths[b], (int64_t)0), cap);
  const Seen seen = seen_by(n - 1, s.window, s.sinks);
  const Steps steps = steps_of(seen, n);
  const int per = share_of(steps, run.splits);
  const int x0 = split * per, x1 = min(x0 + per, steps.count);
  const int shift = __ffs(c.page_size) - 1;
  cint* table = (cint*)(a.table + b * s.table_stride);
  const uint16_t* kc = (const uint16_t*)a.k + hk * c.k_head_stride;
  const uint16_t* vc = (const uint16_t*)a.v + hk * c.v_head_stride;

  // queries: lane (head m16, g4) holds dimensions 32 x + 8 g4 ..
  V8 qf[DC];
  {
    const uint16_t* q = (const uint16_t*)a.q + b * s.q_batch_stride + (h0 + m16) * s.q_head_stride;
#pragma unroll
    for (int x = 0; x < DC; ++x) {
      uint32_t r[4];
      if (run.q_runs)
        load_run<8, true>(r, q + 32 * x + 8 * g4, m16 < nh, D - 32 * x - 8 * g4);
      else
        load_run<8, false>(r, q + 32 * x + 8 * g4, m16 < nh, D - 32 * x - 8 * g4);
      qf[x] = __builtin_bit_cast(V8, U4{r[0], r[1], r[2], r[3]});
    }
  }

  // a step's rows: keys 16 t + m16, values 16 t + 4 g4 + r
  uint32_t kr[2][DC][4], vr[8][VW / 2];
  bool okk[2], okv[8];
  auto page_of = [&](int pos) { return table[pos >> shift]; };
  auto is_page = [&](int p) { return (uint32_t)p < (uint32_t)c.pages; };  // pages < 2^31
  int pg[2];  // page numbers of the step whose keys are loaded next (PAGE > 0)
  auto look = [&](int x) {
    if (PAGE == 0 || x >= x1) return;
    const int pos = steps.at(x) * kStep;
    pg[0] = page_of(pos);
    pg[1] = PAGE == 1 ? page_of(min(pos + 16, (int)(cap - 1))) : pg[0];
  };
  auto load_k = [&](int x, const int (&p)[2]) {
    const int pos = steps.at(x) * kStep;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int j = pos + 16 * t + m16;
      const int pj = PAGE ? p[t] : a.table[b * s.table_stride + (min(j, (int)(cap - 1)) >> shift)];
      okk[t] = is_page(pj);
      const uint16_t* row = kc + (okk[t] ? (int64_t)pj * c.k_page_stride + (j & (c.page_size - 1)) * c.k_token_stride : 0);
#pragma unroll
      for (int y = 0; y < DC; ++y) load_run<8, VEC>(kr[t][y], row + 32 * y + 8 * g4, okk[t], D - 32 * y - 8 * g4);
    }
  };
  auto load_v = [&](int x, const int (&p)[2]) {
    const int pos = steps.at(x) * kStep;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = pos + 16 * (e >> 2) + 4 * g4 + (e & 3);
      const int pj = PAGE ? p[e >> 2] : a.table[b * s.table_stride + (min(j, (int)(cap - 1)) >> shift)];
      okv[e] = is_page(pj);
      const uint16_t* row = vc + (okv[e] ? (int64_t)pj * c.v_page_stride + (j & (c.page_size - 1)) * c.v_token_stride : 0);
      load_run<VW, VEC>(vr[e], row + VW * m16, okv[e], V - VW * m16);
    }
  };

  const float scale = s.scale * 1.44269504088896341f, off = top_power<E>(per);
  floatx4 o[VW] = {};
  float m = -__builtin_huge_valf(), l = 0.f;
  bool any = false;
  int x = x0 + wave;
  int cur[2] = {-1, -1};
  look(x);
  cur[0] = pg[0], cur[1] = pg[1];
  if (x < x1) load_k(x, cur);
  for (; x < x1; x += kWaves) {
    load_v(x, cur);
    look(x + kWaves);
    const int pos = steps.at(x) * kStep;
    floatx4 z[2] = {};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int y = 0; y < DC; ++y)
        z[t] = mfma16(__builtin_bit_cast(V8, U4{kr[t][y][0], kr[t][y][1], kr[t][y][2], kr[t][y][3]}), qf[y], z[t]);
    if (x + kWaves < x1) {
      cur[0] = pg[0], cur[1] = pg[1];
      load_k(x + kWaves, cur);
    }
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = z[e >> 2][e & 3] * scale;
      asm("" : "+v"(w[e]));  // rounded: the maximum is one of them
    }
    // positions that are not seen, here or for want of a page
    bool all = pos + kStep <= n && (pos + kStep <= seen.first || pos >= seen.near);
    if (PAGE)
      all = all && okv[0] && okv[4];
    else
      all = false;
    if (!all) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = pos + 16 * (e >> 2) + 4 * g4 + (e & 3);
        const bool in = okv[e] && j < n && (j < seen.first || j >= seen.near);
        w[e] = in ? w[e] : -__builtin_huge_valf();
        any = any || in;
#pragma unroll
        for (int i = 0; i < VW / 2; ++i) vr[e][i] = in ? vr[e][i] : 0;  // no weight of 0 meets a NaN
      }
    } else {
      any = true;
    }
    if (run.zstride && m16 < nh) {
      float* zp = run.z + (bh0 + m16) * run.zstride + pos + 4 * g4;
      *(floatx4*)zp = floatx4{w[0], w[1], w[2], w[3]};
      *(floatx4*)(zp + 16) = floatx4{w[4], w[5], w[6], w[7]};
    }
    float top = w[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, w[e]);
    if (__any(top > m)) {
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float m1 = fmaxf(m, top);
      const float fade = m == -__builtin_huge_valf() ? 0.f : __builtin_amdgcn_exp2f(m - m1);
      m = m1;
      l *= fade;
#pragma unroll
      for (int i = 0; i < VW; ++i) o[i] *= fade;
    }
    const float from = m == -__builtin_huge_valf() ? 0.f : m;
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // in two steps: where scores are so large that off vanishes beside them, the largest weight is still 2^off
      p[e] = __builtin_amdgcn_exp2f((w[e] - from) + off);
      l += p[e];
    }
    V8 hi, lo;
    two_terms<E, true>(p, 1.f, hi, lo);
#pragma unroll
    for (int i = 0; i < VW; ++i) {  // column VW m16 + i of the eight rows
      U4 u;
#pragma unroll
      for (int y = 0; y < 4; ++y)
        u[y] = __builtin_amdgcn_perm(vr[2 * y + 1][i / 2], vr[2 * y][i / 2], i & 1 ? 0x07060302u : 0x05040100u);
      const V8 vf = __builtin_bit_cast(V8, u);
      o[i] = mfma16(vf, lo, o[i]);
      o[i] = mfma16(vf, hi, o[i]);
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  // what is seen is so for all heads, but each lane has looked at eight of a step's positions only
  if (__any(any) && m == -__builtin_huge_valf() && l == 0.f) l = kAllMinusInf;

  // the waves together: element 4 VW g4 + VW r + i of head m16 is o[i][r]
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int i = 0; i < VW; ++i) part[wave][m16][4 * VW * g4 + VW * r + i] = o[i][r];
  if (lane < 16) {
    ml[wave][0][lane] = m;
    ml[wave][1][lane] = l;
  }
  __syncthreads();
  for (int it = threadIdx.x; it < nh * VP; it += 64 * kWaves) {
    const int h = it / VP, d = it % VP;
    float M = ml[0][0][h], L = 0.f, O = 0.f, f[kWaves];
#pragma unroll
    for (int y = 1; y < kWaves; ++y) M = fmaxf(M, ml[y][0][h]);
    bool none = false;
#pragma unroll
    for (int y = 0; y < kWaves; ++y) {
      const float my = ml[y][0][h], ly = ml[y][1][h];
      none = none || ly == kAllMinusInf;
      f[y] = my == -__builtin_huge_valf() ? 0.f : __builtin_amdgcn_exp2f(my - M);
      L = fmaf(ly, f[y], L);  // also where f is 0: what is no number stays so
    }
    const float by = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
    for (int y = 0; y < kWaves; ++y) O = fmaf(part[y][h][d], f[y] * by, O);
    if (none && L == 0.f) L = kAllMinusInf;
    if (run.splits == 1 && d < V)
      ((T*)a.o)[b * s.o_batch_stride + (h0 + h) * s.o_head_stride + d] = (T)(L == 0.f ? 0.f : L == kAllMinusInf ? __builtin_nanf("") : O);
    const int64_t to = (bh0 + h) * run.splits + split;
    if (run.ml && d == 0) run.ml[to] = float2{M, L};
    if (run.splits > 1 && d < V) run.o[to * V + d] = O;
  }
}

// Joins the splits.  The first blocks take a sequence's head each: its outputs.  The
// others take positions of a sequence and key head: their weights, from the scores that
// were kept.  Both begin with the maxima and sums of all splits, a lane for each.
template <class E>
__global__ __launch_bounds__(1024) void k_tok_paged_join(PagedRun run, int heads_blocks, int mass_blocks) {
  typedef typename E::T T;
  __shared__ float fade[kMaxSplits], sums[16][128];
  extern __shared__ float lds[];  // maximum and 1 / sum of each head of the group
  const PagedArgs& a = run.a;
  const ncodec_cache_shape& c = a.c;
  const ncodec_paged_shape& s = a.s;
  const int V = c.value_dim, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  // maximum and 1 / sum of head bh, in every lane of a wave; f: what the splits' means count
  const auto join = [&](int64_t bh, float (&f)[kMaxSplits / 64]) {
    const float2* ml = run.ml + bh * run.splits;
    float M = -__builtin_huge_valf(), L = 0.f, m[kMaxSplits / 64], l[kMaxSplits / 64];
    bool none = false;
#pragma unroll
    for (int y = 0; y < kMaxSplits / 64; ++y) {
      const float2 v = 64 * y + lane < run.splits ? ml[64 * y + lane] : float2{-__builtin_huge_valf(), 0.f};
      m[y] = v.x;
      l[y] = v.y;
      M = fmaxf(M, v.x);
    }
    for (int w = 32; w; w >>= 1) M = fmaxf(M, __shfl_xor(M, w, 64));
#pragma unroll
    for (int y = 0; y < kMaxSplits / 64; ++y) {
      none = none || l[y] == kAllMinusInf;
      f[y] = m[y] == -__builtin_huge_valf() ? 0.f : __builtin_amdgcn_exp2f(m[y] - M);
      L = fmaf(l[y], f[y], L);
    }
    for (int w = 32; w; w >>= 1) L += __shfl_xor(L, w, 64);
    if (__any(none) && L == 0.f) L = __builtin_nanf("");
    const float by = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
    for (int y = 0; y < kMaxSplits / 64; ++y) f[y] *= l[y] * by;
    return float2{M, by};
  };
  if ((int)blockIdx.x < heads_blocks) {
    const int64_t bh = blockIdx.x, b = bh / s.heads;
    float f[kMaxSplits / 64];
    const float2 ml = join(bh, f);
    if (wave == 0) {
#pragma unroll
      for (int y = 0; y < kMaxSplits / 64; ++y) fade[64 * y + lane] = f[y];
    }
    __syncthreads();
    float sum[2] = {};
    const float* o = run.o + bh * run.splits * V;
    const int d0 = min(lane, V - 1), d1 = min(lane + 64, V - 1);
    for (int x = wave; x < run.splits; x += 8 * waves) {
      float v[8][2];
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const float* ox = o + (int64_t)min(x + y * waves, run.splits - 1) * V;
        v[y][0] = ox[d0];
        v[y][1] = ox[d1];
      }
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const float fx = x + y * waves < run.splits ? fade[x + y * waves] : 0.f;  // 0: the last split once more
        sum[0] = fmaf(v[y][0], fx, sum[0]);
        sum[1] = fmaf(v[y][1], fx, sum[1]);
      }
    }
    sums[wave][lane] = sum[0];
    sums[wave][lane + 64] = sum[1];
    __syncthreads();
    const int d = threadIdx.x;
    if (d < V) {
      float O = 0.f;
      for (int w = 0; w < waves; ++w) O += sums[w][d];
      ((T*)a.o)[b * s.o_batch_stride + (bh - b * s.heads) * s.o_head_stride + d] = (T)(ml.y == 0.f ? 0.f : O);
    }
    return;
  }
  const uint32_t block = (blockIdx.x - heads_blocks) % (uint32_t)mass_blocks, bk = (blockIdx.x - heads_blocks) / (uint32_t)mass_blocks;
  const int64_t b = bk / (uint32_t)c.kv_heads;
  const int group = s.heads / c.kv_heads;
  const int64_t bh0 = b * s.heads + (int64_t)(bk % (uint32_t)c.kv_heads) * group, cap = s.columns * c.page_size;
  const int n = (int)min(max((int64_t)a.lengths[b], (int64_t)0), c.pages ? cap : 0), shift = __ffs(c.page_size) - 1;
  const Seen seen = seen_by(n - 1, s.window, s.sinks);
  if (block * (int64_t)blockDim.x >= seen.count) return;
  for (int g = wave; g < group; g += waves) {
    float f[kMaxSplits / 64];
    const float2 ml = join(bh0 + g, f);
    if (lane == 0) {
      lds[2 * g] = ml.x;
      lds[2 * g + 1] = ml.y;
    }
  }
  __syncthreads();
  float* mass = a.mass + (int64_t)bk * cap;
  const float off = top_power<E>(share_of(steps_of(seen, n), run.splits));
  for (int64_t x = block * (int64_t)blockDim.x + threadIdx.x; x < seen.count; x += (int64_t)mass_blocks * blockDim.x) {
    const int j = seen.at((int)x);
    const int32_t page = a.table[b * s.table_stride + (j >> shift)];
    const float before = mass[j];
    float w = 0.f;
    for (int g = 0; g < group; ++g)
      w = fmaf(__builtin_amdgcn_exp2f((run.z[(bh0 + g) * run.zstride + j] - lds[2 * g]) + off), lds[2 * g + 1], w);
    if ((uint32_t)page < (uint32_t)c.pages) mass[j] = before + w;
  }
}

// Splits: up to three workgroups a CU, which is what their registers leave room for with
// heads of 128 (us of the first launch with 512 / 768 / 1024 / 2048 workgroups: 64 ragged sequences of
// 4 key heads 131 / 121 / 132 / 131, one of 130,560 tokens 53 / 57 / 57 / 57, 8 of 8 key heads of 64 + 64
// 19.7 / 18.2 / 21.1 / 21.0), each of two rounds of its waves at least (one round: 25.3).
struct Plan {
  int splits, head_tiles;
  int64_t zstride;
  size_t ml_at, z_at, bytes;  // outputs of splits first
};
Plan plan_of(const ncodec_cache_shape& c, const ncodec_paged_shape& s, bool mass) {
  Plan p;
  const int64_t group = s.heads / c.kv_heads, bh = s.batch * s.heads;
  p.head_tiles = (int)((group + kHeads - 1) / kHeads);
  const int64_t base = std::max<int64_t>(1, s.batch * c.kv_heads * p.head_tiles);
  int64_t most = s.columns * c.page_size;  // positions that may be seen
  if (s.window) most = std::min(most, s.window + s.sinks);
  const int64_t rounds = (most + kStep * kWaves - 1) / (kStep * kWaves);
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({768 / base, rounds / 2, kMaxSplits}));
  p.zstride = mass ? (s.columns * c.page_size + kStep - 1) / kStep * kStep : 0;
  const auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  p.ml_at = p.splits > 1 ? up((size_t)bh * p.splits * c.value_dim * 4) : 0;
  p.z_at = p.ml_at + (p.splits > 1 || mass ? up((size_t)bh * p.splits * 8) : 0);
  p.bytes = p.z_at + (size_t)bh * p.zstride * 4;
  return p;
}

template <class E, int DC, int VW, int PAGE, bool VEC>
hipError_t go(const PagedRun& run, hipStream_t st) {
  const int64_t bk = run.a.s.batch * run.a.c.kv_heads;
  launch(k_tok_paged<E, DC, VW, PAGE, VEC>, dim3((unsigned)(bk * run.head_tiles * run.splits)), dim3(64 * kWaves), st, run);
  return hipGetLastError();
}
template <class E, int DC, int VW>
hipError_t by_page(const PagedRun& run, bool vec, hipStream_t st) {
  const int page = run.a.c.page_size;
  if (!vec) return page >= 32 ? go<E, DC, VW, 2, false>(run, st) : go<E, DC, VW, 0, false>(run, st);
  if (page >= 32) return go<E, DC, VW, 2, true>(run, st);
  if (page == 16) return go<E, DC, VW, 1, true>(run, st);
  return go<E, DC, VW, 0, true>(run, st);
}

template <class E>
hipError_t run_paged(const PagedArgs& a, hipStream_t st) {
  const ncodec_cache_shape& c = a.c;
  const ncodec_paged_shape& s = a.s;
  const Plan p = plan_of(c, s, a.mass != nullptr);
  char* ws = (char*)a.ws;
  const bool join = p.splits > 1 || a.mass;
  const bool q_runs = c.head_dim % 8 == 0 && (uintptr_t)a.q % 16 == 0 && s.q_batch_stride % 8 == 0 && s.q_head_stride % 8 == 0;
  const PagedRun run{a, p.splits, p.head_tiles, q_runs, p.zstride, join ? (float2*)(ws + p.ml_at) : nullptr, (float*)ws, (float*)(ws + p.z_at)};
  const bool vec = c.head_dim % 8 == 0 && c.value_dim % 8 == 0 && (uintptr_t)a.k % 16 == 0 && (uintptr_t)a.v % 16 == 0 &&
                   c.k_page_stride % 8 == 0 && c.k_token_stride % 8 == 0 && c.k_head_stride % 8 == 0 &&
                   c.v_page_stride % 8 == 0 && c.v_token_stride % 8 == 0 && c.v_head_stride % 8 == 0;
  const hipError_t e = c.head_dim <= 64 ? (c.value_dim <= 64 ? by_page<E, 2, 4>(run, vec, st) : by_page<E, 2, 8>(run, vec, st))
                                        : (c.value_dim <= 64 ? by_page<E, 4, 4>(run, vec, st) : by_page<E, 4, 8>(run, vec, st));
  if (e != hipSuccess || !join) return e;
  const int64_t bk = s.batch * c.kv_heads, group = s.heads / c.kv_heads;
  const unsigned threads = p.splits > 32 ? 1024 : 256;
  const int64_t heads_blocks = p.splits > 1 ? s.batch * s.heads : 0;
  int64_t mass_blocks = 0;
  if (a.mass)
    mass_blocks = std::max<int64_t>(1, std::min((s.columns * c.page_size + threads - 1) / threads, 2048 / bk));
  hipLaunchKernelGGL(k_tok_paged_join<E>, dim3((unsigned)(heads_blocks + bk * mass_blocks)), dim3(threads), (unsigned)(8 * group),
                     st, run, (int)heads_blocks, (int)mass_blocks);
  return hipGetLastError();
}

}  // namespace

size_t paged_workspace_bytes(const ncodec_cache_shape& c, const ncodec_paged_shape& s, bool mass) {
  return s.batch ? plan_of(c, s, mass).bytes : 0;
}

hipError_t launch_paged_attention(const PagedArgs& a, hipStream_t st) {
  return a.c.dtype == NCODEC_DTYPE_FP16 ? run_paged<F16>(a, st) : run_paged<BF16>(a, st);
}

}  // namespace nc
