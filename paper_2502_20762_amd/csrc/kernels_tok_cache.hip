// The upkeep of a paged cache: new tokens into its pages, and eviction by
// accumulated attention weight.  Both move rows, bound by the bytes; the choice of the
// tokens to keep is a radix selection in three rounds of 11, 11 and 10 bits.
//
// 130,560 tokens of 4 heads of 128 + 128 into the cache, 535 MB: 108 us (4.9 TB/s, a large
// copy's rate).  64 sequences of up to 2,040 tokens cut to 1,020, 8 heads of 64 + 64: 11 us for the
// choice and 51 for the rows (196 MB, 3.9 TB/s; heads of a token side by side in the grid were no
// faster), one of 130,560 to 32,640, 4 heads of 128 + 128: four launches of 5, 8, 8 and 11.5 us,
// each waiting for the counts of the one before, and 35 for the rows (134 MB, 3.9 TB/s).
#include <algorithm>

#include "token_rules.hpp"
#include "tokens.hpp"

namespace nc {
namespace {

// ---- rows --------------------------------------------------------------------
// A workgroup moves `rows` rows (tokens of an append, kept positions of an eviction),
// each of `heads` heads of uk + uv units of U elements, a thread up to eight of them at a
// time.  Where the rows lie is looked up once, into LDS.
constexpr int kUnits = 8, kMaxRows = 128;

struct Split {
  int rows;            // of a workgroup
  int dk, dv, uk, uv;  // elements and units of a head's key and value
  uint64_t row, k, v;  // ceil(2^32 / units of a row, uk, uv): quotients of indices below 2^26
};
__device__ __forceinline__ int quotient(uint32_t i, uint64_t magic) { return (int)((i * magic) >> 32); }

// from(r, h, v), to(r, h, v): first element of row r's head h, key or value, or NULL.  A
// head's last unit ends with it: where its elements are no multiple of U it moves
// some of the unit before once more.
template <int U, bool ALIGNED, class From, class To>
__device__ __forceinline__ void move_rows(const Split& s, int rows, int heads, From from, To to) {
  typedef uint16_t T __attribute__((ext_vector_type(U == 1 ? 2 : U)));
  typedef T Loose __attribute__((aligned(2)));
  const int per = heads * (s.uk + s.uv), all = rows * per;
  const int threads = blockDim.x;
  for (int i0 = threadIdx.x; i0 < all; i0 += kUnits * threads) {
    T v[kUnits];
    uint16_t* p[kUnits];
#pragma unroll
    for (int x = 0; x < kUnits; ++x) {
      const int i = i0 + threads * x;
      p[x] = nullptr;
      if (i >= all) continue;
      const int r = s.rows == 1 ? 0 : quotient(i, s.row), q = i - r * per;
      const bool value = q >= heads * s.uk;
      const int y = value ? q - heads * s.uk : q, h = quotient(y, value ? s.v : s.k), u = y - h * (value ? s.uv : s.uk);
      uint16_t* dst = to(r, h, value);
      const uint16_t* src = from(r, h, value);
      if (!dst || !src) continue;
      const int d = ALIGNED ? U * u : min(U * u, (value ? s.dv : s.dk) - U);
      p[x] = dst + d;
      if (U == 1)
        v[x][0] = src[d];
      else if (ALIGNED)
        v[x] = *(const T*)(src + d);
      else
        __builtin_memcpy(&v[x], src + d, sizeof(T));
    }
#pragma unroll
    for (int x = 0; x < kUnits; ++x) {
      if (!p[x]) continue;
      // device memory, which the compiler does not see behind the NULL
      if (U == 1)
        *(__attribute__((address_space(1))) uint16_t*)p[x] = v[x][0];
      else if (ALIGNED)
        *(__attribute__((address_space(1))) T*)p[x] = v[x];
      else
        *(__attribute__((address_space(1))) Loose*)p[x] = v[x];
    }
  }
}

// Units of 16 bytes wherever heads are that wide, at the alignment of an element where
// bases or strides are no better (33,011 tokens of 3 sequences, 4 heads of 75 and 128: 275 us
// in single elements).
bool runs(std::initializer_list<int64_t> sizes, std::initializer_list<const void*> bases) {
  int64_t all = 0;
  for (int64_t v : sizes) all |= v;
  for (const void* p : bases) all |= (int64_t)((uintptr_t)p / 2);
  return all % 8 == 0;
}
Split split_of(const ncodec_cache_shape& c, int heads, int unit, int64_t rows) {
  Split s;
  s.dk = c.head_dim;
  s.dv = c.value_dim;
  s.uk = (c.head_dim + unit - 1) / unit;
  s.uv = (c.value_dim + unit - 1) / unit;
  const int64_t per = (int64_t)heads * (s.uk + s.uv);
  s.rows = (int)std::max<int64_t>(1, std::min<int64_t>({2048 / per, kMaxRows, rows}));
  const auto magic = [](uint64_t d) { return (((uint64_t)1 << 32) + d - 1) / d; };
  s.row = magic(per);
  s.k = magic(s.uk);
  s.v = magic(s.uv);
  return s;
}

template <int U, bool ALIGNED>
__global__ __launch_bounds__(256) void k_tok_append(AppendArgs a, Split sp, int64_t first, int64_t blocks) {
  __shared__ int64_t page[kMaxRows];  // -1: the token goes nowhere
  __shared__ int line[kMaxRows];
  const ncodec_cache_shape& c = a.c;
  const ncodec_append_shape& s = a.s;
  const int64_t block = first + blockIdx.x, b = block / blocks, i0 = block % blocks * sp.rows, cap = s.columns * c.page_size;
  const int64_t count = a.counts ? min(max((int64_t)a.counts[b], (int64_t)0), s.tokens) : s.tokens;
  const int rows = (int)min((int64_t)sp.rows, count - i0);
  if (rows <= 0) return;
  if ((int)threadIdx.x < rows) {
    const int64_t j = a.starts[b] + i0 + threadIdx.x;
    int64_t p = -1;
    if (j >= 0 && j < cap) {
      p = a.table[b * s.table_stride + (j >> (__ffs(c.page_size) - 1))];
      if (p < 0 || p >= c.pages) p = -1;
    }
    page[threadIdx.x] = p;
    line[threadIdx.x] = (int)(j & (c.page_size - 1));
    if (a.mass && p >= 0)
      for (int h = 0; h < c.kv_heads; ++h) a.mass[(b * c.kv_heads + h) * cap + j] = 0.f;
  }
  __syncthreads();
  const uint16_t* k = (const uint16_t*)a.k + b * s.k_batch_stride + i0 * s.k_token_stride;
  const uint16_t* v = (const uint16_t*)a.v + b * s.v_batch_stride + i0 * s.v_token_stride;
  move_rows<U, ALIGNED>(
      sp, rows, c.kv_heads,
      [&](int r, int h, bool value) {
        return value ? v + r * s.v_token_stride + h * s.v_head_stride : k + r * s.k_token_stride + h * s.k_head_stride;
      },
      [&](int r, int h, bool value) -> uint16_t* {
        const int64_t p = page[r];
        if (p < 0) return nullptr;
        return value ? (uint16_t*)a.v_cache + p * c.v_page_stride + line[r] * c.v_token_stride + h * c.v_head_stride
                     : (uint16_t*)a.k_cache + p * c.k_page_stride + line[r] * c.k_token_stride + h * c.k_head_stride;
      });
}

// Rows of positions x0 .. x0 + rows - 1 of a sequence's head, to the new pages.
struct Places {
  int64_t from[kMaxRows], to[kMaxRows];  // pages; to -1: not copied
  int from_line[kMaxRows], to_line[kMaxRows];
};
template <int U, bool ALIGNED>
__device__ __forceinline__ void move_kept(const EvictArgs& a, const Split& sp, Places& at, int64_t bh, int64_t x0, int rows) {
  const ncodec_cache_shape& c = a.c;
  const ncodec_evict_shape& s = a.s;
  const int64_t b = bh / c.kv_heads;
  const int h = (int)(bh % c.kv_heads), shift = __ffs(c.page_size) - 1;
  const int32_t* kept = a.kept + bh * s.keep + x0;
  for (int r = threadIdx.x; r < rows; r += blockDim.x) {
    const int32_t j = kept[r];
    const int64_t x = x0 + r;
    int64_t p = -1, q = -1;
    if (j >= 0) {
      p = a.table[b * s.table_stride + (j >> shift)];
      q = a.new_table[b * s.new_table_stride + (x >> shift)];
      if (p < 0 || p >= c.pages || q < 0 || q >= c.pages) q = -1;
    }
    at.from[r] = p;
    at.to[r] = q;
    at.from_line[r] = j & (c.page_size - 1);
    at.to_line[r] = (int)(x & (c.page_size - 1));
  }
  __syncthreads();
  uint16_t *k = (uint16_t*)a.k_cache + h * c.k_head_stride, *v = (uint16_t*)a.v_cache + h * c.v_head_stride;
  move_rows<U, ALIGNED>(
      sp, rows, 1,
      [&](int r, int, bool value) -> const uint16_t* {
        if (at.to[r] < 0) return nullptr;
        return value ? v + at.from[r] * c.v_page_stride + at.from_line[r] * c.v_token_stride
                     : k + at.from[r] * c.k_page_stride + at.from_line[r] * c.k_token_stride;
      },
      [&](int r, int, bool value) {
        return value ? v + at.to[r] * c.v_page_stride + at.to_line[r] * c.v_token_stride
                     : k + at.to[r] * c.k_page_stride + at.to_line[r] * c.k_token_stride;
      });
}

template <int U, bool ALIGNED>
__global__ __launch_bounds__(256) void k_tok_evict_move(EvictArgs a, Split sp, int64_t first, int64_t blocks) {
  __shared__ Places at;
  // The last positions of what keeps fewer are empty: they take turns over the XCDs and their engines, to
  // which workgroups go in order (64 sequences of up to 2,040 tokens: 65.7 -> 61.2 us a call).
  const int64_t block = first + blockIdx.x, bh = block / blocks, x0 = (block + bh + bh / 4) % blocks * sp.rows;
  if (a.kept[bh * a.s.keep + x0] < 0) return;  // the kept ones come first
  move_kept<U, ALIGNED>(a, sp, at, bh, x0, (int)min((int64_t)sp.rows, a.s.keep - x0));
}

// ---- which tokens are kept --------------------------------------------------
constexpr int kBins = 2048, kMost = 8;  // kMost: positions of a thread at most
constexpr int kShift[3] = {21, 10, 0};                           // of a round's 11, 11 and 10 bits

struct PickRun {
  EvictArgs a;
  int segments;   // of a sequence; more than one meet in the workspace:
  int32_t* hist;  // batch x kv_heads x 3 rounds x segments x kBins
  int32_t* meta;  // batch x kv_heads x (2 rounds x (bits so far, still wanted) + segments: heavier ones of each)
};

// A key whose order is that of the weights, -0 as 0 and a NaN above all.
__device__ __forceinline__ uint32_t weight_key(float f) {
  if (f != f) return 0xffffffffu;
  const uint32_t u = __float_as_uint(f + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// What a workgroup knows of its sequence and head.
struct Pick {
  int n, m, lo, hi, want;  // tokens, kept ones, [lo, hi) to choose from, how many of those
};
__device__ __forceinline__ Pick pick_of(const EvictArgs& a, int64_t bh) {
  const ncodec_evict_shape& s = a.s;
  Pick p;
  p.n = (int)min(max((int64_t)a.lengths[bh / a.c.kv_heads], (int64_t)0), s.columns * a.c.page_size);
  p.m = (int)min((int64_t)p.n, s.keep);
  p.lo = (int)min(s.sinks, (int64_t)p.n);
  p.hi = (int)max((int64_t)p.lo, p.n - s.recent);
  p.want = p.m - p.lo - (p.n - p.hi);
  return p;
}

// Exclusive sum over the workgroup's threads, and the total in `all`.
__device__ __forceinline__ int block_scan(int v, int* lds, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  int sum = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(sum, d, 64);
    sum += lane >= d ? up : 0;
  }
  if (lane == 63) lds[wave] = sum;
  __syncthreads();
  int before = 0;
  all = 0;
  for (int w = 0; w < waves; ++w) {
    before += w < wave ? lds[w] : 0;
    all += lds[w];
  }
  __syncthreads();
  return before + sum - v;
}

// The bin, from the top, in which the want-th (want >= 1) value lies, and how many lie
// above it.  bins(x): count of bin x.
template <class Bins>
__device__ __forceinline__ int2 find_bin(Bins bins, int want, int* lds, int2* found) {
  const int per = kBins / (int)blockDim.x, top = kBins - 1 - (int)threadIdx.x * per;
  int mine = 0, all;
  for (int x = 0; x < per; ++x) mine += bins(top - x);
  int above = block_scan(mine, lds, all);
  if (above < want && want <= above + mine)
    for (int x = 0; x < per; ++x) {
      const int c = bins(top - x);
      if (above < want && want <= above + c) *found = int2{top - x, above};
      above += c;
    }
  __syncthreads();
  return *found;
}

struct Chosen {
  uint32_t key;      // what is heavier is kept,
  int equal;         // and of what weighs as much so many, the earliest
  int sure, ties;    // heavier (or fixed) ones and equals before this segment
};
template <int kMine>
__device__ __forceinline__ void write_kept(const EvictArgs& a, int64_t bh, const Pick& p, const Chosen& ch, int j0, int segment,
                                           int segments, const uint32_t (&u)[kMine], int* lds, uint16_t* list) {
  const ncodec_evict_shape& s = a.s;
  const int64_t new_cap = s.new_columns * a.c.page_size;
  int32_t* kept = a.kept + bh * s.keep;
  float* new_mass = a.new_mass + bh * new_cap;
  int sure = 0, ties = 0;
#pragma unroll
  for (int e = 0; e < kMine; ++e) {
    const int j = j0 + e;
    const bool mid = j >= p.lo && j < p.hi;
    sure += j < p.n && (!mid || u[e] > ch.key) ? 1 : 0;
    ties += mid && u[e] == ch.key ? 1 : 0;
  }
  int all;
  const int before = block_scan(sure | ties << 16, lds, all);  // both below 2^14
  // in order into LDS, and from there next to each other (8,192 positions: 7 us of scattered stores)
  const int first = ch.sure + min(ch.ties, ch.equal);
  const int count = (all & 0xffff) + min(ch.ties + (all >> 16), ch.equal) - min(ch.ties, ch.equal);
  sure = before & 0xffff;
  ties = ch.ties + (before >> 16);
#pragma unroll
  for (int e = 0; e < kMine; ++e) {
    const int j = j0 + e;
    const bool mid = j >= p.lo && j < p.hi, is = j < p.n && (!mid || u[e] > ch.key), tie = mid && u[e] == ch.key;
    if (is || (tie && ties < ch.equal)) list[sure + min(ties, ch.equal) - min(ch.ties, ch.equal)] = (uint16_t)(kMine * threadIdx.x + e);
    sure += is ? 1 : 0;
    ties += tie ? 1 : 0;
  }
  __syncthreads();
  const float* mass = a.mass + bh * s.columns * a.c.page_size;
  const int start = j0 - kMine * (int)threadIdx.x;
  for (int x = threadIdx.x; x < count; x += blockDim.x) {
    const int j = start + list[x];
    kept[first + x] = j;
    new_mass[first + x] = mass[j];
  }
  const int64_t step = (int64_t)segments * blockDim.x;
  for (int64_t x = p.m + (int64_t)segment * blockDim.x + threadIdx.x; x < new_cap; x += step) {
    if (x < s.keep) kept[x] = -1;
    new_mass[x] = 0.f;
  }
  if (segment == 0 && threadIdx.x == 0 && bh % a.c.kv_heads == 0) a.new_lengths[bh / a.c.kv_heads] = p.m;
}

template <int kMine>
__device__ __forceinline__ void load_keys(const float* mass, int j0, int end, uint32_t (&u)[kMine]) {
  float w[kMine];
  if (j0 + kMine <= end) {
    floatx4 v[kMine / 4];
    __builtin_memcpy(v, mass + j0, sizeof(v));
#pragma unroll
    for (int e = 0; e < kMine; ++e) w[e] = v[e / 4][e % 4];
  } else {
#pragma unroll
    for (int e = 0; e < kMine; ++e) w[e] = j0 + e < end ? mass[j0 + e] : 0.f;
  }
#pragma unroll
  for (int e = 0; e < kMine; ++e) u[e] = weight_key(w[e]);
}

// A workgroup for a whole sequence and head, of up to 1024 kMine positions.  U > 0: it also
// moves the rows.
template <int kMine, int U, bool ALIGNED>
__global__ __launch_bounds__(1024) void k_tok_evict_pick(EvictArgs a, Split sp, int64_t first) {
  __shared__ int hist[kBins], lds[16];
  __shared__ uint16_t list[1024 * kMine];
  __shared__ Places at;
  __shared__ int2 found;
  const int64_t bh = first + blockIdx.x;
  const Pick p = pick_of(a, bh);
  const int j0 = threadIdx.x * kMine;
  uint32_t u[kMine];
  load_keys(a.mass + bh * a.s.columns * a.c.page_size, j0, p.n, u);
  Chosen ch = {0xffffffffu, 0, 0, 0};
  if (p.want == p.hi - p.lo) {  // all of them: no choice
    ch = {0u, p.want, 0, 0};
  } else if (p.want > 0) {
    uint32_t bits = 0;
    int want = p.want;
#pragma unroll
    for (int round = 0; round < 3; ++round) {
      for (int x = threadIdx.x; x < kBins; x += blockDim.x) hist[x] = 0;
      __syncthreads();
#pragma unroll
      for (int e = 0; e < kMine; ++e) {
        const int j = j0 + e;
        if (j >= p.lo && j < p.hi && (round == 0 || (u[e] ^ bits) >> kShift[round ? round - 1 : 0] == 0))
          atomicAdd(&hist[u[e] >> kShift[round] & (kBins - 1)], 1);
      }
      __syncthreads();
      const int2 f = find_bin([&](int x) { return hist[x]; }, want, lds, &found);
      bits |= (uint32_t)f.x << kShift[round];
      want -= f.y;
      __syncthreads();
    }
    ch = {bits, want, 0, 0};
  }
  write_kept(a, bh, p, ch, j0, 0, 1, u, lds, list);
  if constexpr (U > 0) {
    for (int64_t x0 = 0; x0 < p.m; x0 += kMaxRows) {
      __syncthreads();  // the list is written, and the places before are read
      move_kept<U, ALIGNED>(a, sp, at, bh, x0, (int)min((int64_t)kMaxRows, p.m - x0));
    }
  }
}

// The same for longer ones, a workgroup a segment and a launch a round: round 0 to 2
// count their bits, and the launch after each finds the bin from all segments' counts.
// 1024 threads, two bins each.
template <int ROUND>
__global__ __launch_bounds__(1024) void k_tok_evict_round(PickRun run, int64_t first) {
  constexpr int kMine = kMost;
  __shared__ int hist[kBins], lds[16];
  __shared__ uint16_t list[1024 * kMine];
  __shared__ int2 found;
  const EvictArgs& a = run.a;
  const int S = run.segments, segment = (int)((first + blockIdx.x) % S);
  const int64_t bh = (first + blockIdx.x) / S;
  const Pick p = pick_of(a, bh);
  const int j0 = segment * kSegment + threadIdx.x * kMine;
  uint32_t u[kMine];
  load_keys(a.mass + bh * a.s.columns * a.c.page_size, j0, p.n, u);
  int32_t* hists = run.hist + bh * 3 * S * kBins;
  int32_t* meta = run.meta + bh * (4 + S);
  const bool choice = p.want > 0 && p.want < p.hi - p.lo;
  if (!choice && ROUND < 3) return;
  uint32_t bits = 0;
  int want = p.want;
  Chosen ch = p.want == p.hi - p.lo ? Chosen{0u, p.want, 0, 0} : Chosen{0xffffffffu, 0, 0, 0};
  if (choice && ROUND > 0) {
    const int32_t* last = hists + (ROUND - 1) * S * kBins;
    if (ROUND > 1) {
      bits = meta[2 * (ROUND - 2)];
      want = meta[2 * (ROUND - 2) + 1];
    }
    // this thread's two bins, from the top: of all segments, and of this one (in the last
    // round, of those before it)
    const int bin = kBins - 2 - 2 * (int)threadIdx.x;
    int2 sum = {0, 0}, part = {0, 0};
    for (int y0 = 0; y0 < S; y0 += 8) {
      int2 c[8];
#pragma unroll
      for (int y = 0; y < 8; ++y) c[y] = *(const int2*)(last + (int64_t)min(y0 + y, S - 1) * kBins + bin);
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const bool in = y0 + y < S, mine = in && (ROUND < 3 ? y0 + y == segment : y0 + y < segment);
        sum.x += in ? c[y].x : 0;
        sum.y += in ? c[y].y : 0;
        part.x += mine ? c[y].x : 0;
        part.y += mine ? c[y].y : 0;
      }
    }
    const int2 f = find_bin([&](int x) { return x == bin ? sum.x : sum.y; }, want, lds, &found);
    bits |= (uint32_t)f.x << kShift[ROUND - 1];
    want -= f.y;
    int sure = (bin > f.x ? part.x : 0) + (bin + 1 > f.x ? part.y : 0), all;
    int ties = (bin == f.x ? part.x : 0) + (bin + 1 == f.x ? part.y : 0);
    if (ROUND == 3)
      for (int y = threadIdx.x; y < segment; y += blockDim.x) sure += meta[4 + y];
    block_scan(sure, lds, all);
    sure = all;
    if (ROUND == 3) {
      block_scan(ties, lds, all);
      ties = all;
    }
    if (ROUND < 3) {
      if (threadIdx.x == 0) {
        if (segment == 0) {
          meta[2 * (ROUND - 1)] = bits;
          meta[2 * (ROUND - 1) + 1] = want;
        }
        meta[4 + segment] = (ROUND == 1 ? 0 : meta[4 + segment]) + sure;
      }
    } else {
      ch = {bits, want, sure, ties};
    }
  }
  if (ROUND < 3) {
    for (int x = threadIdx.x; x < kBins; x += blockDim.x) hist[x] = 0;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kMine; ++e) {
      const int j = j0 + e;
      if (j >= p.lo && j < p.hi && (ROUND == 0 || (u[e] ^ bits) >> kShift[ROUND ? ROUND - 1 : 0] == 0))
        atomicAdd(&hist[u[e] >> kShift[ROUND < 3 ? ROUND : 0] & (kBins - 1)], 1);
    }
    __syncthreads();
    for (int x = threadIdx.x; x < kBins; x += blockDim.x) hists[(ROUND * S + segment) * kBins + x] = hist[x];
    return;
  }
  // the fixed ones before this segment, and where nothing is chosen all or none of the others
  const int start = min(segment * kSegment, p.n);
  ch.sure += min(start, p.lo) + max(0, start - p.hi);
  if (p.want == p.hi - p.lo) ch.sure += max(0, min(start, p.hi) - p.lo);
  write_kept(a, bh, p, ch, j0, segment, S, u, lds, list);
}

template <int U, bool ALIGNED>
hipError_t append(const AppendArgs& a, hipStream_t st) {
  const Split sp = split_of(a.c, a.c.kv_heads, U, a.s.tokens);
  const int64_t blocks = (a.s.tokens + sp.rows - 1) / sp.rows, all = a.s.batch * blocks;
  // a launch counts its threads in 32 bits
  for (int64_t first = 0; first < all; first += 1 << 23) {
    launch(k_tok_append<U, ALIGNED>, dim3((unsigned)std::min<int64_t>(all - first, 1 << 23)), dim3(256), st, a, sp, first, blocks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <int U, bool ALIGNED>
hipError_t move(const EvictArgs& a, hipStream_t st) {
  const Split sp = split_of(a.c, 1, U, a.s.keep);
  const int64_t blocks = (a.s.keep + sp.rows - 1) / sp.rows, all = a.s.batch * a.c.kv_heads * blocks;
  for (int64_t first = 0; first < all; first += 1 << 23) {
    launch(k_tok_evict_move<U, ALIGNED>, dim3((unsigned)std::min<int64_t>(all - first, 1 << 23)), dim3(256), st, a, sp, first, blocks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

constexpr int64_t kMostBlocks = 1 << 21;  // of up to 1024 threads, which a launch counts in 32 bits

// Four positions a thread where 1024 threads hold them all (64 sequences of 2040, 8 heads:
// 10.6 us, 12.8 with eight).
template <int kMine, int U, bool ALIGNED>
hipError_t pick(const EvictArgs& a, const Split& sp, hipStream_t st) {
  const int64_t blocks = a.s.batch * a.c.kv_heads, positions = a.s.columns * a.c.page_size;
  unsigned threads = 64;  // a power of two, so that they share the bins evenly
  while (threads * kMine < positions) threads *= 2;
  if (U > 0) threads = std::max(threads, 256u);
  for (int64_t first = 0; first < blocks; first += kMostBlocks) {
    launch(k_tok_evict_pick<kMine, U, ALIGNED>, dim3((unsigned)std::min(blocks - first, kMostBlocks)), dim3(threads), st, a, sp, first);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <int ROUND>
hipError_t round(const PickRun& run, int64_t blocks, hipStream_t st) {
  for (int64_t first = 0; first < blocks; first += kMostBlocks) {
    launch(k_tok_evict_round<ROUND>, dim3((unsigned)std::min(blocks - first, kMostBlocks)), dim3(1024), st, run, first);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

int64_t segments_of(const ncodec_cache_shape& c, const ncodec_evict_shape& s) {
  return std::max<int64_t>(1, (s.columns * c.page_size + kSegment - 1) / kSegment);
}
size_t hist_bytes(const ncodec_cache_shape& c, const ncodec_evict_shape& s, int64_t segments) {
  return (size_t)(s.batch * c.kv_heads) * 3 * segments * kBins * 4;
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t st) {
  const ncodec_cache_shape& c = a.c;
  const ncodec_append_shape& s = a.s;
  if (c.head_dim < 8 || c.value_dim < 8) return append<1, false>(a, st);
  const bool aligned = runs({c.head_dim, c.value_dim, c.k_page_stride, c.k_token_stride, c.k_head_stride, c.v_page_stride,
                             c.v_token_stride, c.v_head_stride, s.k_batch_stride, s.k_token_stride, s.k_head_stride,
                             s.v_batch_stride, s.v_token_stride, s.v_head_stride},
                            {a.k, a.v, a.k_cache, a.v_cache});
  return aligned ? append<8, true>(a, st) : append<8, false>(a, st);
}

size_t evict_workspace_bytes(const ncodec_cache_shape& c, const ncodec_evict_shape& s) {
  const int64_t segments = segments_of(c, s);
  if (segments == 1) return 0;
  return hist_bytes(c, s, segments) + (size_t)(s.batch * c.kv_heads) * (4 + segments) * 4;
}

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t st) {
  const ncodec_cache_shape& c = a.c;
  const ncodec_evict_shape& s = a.s;
  const int64_t bk = s.batch * c.kv_heads, segments = segments_of(c, s), positions = s.columns * c.page_size;
  const bool wide = c.head_dim >= 8 && c.value_dim >= 8;
  const bool aligned = runs({c.head_dim, c.value_dim, c.k_page_stride, c.k_token_stride, c.k_head_stride, c.v_page_stride,
                             c.v_token_stride, c.v_head_stride},
                            {a.k_cache, a.v_cache});
  if (evict_in_one(positions, s.keep, c.head_dim + c.value_dim)) {
    const Split sp = split_of(c, 1, wide ? 8 : 1, kMaxRows);
    return !wide ? pick<4, 1, false>(a, sp, st) : aligned ? pick<4, 8, true>(a, sp, st) : pick<4, 8, false>(a, sp, st);
  }
  hipError_t e = hipSuccess;
  if (segments == 1) {
    e = positions <= 4096 ? pick<4, 0, false>(a, Split{}, st) : pick<8, 0, false>(a, Split{}, st);
  } else {
    const PickRun run{a, (int)segments, (int32_t*)a.ws, (int32_t*)((char*)a.ws + hist_bytes(c, s, segments))};
    e = round<0>(run, bk * segments, st);
    if (e == hipSuccess) e = round<1>(run, bk * segments, st);
    if (e == hipSuccess) e = round<2>(run, bk * segments, st);
    if (e == hipSuccess) e = round<3>(run, bk * segments, st);
  }
  if (e != hipSuccess) return e;
  return !wide ? move<1, false>(a, st) : aligned ? move<8, true>(a, st) : move<8, false>(a, st);
}

}  // namespace nc
