// Which kernel of a token operator takes a call, by sizes, type and alignment
// alone.  Plain host code, so that tests can hold their sizes to it.
#pragma once
#include <algorithm>
#include <cstdint>

namespace nc {

// ---- matrix product
// rowsT: few rows, T of them a workgroup; tiles: weight rows x tokens, loaded
// directly to LDS (dma) or through registers (reg), in stages of 32 or 64 along K.
enum class LinearKernel {
  rows16, rows32, rows64, reg128x64, reg128x128, reg256x256, dma128x64, dma128x128, dma256x128k32, dma256x128k64, dma256x256
};

// Which kernel, by the size alone (times in us, bf16, both sides; m x k -> n, n the
// weight rows).
//  - Few outputs go to the rows kernel, whose waves share K: 130 x 2048 -> 1024
//    10.4 there and 19.5 on the smallest tile; the two meet at about 2^19 outputs
//    (512 x 1024 -> 1024: 11.9 and 11.7; 1000 x 256 -> 1024: 7.9 and 5.9).
//    Its own token blocks grow with the outputs: 64 x 1024 -> 1024 4.1 / 5.0 / 7.1 with
//    16 / 32 / 64 tokens, 512 x 256 -> 256 4.0 / 3.1 / 3.8, 1000 x 1024 -> 256 9.5 / 7.9 / 7.3.
//  - Then the largest tile (features x tokens) that still leaves work for most CUs: 256 x 256
//    from 150 of them on (14793 x 2048 -> 712 64 us, 69 in 256 x 128, 68 in 128 x 128; with 128 of
//    them, 8160 x 1024 -> 1024, 31.5 against 24.1), 256 x 128 in stages of 64 from 150 of those (8160
//    x 2048 -> 1024 41.5, 50 in 128 x 128; with 128 of them, 8160 x 2048 -> 512, 33 against 28),
//    128 x 64 up to three a CU (3000 x 1024 -> 1024 15.0, 18 in 128 x 128), else 128 x 128.
//  - Short contractions, K < 512, are mostly epilogue and stay with the small tiles (6000 x
//    256 -> 1024 9.9 in 128 x 64, 11.4 in 256 x 128), and up to K = 512 a large product takes
//    256 x 128 in stages of 32: two workgroups a CU, one's epilogue behind the other's
//    products (32640 x 512 -> 2048 with GELU, fp16: 121 to 127, 133 to 139 in 256 x 256).
// Rows that are not 16-byte aligned go through registers; tiles of three sizes.
// nf: weight rows; direct: rows are whole 16-byte units.
inline LinearKernel linear_rule(int64_t m, int64_t nf, int64_t k, bool direct) {
  const int64_t outs = m * nf;
  if (m <= 16 || outs <= ((int64_t)1 << 19)) {
    if (m <= 16 || outs <= 96 * 1024) return LinearKernel::rows16;
    if (m <= 32 || outs <= 192 * 1024) return LinearKernel::rows32;
    return LinearKernel::rows64;
  }
  const auto tiles = [&](int64_t f, int64_t tok) { return ((m + tok - 1) / tok) * ((nf + f - 1) / f); };
  const bool small = tiles(128, 64) <= 768;
  if (!direct) {
    if (tiles(256, 256) >= 150) return LinearKernel::reg256x256;
    return small ? LinearKernel::reg128x64 : LinearKernel::reg128x128;
  }
  if (k <= 512 && tiles(256, 256) >= 512) return LinearKernel::dma256x128k32;
  if (k >= 512 && tiles(256, 256) >= 150) return LinearKernel::dma256x256;
  if (k >= 512 && tiles(256, 128) >= 150) return LinearKernel::dma256x128k64;
  return small ? LinearKernel::dma128x64 : LinearKernel::dma128x128;
}

// ---- attention with a decay
constexpr int kChunk = 64;  // tokens

// Sequences shorter than this run the recurrence, which takes a step of 1 to 2 us for
// every token where a chunk takes the same time for 1 and 64.  us there / in a chunk: 4
// tokens 7.0 / 8.4 with 8 heads of 64 x 64, 8.2 / 11.4 with 8 of 128 x 128, 18.6 / 19.8 with
// 512 of these; 6 tokens 9.2 / 8.5, 10.7 / 11.4, 22.2 / 19.8.
constexpr int64_t kRecurTokens = 6;

struct DecayPlan {
  bool chunked;
  int seg_chunks, nseg;
};

// One wave a SIMD (1,024 of them) is where splitting a sequence stops to pay for
// the second pass over k and v: 512 heads of 8 chunks of 64 x 64 take 43 us whole and 52 in
// halves.  Below that the sequences are cut into two waves for each SIMD, in
// segments of two chunks at least (16 heads of 510 chunks, 64 x 64: 93 us in 64 segments, 117
// in 32, 106 in 128; 8 heads of 128 chunks: 32.0 us in twos, 34.1 singly in fp16, 32.7 and
// 33.8 in bf16).  Two waves are resident on a SIMD where a workgroup has four, or
// two and a head_dim up to 64; with fewer waves the LDS of the workgroups, and at
// 128 x 64 the registers, leave room for one or less, and the others follow (8 heads of
// 128 chunks: 64 x 32 24 us, 128 x 32 32, 128 x 64 41).
inline DecayPlan decay_rule(int64_t bh, int64_t tokens, int64_t value_dim) {
  DecayPlan p{tokens >= kRecurTokens, 0, 1};
  const int64_t chunks = (tokens + kChunk - 1) / kChunk;
  if (!p.chunked || bh == 0) return p;
  const int64_t waves = value_dim <= 32 ? 1 : value_dim <= 64 ? 2 : 4;
  int64_t nseg = 1;
  if (bh * waves < 1024) nseg = std::max<int64_t>(1, std::min(chunks / 2, 2048 / (bh * waves)));
  const int64_t per = (chunks + nseg - 1) / nseg;
  p.seg_chunks = (int)per;
  p.nseg = (int)((chunks + per - 1) / per);
  return p;
}

}  // namespace nc
