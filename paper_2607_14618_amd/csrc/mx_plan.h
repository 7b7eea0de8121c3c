// The microscaled 4-bit operators' host side: sizes of the packed layout and which kernel, tile and split a call takes.
// No device code, so that the host tests read the same rules.  Not part of the public ABI.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "internal.h"

namespace polyq {
namespace mx {

constexpr int kBlock = POLYQ_MX_BLOCK;  // values that share a scale
constexpr int kRows = 16;               // rows of a packed tile: the rows of one matrix instruction
constexpr int kChunk = 128;             // values of a row that one matrix instruction takes
constexpr int kChunkBytes = kRows * kChunk / 2;
constexpr int kRec = 4 * kChunk;        // values of a row that one 4-byte word of scales covers
constexpr int kScaleBytes = 256;        // scales of a record: a word per lane, its byte c of chunk c
constexpr int kRecBytes = kScaleBytes + 4 * kChunkBytes;

__host__ __device__ inline int div_up(int a, int b) { return (a + b - 1) / b; }
__host__ __device__ inline int chunks_of(int k) { return div_up(k, kChunk); }
__host__ __device__ inline int records_of(int k) { return div_up(k, kRec); }
__host__ __device__ inline int tiles_of(int rows) { return div_up(rows, kRows); }
__host__ __device__ inline int64_t tile_bytes(int k) {
  return static_cast<int64_t>(records_of(k)) * kScaleBytes + static_cast<int64_t>(chunks_of(k)) * kChunkBytes;
}

// The work-items of a launch have to stay below 2^32 (in each dimension of its grid).
constexpr int64_t kMaxItems = (1ll << 32) - 1;
inline bool launch_fits(int64_t groups, int threads) { return groups <= kMaxItems / threads; }
// Work-groups of one item per thread, as many as a launch holds: the kernel walks what is left with the grid's stride.
inline uint32_t striding_groups(int64_t items, int threads) {
  return static_cast<uint32_t>(std::min((items + threads - 1) / threads, kMaxItems / threads));
}

// Quantization and back: a work-group of 256 per record of a tile (`padded`: rows to whole 64).
inline int64_t record_groups(int32_t rows, int32_t k, bool padded) {
  return (padded ? align_up(rows, 64) / kRows : tiles_of(rows)) * static_cast<int64_t>(records_of(k));
}

// ------------------------------------------------------------------ products
// Which kernel a product of more than 16 tokens takes, by estimates in microseconds.
//   split, TM = 1 or 2 token tiles of 32: 3 us, and the longest of what its work-groups read at 12 MB/us (L2), of
//     one's own reading at 45 KB/us and of the weights at 5 MB/us (memory);
//   gemm, 256 rows (gated 128 of each) x 32 TM tokens, TM = 1 .. 4: 5.5 us, and the longer of its chunks and of the
//     weights at 4.5 MB/us.  A chunk takes a work-group alone on its compute unit {0.15, 0.20, 0.28, 0.36} us,
//     several {0.20, 0.31, 0.40, 0.50} each.  The weights' term is the same for every TM; where it decides, the largest
//     tile is taken, which is not always the fastest (gated of 77 below: 33 and not 23).
// Measured, split 1 / split 2 / gemm of TM = 1, 2, 3, 4 (us): linear of 77 tokens, 5120 x 5120: 9.9 / 10.1 / 11.3, 12.9,
// 17.8, 21.0; of 256: 19.8 / 17.9 / 11.5, 13.4, 17.5, 20.6; of 64, 5120 x 13824: 17.6 / 20.7 / -, 33.8; of 1000: 108 / 108
// / 72, 53.6, 46.8, 58.7; of 2000: - / - / 137, 94.9, 81.1, 89.6; gated of 77, 13824 x 5120: 45 / 34 / -, 23, 28, 33; of
// 2000: - / - / -, 189, 159, 154.
struct Choice {
  bool split;
  int tm;
};
inline Choice choose(int64_t m, int64_t n, int64_t k, int mats) {
  static const double alone[4] = {0.15, 0.20, 0.28, 0.36}, shared[4] = {0.20, 0.31, 0.40, 0.50};
  const double row = static_cast<double>(tile_bytes(static_cast<int>(k))) / kRows, weights = row * n * mats;
  const int64_t chunks = chunks_of(static_cast<int>(k));
  Choice best = {true, 1};
  double least = 0;
  for (int tm = 1; tm <= 2; ++tm) {
    const int64_t groups = (n + 31) / 32 * ((m + 32 * tm - 1) / (32 * tm));
    const double bytes = row * 32 * (mats + tm);
    const double t = 3 + std::max({groups * bytes / 12e6, std::max(1.0, groups / 256.0) * bytes / 45e3, weights / 5e6});
    if (tm == 1 || t < least) least = t, best = {true, tm};
  }
  if (m <= 32) return {true, 1};
  for (int tm = 1; tm <= 4; ++tm) {
    const int64_t groups = (n * mats + 255) / 256 * ((m + 32 * tm - 1) / (32 * tm)), each = (groups + 255) / 256;
    const double t = 5.5 + std::max(chunks * (each == 1 ? alone[tm - 1] : each * shared[tm - 1]), weights / 4.5e6);
    if (t <= least) least = t, best = {false, tm};
  }
  return best;
}

// Its launch over n rows of each weight and m tokens (with the padding that it writes).
struct Launch {
  int64_t groups;
  int threads;
};
inline Launch product_launch(Choice c, int64_t m, int64_t n, int mats) {
  const int64_t token_blocks = (m + 32 * c.tm - 1) / (32 * c.tm);
  if (c.split) return {(n + 31) / 32 * token_blocks, c.tm == 1 || mats == 1 ? 512 : 256};
  return {(n * mats + 255) / 256 * token_blocks, 256};
}

inline bool product_fits(int64_t m, int64_t n, int64_t k, int mats, int64_t m_written, int64_t n_written) {
  const Launch l = product_launch(choose(m, n, k, mats), m_written, n_written, mats);
  return launch_fits(l.groups, l.threads);
}

// ------------------------------------------------------------------ gradients
constexpr int kStep = 64;          // r of a stage
constexpr int kMaxRows = 1 << 21;  // tokens and output channels: a work-group's S is reached with 32-bit offsets

// One gradient product's tile (l x s) and splits: 256 x 256 by eight waves where that makes 128 tiles, or 256 x 64 by four;
// of dx, whose small tiles take all terms in one stage, 128 x 64 where those are few, which makes the stages
// shorter and more of them at once.  256 x 64 / 128 x 64, dx with its sums (us): 64 tokens, 1024 x 5120 fp32 26.3 / 17.7, 5120 x
// 5120 bf16 24.3 / 23.6; 500 tokens, 5120 x 13824 102 / 110.
// The reduction (`steps` stages of each of `terms`) is split where rounds of whole tiles leave much of the GPU idle; a split
// costs its partial sums, about as much as 8 stages, and has at least 8.
struct Shape {
  int l, s, l_blocks, s_blocks, splits;
};
inline Shape grad_shape(bool dw, int l, int s, int outs, int steps, int terms) {
  Shape h;
  const bool big = static_cast<int64_t>(div_up(l, 256)) * div_up(s, 256) * outs >= 128;
  const bool few = !dw && static_cast<int64_t>(div_up(l, 256)) * div_up(s, 64) <= 64;
  h.l = few ? 128 : 256, h.s = big ? 256 : 64;
  h.l_blocks = div_up(l, h.l), h.s_blocks = div_up(s, h.s);
  const int64_t groups = static_cast<int64_t>(h.l_blocks) * h.s_blocks * outs;
  const int stages = dw || big ? steps * terms : steps, slots = big ? kCUs : few ? 4 * kCUs : 2 * kCUs;  // slots: work-groups at once
  h.splits = 1;
  int64_t best = -1;
  for (int n = 1; n <= 32 && (n == 1 || stages / n >= 8); ++n) {
    const int64_t rounds = (groups * n + slots - 1) / slots, cost = rounds * ((stages + n - 1) / n + (n > 1 ? 8 : 0));
    if (best < 0 || cost < best) best = cost, h.splits = n;
  }
  return h;
}

// Its launches, the sum over the splits of outputs of `rows` x k among them.
inline bool shape_fits(const Shape& h, int outs, int64_t rows, int64_t k) {
  return launch_fits(static_cast<int64_t>(h.l_blocks) * h.s_blocks * outs, h.s == 256 ? 512 : 256) &&
         (h.splits == 1 || launch_fits((rows * k + 1023) / 1024, 256));
}
// Transposing packed activations: a work-group of four waves per four chunks of tiles of m_pad rows.
inline int64_t transpose_groups(int32_t m_pad, int32_t k) {
  return (static_cast<int64_t>(m_pad / kRows) * chunks_of(k) + 3) / 4;
}

}  // namespace mx
}  // namespace polyq
