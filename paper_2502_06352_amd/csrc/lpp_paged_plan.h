// How a call of paged attention is cut: the shape of its blocks, the ranges of its keys, how these are joined.  Host code alone:
// tests/test_paged_plan.py compiles it by itself and holds the tests' inputs to the paths that they are for.
#ifndef LPP_PAGED_PLAN_H_
#define LPP_PAGED_PLAN_H_

#include <math.h>

#include <algorithm>

#include "lpp_internal.h"

namespace {

struct PagedPlan {
  int shape, rows, kt, wk;           // bf16: which of kShapes; rows of a block, keys of a tile, waves along the keys
  int row_blocks, nsplit, range;
  bool join_later;
  size_t lds;
  size_t o_bytes, ml_bytes;          // partials
};

// Shapes of a bf16 block, and what a round of its waves (kt * wk keys) costs in microseconds: with heads of 64 and of 128
// numbers, the block by itself on a compute unit and each of many there.  Fitted to the times of 240 inputs (1 to 384 heads in
// all, 1 to 8192 rows, 16 to 32768 keys, two thirds of the batches of mixed lengths) with 1 to 128 ranges of keys, joined in
// both ways.
struct Shape { int wr, wk, kt, st; int resident[2]; float alone[2], each[2]; };
constexpr Shape kShapes[] = {
    {1, 4, 32, 1, {4, 2}, {0.87f, 1.16f}, {0.33f, 1.39f}},
    {1, 8, 32, 1, {2, 1}, {1.23f, 1.19f}, {0.74f, 2.07f}},
    {2, 4, 32, 2, {2, 1}, {0.87f, 0.89f}, {0.52f, 1.40f}},
    {4, 1, 64, 2, {3, 2}, {0.95f, 1.25f}, {0.55f, 0.99f}},
    {4, 2, 32, 2, {2, 1}, {0.74f, 0.76f}, {0.58f, 1.14f}},
};
constexpr int kRanges[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128};

// What adding up the ranges of a launch costs: by the block that finishes last (bytes: of a row tile) or in a launch of its
// own, which reads with all compute units but costs a caller without a graph another 4 us of host time.  (1 head, 108 rows,
// 21419 keys in 16 ranges: 32.6 us and 23.1, replayed; 8 heads, 4 rows, 2400 keys in 10: 10.7 and 10.4.)
inline float join_last(float bytes) { return 3.2f + bytes / 18900.f; }
inline float join_launch(float bytes) { return 6.f + bytes / 3090000.f; }

// The shape and the number of ranges whose estimate is least: rounds of a block, each as long as a compute unit takes with the
// blocks that fall to it, or what the memory takes for the keys and values, a fixed cost for every block of a compute unit, and
// the joining.  Blocks of a chunk longer than any tree see half of the new keys on average, and as they are of all lengths, the
// longest first, they fill the chip more evenly.  The choices take 1.02 times the best measured one over the inputs above, one
// in thirty of them more than 1.15 times, at worst 1.29, and 1.05 times over 80 others of few rows and long caches, at worst
// 1.38; blocks of 32, 64 or 128 rows by the number of rows alone took up to 8 times that.
inline PagedPlan plan_paged(const lpp_paged* cache, int64_t B, int gq, int64_t M, int64_t S) {
  PagedPlan p{};
  const int64_t R = M * gq, heads = B * cache->Hkv;
  const int Dh = cache->Dh, d = Dh == 128;
  const bool bf16 = cache->dtype == LPP_BF16;
  const Shape f32[2] = {{1, Dh == 64 ? 16 : 8, 16, 0, {1, 1}, {3.3f, 3.2f}, {3.1f, 3.2f}}, {2, 8, 16, 0, {1, 1}, {3.0f, 5.2f}, {2.9f, 5.5f}}};
  float best = INFINITY;
  const float memory = (float)heads * (float)(S + M) * (float)(Dh * (bf16 ? 4 : 8)) / 9.e6f;   // (two thirds of the inputs were shorter than S)
  for (int i = 0; i < (bf16 ? (int)(sizeof(kShapes) / sizeof(kShapes[0])) : 2); ++i) {
    const Shape& h = bf16 ? kShapes[i] : f32[i];
    const int rows = h.wr * (bf16 ? 32 : 16);
    if (i > 0 && h.wr > 1 && R <= rows / 2) break;   // (no block has more rows than the next smaller one would)
    const int64_t row_blocks = (R + rows - 1) / rows, units = heads * row_blocks;
    const int tiles = (int)((S + h.kt - 1) / h.kt + (M + h.kt - 1) / h.kt), rounds = (tiles + h.wk - 1) / h.wk;
    const bool causal = M > LPP_MAX_ROWS;
    const float seen = causal ? 1.f - 0.5f * (float)((M + h.kt - 1) / h.kt) / (float)tiles : 1.f, full = causal ? 0.35f : 0.75f;
    int before = 0;
    for (const int g : kRanges) {
      const int per = (rounds + std::min(g, rounds) - 1) / std::min(g, rounds), ranges = (rounds + per - 1) / per;
      if (ranges == before) continue;                // (as many as the last choice)
      before = ranges;
      const int64_t blocks = units * ranges;
      if (ranges > 1 && blocks * rows * (Dh + 2) * 4 >= (int64_t)1 << 31) break;      // (32-bit offsets into the parts)
      const float each = (float)blocks / (float)cache->n_cu, k = ceilf(each);
      const float load = (1.f - full) * std::max(1.f, each * seen) + full * k * seen;      // (between the average and the fullest)
      const float turns = 1.f + (ceilf(k / (float)h.resident[d]) - 1.f) * seen;
      float t = std::max((float)per * std::max(h.alone[d] * turns, h.each[d] * load), memory) + 0.87f * k;
      bool later = false;
      if (ranges > 1) {
        const float bytes = (float)ranges * (float)std::min<int64_t>(R, rows) * (float)(Dh * 4);
        const float last = units <= LPP_COUNTER_SLOTS ? join_last(bytes) : INFINITY, launch = join_launch(bytes * (float)units);
        later = launch < last;
        t += std::min(last, launch);
      }
      if (t < best) {
        best = t;
        p.shape = i; p.rows = rows; p.kt = h.kt; p.wk = h.wk;
        p.row_blocks = (int)row_blocks; p.nsplit = ranges; p.range = per * h.wk; p.join_later = later;
        const size_t merge = h.wk > 1 ? (size_t)h.wk * rows * (Dh + 4) * sizeof(float) : 0;
        p.lds = std::max((size_t)h.st * h.wk * 2 * h.kt * Dh * 2, merge);
      }
      if (per == 1 || (ranges > 1 && each > 8.f)) break;
    }
  }
  const size_t parts = p.nsplit > 1 ? (size_t)heads * p.row_blocks * p.nsplit * p.rows : 0;
  p.o_bytes = lpp_align_up(parts * Dh * sizeof(float), 256);
  p.ml_bytes = lpp_align_up(parts * 2 * sizeof(float), 256);
  return p;
}

// Whether blocks look at all items' lengths: where blocks are long enough to pay for it (half a microsecond each), ranges of three
// rounds or more in launches of up to two blocks a compute unit, which shorter ranges fill better (3 items, 48 heads over 12 of
// 128, 277 rows, 708 to 2124 keys, 972 blocks: 73 us, 86 with shorter ones); without ranges, eight rounds or more in launches that
// do not fit at once.
inline bool looks_at_lengths(const lpp_paged* cache, int64_t B, const PagedPlan& p) {
  const int64_t blocks = B * cache->Hkv * p.nsplit * p.row_blocks, n_cu = cache->n_cu;
  const int per = p.range / p.wk;
  return B > 1 && B <= 64 && (p.nsplit > 1 ? per >= 3 && blocks <= 2 * n_cu : per >= 8 && blocks > n_cu);
}

}  // namespace

#endif  // LPP_PAGED_PLAN_H_
