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
  size_t o_bytes, ml_bytes;          // parts of rows: numbers, references and sums
  void room_for(int64_t part_rows, int Dh) {
    o_bytes = lpp_align_up((size_t)part_rows * Dh * sizeof(float), 256);
    ml_bytes = lpp_align_up((size_t)part_rows * 2 * sizeof(float), 256);
  }
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
constexpr int kMostRanges = 128;
// (float32: the second row is of two tiles of 16 rows)
inline Shape shape_of(const lpp_paged* cache, int i) {
  if (cache->dtype == LPP_BF16) return kShapes[i];
  if (i == 0) return {1, cache->Dh == 64 ? 16 : 8, 16, 0, {1, 1}, {3.3f, 3.2f}, {3.1f, 3.2f}};
  return {2, 8, 16, 0, {1, 1}, {3.0f, 5.2f}, {2.9f, 5.5f}};
}
inline int shapes(const lpp_paged* cache) { return cache->dtype == LPP_BF16 ? (int)(sizeof(kShapes) / sizeof(kShapes[0])) : 2; }
inline int rows_of(const lpp_paged* cache, const Shape& h) { return h.wr * (cache->dtype == LPP_BF16 ? 32 : 16); }
// Whether blocks of shape i are for R rows: no block has more rows than the next smaller one would.
inline bool fits_rows(int i, const Shape& h, int rows, int64_t R) { return i == 0 || h.wr == 1 || R > rows / 2; }
inline int64_t rounds_of(const Shape& h, int64_t M, int64_t S) {
  return ((S + h.kt - 1) / h.kt + (M + h.kt - 1) / h.kt + h.wk - 1) / h.wk;
}

// Rows of parts that a launch has at most: 6 blocks of the largest shape a compute unit (102 MB with heads of 128 numbers).  Without a
// limit batches that fill the chip many times over are cut in two for a percent or two, by the estimate, and up to gigabytes
// of parts.  (56 calls that limits of 512, 768 or 1024 rows concern, 100 to 600 us: 0.95, 0.94 and 0.97 of the time without, at worst
// 1.16, 1.13 and 1.04; 100 items of 123 rows, 16 heads over 8 of 128, up to 4161 keys: 469 us without, 287 with.)
inline int64_t most_part_rows(const lpp_paged* cache) { return (int64_t)cache->n_cu * 768; }

// Room for the parts of every call of up to B items, M rows of gq heads and S positions: whatever shape and number of ranges each of
// them is cut into.  It grows with all of these, so that a caller may make its workspace once.
inline size_t paged_room(const lpp_paged* cache, int64_t B, int gq, int64_t M, int64_t S) {
  const int64_t R = M * gq, heads = B * cache->Hkv;
  int64_t most = 0;
  for (int i = 0; i < shapes(cache); ++i) {
    const Shape h = shape_of(cache, i);
    const int rows = rows_of(cache, h);
    if (!fits_rows(i, h, rows, R)) break;
    const int64_t rounds = rounds_of(h, M, S), units = heads * ((R + rows - 1) / rows);
    if (rounds > 1) most = std::max(most, std::min(units * std::min<int64_t>(rounds, kMostRanges) * rows, most_part_rows(cache)));
  }
  PagedPlan p{};
  p.room_for(most, cache->Dh);
  return p.o_bytes + p.ml_bytes;
}

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
  float best = INFINITY;
  const float memory = (float)heads * (float)(S + M) * (float)(Dh * (bf16 ? 4 : 8)) / 9.e6f;   // (two thirds of the inputs were shorter than S)
  for (int i = 0; i < shapes(cache); ++i) {
    const Shape h = shape_of(cache, i);
    const int rows = rows_of(cache, h);
    if (!fits_rows(i, h, rows, R)) break;
    const int64_t row_blocks = (R + rows - 1) / rows, units = heads * row_blocks;
    const int tiles = (int)((S + h.kt - 1) / h.kt + (M + h.kt - 1) / h.kt), rounds = (int)rounds_of(h, M, S);
    const bool causal = M > LPP_MAX_ROWS;
    const float seen = causal ? 1.f - 0.5f * (float)((M + h.kt - 1) / h.kt) / (float)tiles : 1.f, full = causal ? 0.35f : 0.75f;
    int before = 0;
    for (const int g : kRanges) {
      const int per = (rounds + std::min(g, rounds) - 1) / std::min(g, rounds), ranges = (rounds + per - 1) / per;
      if (ranges == before) continue;                // (as many as the last choice)
      before = ranges;
      const int64_t blocks = units * ranges;
      if (ranges > 1 && blocks * rows > most_part_rows(cache)) break;                 // (32-bit offsets into the parts, too)
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
  p.room_for(p.nsplit > 1 ? heads * p.row_blocks * p.nsplit * p.rows : 0, Dh);
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
