// Attention of new tokens over a key/value cache in pages: the rows of a draft tree (paper App. A.2; every row sees the cache,
// its ancestors and itself) or causal chunks (row i of an item sees the cache and rows 0 .. i).
//
// The query heads that share a key/value head lie together: row r of a (item, key/value head) is query head r % gq of tree or
// chunk row r / gq, so that keys and values are read once for all of them and a single token fills as many rows of a matrix tile
// as it has heads in a group.
//
// bf16.  Tiles of KT keys, those of the cache first, then those of the new rows.
//   S^T[keys x rows] = K Q^T    (MFMA 32x32x16; a lane has one row and half of the keys)
//   softmax down the keys, almost all of it inside a lane; a row's reference maximum moves only when a score exceeds it by 2^8
//   O^T[Dh x rows] += V^T P^T   (P stays in the lane that formed it; V comes through the transposing LDS read)
// K and V go from memory to LDS without passing registers; the next tile's are on their way while one is worked on.  16-byte
// pieces of a row lie in LDS in an order that depends on the row (swizzle), so that neither product's reads meet on a bank; the
// order is made by where each lane reads from, as a wave's 64 pieces always land one behind the other.
// A weight is 2^(s scale - reference) by one fused operation, and the reference the rounded product of the largest s: half of its last
// place is in all of a row's exponents, 64 at scores of 10^9, which numbers and sums can take.
// Sums, maxima and accumulators are float32.  P is rounded to bf16 for the second product, as its inputs are; a row's sum is
// taken of the rounded weights.
//
// float32.  16 rows a block, its waves take 16-key tiles in turn, both products on the float32 matrix cores straight from the loads.
//
// A (item, key/value head)'s keys are cut into ranges where the launch would leave compute units idle; the block of a row tile
// that finishes last, or a launch of its own, adds the ranges' parts up in their order.
//
// What bounds it (replayed; a copy moves 4.95 TB/s here, a large bf16 product reaches 1138 TFLOP/s): single tokens over long
// caches the memory, 206 us and 5.5 TB/s for 16 items of 2048 to 32768 keys, 32 heads over 8 of 128.  Long chunks the matrix
// cores' feed, 394 us and 980 TFLOP/s for 2 x 2048 rows over 8192 and 4096 keys (matrix cores busy 47 % of the cycles, vector
// instructions 42 %, no bank conflicts).  Wide trees of heads of 64 the softmax, 64 us and 430 TFLOP/s for 16 trees of 129
// rows, 24 heads over 8, up to 4096 keys (vector instructions 54 %, matrix cores 25 %, one after the other in a wave: a tile's 16
// exponentials a lane, their products, maxima and sums take longer than its 8 matrix instructions; the keys and values that come
// in are 35 bytes a ns and compute unit of the 58 seen at most).  Small calls the latency of one round: 11 us for a token over 2400
// keys.
#include <math.h>

#include <algorithm>

#include "lpp_device.h"
#include "lpp_internal.h"
#include "lpp_overlap.h"
#include "lpp_paged_plan.h"
#include "lpp_reciprocal.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kMasked = -1.0e30f;  // finite stand-in for -inf
constexpr float kLazy = 8.0f;        // log2 of the largest weight before a rescale
constexpr float kLog2e = 1.44269504088896340736f;

struct PagedAttnArgs {
  const void* q; const void* kp; const void* vp; const void* kn; const void* vn;
  void* out;
  const int32_t* table; const int32_t* seq_len; const int32_t* row_len;
  const uint64_t* anc;               // tree, or null: a causal chunk
  int32_t words;
  int32_t Hkv, gq, M, S;
  uint32_t rc_gq;
  int32_t table_stride, page_shift, n_pages;
  int32_t row_blocks, nsplit, range; // blocks of rows of a (item, head); ranges of its keys, of so many tiles
  int32_t share;                     // items (at most 64) that are looked at by their own lengths: with ranges these are cut by them, without
                                     // the longest begin; 0: every item has nsplit ranges and its turn
  uint32_t units, whole;             // (item, head, range), and how many of them in eights
  float scale;                       // bf16: times log2 e
  float* ws_o;                       // [item, head, row block][nsplit][ROWS][Dh] unnormalised parts
  float* ws_ml;                      // [item, head, row block][nsplit][ROWS][2]  reference maximum and sum
  uint32_t ws_o_bytes, ws_ml_bytes;
  int32_t* counters;                 // [item, head, row block] zero between calls
  int32_t join_later;                // ranges are joined by a kernel of their own
};

// Sum of x over this lane and those before it.
__device__ __forceinline__ uint32_t sum_up_to(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, false);     // row_shr:1, 2, 4, 8: inside sixteen lanes
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false);     // row_bcast:15 into the second and fourth sixteen
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false);     // row_bcast:31 into the upper half
  return x;
}

// The items' lengths, lane i has item i's: cached keys, new rows, and the tiles of both.
struct Lengths {
  int seq, rows;
  uint32_t tiles;
  __device__ __forceinline__ Lengths(const PagedAttnArgs& a, int kt) {
    const int i = min((int)(threadIdx.x & 63), a.share - 1);
    seq = a.seq_len ? min(max(a.seq_len[i], 0), a.S) : a.S;
    rows = a.row_len ? min(max(a.row_len[i], 0), a.M) : a.M;
    tiles = rows > 0 ? (uint32_t)((seq + kt - 1) / kt + (rows + kt - 1) / kt) : 0u;
  }
};

// The item whose turn is number `turn` when the longest begin, so that what is left at the end is short.  (8 chunks of 512
// rows, 32 heads over 8 of 128 numbers, up to 8192 keys: in the batch's order 335 us if that is the shortest first, 279
// shuffled, 264 the longest first; so 262 in any order.  16 trees of 129 rows, 24 heads over 8 of 64, up to 4096 keys: 71.8,
// 67.7 and 62.5; so 63.3.)
__device__ __forceinline__ int longest_first(const Lengths& len, int items, int turn) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int j = 0; j < items; ++j) {
    const uint32_t t = (uint32_t)__builtin_amdgcn_readlane((int)len.tiles, j);
    before += t > len.tiles || (t == len.tiles && j < lane) ? 1 : 0;
  }
  return __ffsll(__ballot(before == turn && lane < items)) - 1;
}

// Ranges cut by the lengths that the device alone knows: the plan's blocks are for items of S keys each, and where items are shorter
// the same blocks take ranges as much shorter, down to half (an item then has up to twice as many, which one block may have to
// add up).  All items' ranges are of one size, the least that leaves no more ranges than there are blocks.  Lane i has item i.
// (16 single tokens, 32 heads over 8 of 128 numbers, 2048 to 32768 keys: 206 us, 227 with ranges for 32768 keys.)
struct Shares {
  uint32_t n, end;                   // my item's ranges, and those of all items up to it
  int range;                         // tiles
  __device__ __forceinline__ Shares(const PagedAttnArgs& a, const Lengths& len, int wk) {
    const uint32_t tiles = (int)(threadIdx.x & 63) < a.share ? len.tiles : 0u;
    const uint32_t rounds = (tiles + (uint32_t)wk - 1) / (uint32_t)wk, slots = (uint32_t)(a.share * a.nsplit);
    const uint32_t most = (uint32_t)(a.range / wk), all = (uint32_t)__builtin_amdgcn_readlane((int)sum_up_to(rounds), 63);
    uint32_t per = max((most + 1) / 2, (all + slots - 1) / slots);
    for (;; per = min(most, per + max(per >> 3, 1u))) {              // (at `most` no item has more than nsplit)
      n = (rounds + per - 1) / per;
      end = sum_up_to(n);
      if (per >= most || (uint32_t)__builtin_amdgcn_readlane((int)end, 63) <= slots) break;
    }
    range = (int)per * wk;
  }
  __device__ __forceinline__ int item_of(uint32_t u) const { return __popcll(__ballot(end <= u)); }   // whose range is number u
  __device__ __forceinline__ uint32_t ranges(int b) const { return (uint32_t)__builtin_amdgcn_readlane((int)n, b); }
  __device__ __forceinline__ uint32_t before(int b) const { return (uint32_t)__builtin_amdgcn_readlane((int)(end - n), b); }
};

// By how much the order of n things turns from one i to the next, i n + j being on XCD number (i n + j) mod 8, so that every j
// is on all XCDs.
__device__ __forceinline__ uint32_t turn(uint32_t i, uint32_t n) { return i * min(n & (0u - n), 8u) >> 3; }

// What a block works on.  The row blocks of a (item, head, range) read the same keys and sit on one XCD (block index mod 8) one
// behind the other, as long as there are eight such units; the rest spread over the XCDs.
struct Cell {
  int b, kvh, kvbh, rb, split, range;
  int seq, rows;                     // cached keys, new rows of the item
  uint32_t part;                     // the row tile's parts in the workspace: the first one's number
  __device__ __forceinline__ explicit Cell(const PagedAttnArgs& a, int kt, int wk) {
    const uint32_t id = blockIdx.x, RB = (uint32_t)a.row_blocks;
    uint32_t u;
    if (id < a.whole * RB) {
      const uint32_t n = id >> 3, e = n / RB;
      u = e * 8 + (id & 7);
      rb = (int)(n - e * RB);
    } else {
      const uint32_t t = id - a.whole * RB, left = a.units - a.whole;
      rb = (int)(t / left);
      u = a.whole + t - (uint32_t)rb * left;
    }
    range = a.range;
    uint32_t n = (uint32_t)a.nsplit, first;          // the item's ranges, the units before it
    if (a.share && n == 1) {
      const Lengths len(a, kt);
      b = longest_first(len, a.share, (int)(u / (uint32_t)a.Hkv));
      first = u / (uint32_t)a.Hkv * (uint32_t)a.Hkv;
      seq = __builtin_amdgcn_readlane(len.seq, b);
      rows = __builtin_amdgcn_readlane(len.rows, b);
    } else if (a.share) {
      const Lengths len(a, kt);
      const Shares sh(a, len, wk);
      b = sh.item_of(u / (uint32_t)a.Hkv);
      if (b >= a.share) {                            // behind the last range
        b = kvh = kvbh = split = seq = rows = 0;
        return;
      }
      range = sh.range;
      n = sh.ranges(b);
      first = sh.before(b) * (uint32_t)a.Hkv;
      seq = __builtin_amdgcn_readlane(len.seq, b);
      rows = __builtin_amdgcn_readlane(len.rows, b);
    } else {
      b = (int)(u / (n * (uint32_t)a.Hkv));
      first = (uint32_t)b * n * (uint32_t)a.Hkv;
      seq = a.seq_len ? min(max(a.seq_len[b], 0), a.S) : a.S;
      rows = a.row_len ? min(max(a.row_len[b], 0), a.M) : a.M;
    }
    kvh = (int)((u - first) / n);
    kvbh = b * a.Hkv + kvh;
    // (a head's ranges in an order that turns with the head, so that no XCD has all the first or all the last, which are shorter)
    split = (int)((u - first - (uint32_t)kvh * n + turn((uint32_t)kvbh, n)) % n);
    if (!a.anc) rb = a.row_blocks - 1 - rb;          // a chunk's last rows see most: first
    part = (first + (uint32_t)kvh * n) * RB + (uint32_t)rb * n;
  }
};

// Table entry of a position (past the last: of the last), and the page it names.
__device__ __forceinline__ int entry_of(const PagedAttnArgs& a, int b, int pos, int seq) {
  typedef const __attribute__((address_space(4))) int32_t* table_t;      // scalar loads, whatever is written meanwhile
  return ((table_t)(uintptr_t)a.table)[(int64_t)b * a.table_stride + (min(pos, seq - 1) >> a.page_shift)];
}
__device__ __forceinline__ int page_of(const PagedAttnArgs& a, int entry) { return min(max(entry, 0), a.n_pages - 1); }

// Whether row i sees new key t, 32 of them from t0 on (t0 a multiple of 32).
__device__ __forceinline__ uint32_t sees32(const PagedAttnArgs& a, int row, int t0) {
  if (a.anc) return (uint32_t)(a.anc[(int64_t)row * a.words + (t0 >> 6)] >> (t0 & 63));
  const int n = row - t0 + 1;
  return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u;
}
__device__ __forceinline__ bool sees(const PagedAttnArgs& a, int row, int t) { return (sees32(a, row, t & ~31) >> (t & 31)) & 1u; }

// Infinities and NaN among the new values went into the products as zeros, so that rows that do not see them stay clean; here
// the rows that do get them: four numbers from dimension d of row i, new keys [t0, t1).
template <typename T>
__device__ __forceinline__ void add_odd(const PagedAttnArgs& a, const T* v, int DH, int row, int d, int t0, int t1, float4& o) {
  for (int t = t0; t < t1; ++t) {
    if (!sees(a, row, t)) continue;
    const T* p = v + (int64_t)t * DH + d;
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = sizeof(T) == 2 ? __uint_as_float((uint32_t)p[e] << 16) : __builtin_bit_cast(float, (uint32_t)p[e]);
    o.x += isfinite(x[0]) ? 0.f : x[0]; o.y += isfinite(x[1]) ? 0.f : x[1];
    o.z += isfinite(x[2]) ? 0.f : x[2]; o.w += isfinite(x[3]) ? 0.f : x[3];
  }
}

__device__ __forceinline__ void store_row4(void* out, bool as_bf16, int64_t e, float4 v) {
  if (as_bf16) *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(out) + e) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
  else *reinterpret_cast<float4*>(reinterpret_cast<float*>(out) + e) = v;
}

// Element index of row r of a (item, key/value head) in q and out.
template <int DH>
__device__ __forceinline__ int64_t row_at(const PagedAttnArgs& a, int kvbh, int r, int* m) {
  const int i = (int)div_or_rc((uint32_t)r, (uint32_t)a.gq, a.rc_gq);
  *m = i;
  return (((int64_t)kvbh * a.gq + (r - i * a.gq)) * a.M + i) * DH;
}

// What a part is multiplied by whose reference lies t below (at most 0): references are in units of log 2 for bf16.
template <bool BF16>
__device__ __forceinline__ float part_weight(float t) { return BF16 ? __builtin_amdgcn_exp2f(t) : exp_neg(t); }

// The parts of a row tile's key ranges, added up in their order by the block that finishes last: every wave waits until its own
// stores have completed, the barrier gathers the waves, then the ticket is taken; stores, ticket and loads are device-scope, so
// no cache is written back.
template <int DH, int ROWS, int THREADS, bool BF16>
__device__ __forceinline__ void join_ranges(const PagedAttnArgs& a, const Cell& c, int r0, int R, int ns) {
  __shared__ int s_ticket;
  const int tile = c.kvbh * a.row_blocks + c.rb;
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0)
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __syncthreads();
  if (threadIdx.x == 0) s_ticket = __hip_atomic_fetch_add(&a.counters[tile], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (s_ticket != ns - 1) return;
  constexpr int C4 = DH / 4;
  const __amdgpu_buffer_rsrc_t dev_o = device_buffer(a.ws_o, a.ws_o_bytes), dev_ml = device_buffer(a.ws_ml, a.ws_ml_bytes);
  const uint32_t part0 = c.part * ROWS;
  for (int idx = threadIdx.x; idx < ROWS * C4; idx += THREADS) {
    const int r = idx / C4, c4 = idx % C4;
    if (r0 + r >= R) continue;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float ll = 0.f, mm = kMasked;
    for (int s0 = 0; s0 < ns; s0 += 4) {               // (four ranges at a time: their loads are in flight together)
      float2 ml[4];
      float4 o[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t prow = part0 + (uint32_t)(min(s0 + u, ns - 1) * ROWS + r);
        ml[u] = load_dev2(dev_ml, prow * 8);
        o[u] = load_dev4(dev_o, (prow * DH + c4 * 4) * 4);
      }
      float nm = mm;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (s0 + u < ns) nm = fmaxf(nm, ml[u].x);
      const float keep = part_weight<BF16>(mm - nm);
      acc.x *= keep; acc.y *= keep; acc.z *= keep; acc.w *= keep; ll *= keep;
      mm = nm;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (s0 + u < ns) {
          const float f = part_weight<BF16>(ml[u].x - mm);
          ll += f * ml[u].y;
          acc.x += f * o[u].x; acc.y += f * o[u].y; acc.z += f * o[u].z; acc.w += f * o[u].w;
        }
    }
    const float inv = 1.0f / ll;
    int m;
    const int64_t e = row_at<DH>(a, c.kvbh, r0 + r, &m) + c4 * 4;
    store_row4(a.out, BF16, e, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
  }
  if (threadIdx.x == 0)   // ready for the next call
    __hip_atomic_store(&a.counters[tile], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The same for parts that are many, in a launch of its own: a lane has four numbers of a share of a row's ranges, shares are added in
// their order.
template <int DH, int ROWS, int SHARES, bool BF16>
__global__ __launch_bounds__(256) void paged_attn_join_kernel(PagedAttnArgs a, int kt, int wk) {
  constexpr int C4 = DH / 4, RPB = 256 / (C4 * SHARES), BPT = ROWS / RPB;    // rows of a block, blocks of a row tile
  __shared__ __align__(16) float4 s_o[RPB][SHARES][C4];
  __shared__ float s_m[RPB][SHARES], s_l[RPB][SHARES];
  const int mine = threadIdx.x / (C4 * SHARES);
  const int tile = (int)(blockIdx.x / BPT), r = (int)(blockIdx.x % BPT) * RPB + mine;
  const int kvbh = tile / a.row_blocks, rb = tile - kvbh * a.row_blocks, b = kvbh / a.Hkv, r0 = rb * ROWS;
  const int rows = a.row_len ? min(max(a.row_len[b], 0), a.M) : a.M, R = rows * a.gq;
  if (r0 + r - mine >= R) return;
  const int seq = a.seq_len ? min(max(a.seq_len[b], 0), a.S) : a.S;
  const int fresh = (int)div_or_rc((uint32_t)(min(r0 + ROWS, R) - 1), (uint32_t)a.gq, a.rc_gq) + 1;
  const int T = (seq + kt - 1) / kt + (fresh + kt - 1) / kt;
  int range = a.range;
  uint32_t n = (uint32_t)a.nsplit, first = (uint32_t)b * n * (uint32_t)a.Hkv;        // as in Cell
  if (a.share) {
    const Shares sh(a, Lengths(a, kt), wk);
    range = sh.range;
    n = sh.ranges(b);
    first = sh.before(b) * (uint32_t)a.Hkv;
  }
  const int ns = (T + range - 1) / range;
  if (ns == 1) return;                               // (the block wrote its rows itself)
  const int c4 = threadIdx.x % C4, share = threadIdx.x / C4 % SHARES;
  const int64_t part0 = (int64_t)((first + (uint32_t)(kvbh - b * a.Hkv) * n) * (uint32_t)a.row_blocks + (uint32_t)rb * n) * ROWS + min(r, R - 1 - r0);
  const float4* po = reinterpret_cast<const float4*>(a.ws_o);
  const float2* pm = reinterpret_cast<const float2*>(a.ws_ml);
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float ll = 0.f, mm = kMasked;
  for (int s0 = share; s0 < ns; s0 += 4 * SHARES) {
    float2 ml[4];
    float4 o[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t prow = part0 + (int64_t)min(s0 + u * SHARES, ns - 1) * ROWS;
      ml[u] = pm[prow];
      o[u] = po[prow * C4 + c4];
    }
    float nm = mm;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (s0 + u * SHARES < ns) nm = fmaxf(nm, ml[u].x);
    const float keep = part_weight<BF16>(mm - nm);
    acc.x *= keep; acc.y *= keep; acc.z *= keep; acc.w *= keep; ll *= keep;
    mm = nm;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (s0 + u * SHARES < ns) {
        const float f = part_weight<BF16>(ml[u].x - mm);
        ll += f * ml[u].y;
        acc.x += f * o[u].x; acc.y += f * o[u].y; acc.z += f * o[u].z; acc.w += f * o[u].w;
      }
  }
  s_o[mine][share][c4] = acc;
  if (c4 == 0) { s_m[mine][share] = mm; s_l[mine][share] = ll; }
  __syncthreads();
  if (share > 0 || r0 + r >= R) return;
  float top = kMasked;
#pragma unroll
  for (int w = 0; w < SHARES; ++w) top = fmaxf(top, s_m[mine][w]);
  acc = make_float4(0.f, 0.f, 0.f, 0.f);
  ll = 0.f;
#pragma unroll
  for (int w = 0; w < SHARES; ++w) {
    const float f = part_weight<BF16>(s_m[mine][w] - top);
    const float4 o = s_o[mine][w][c4];
    ll += f * s_l[mine][w];
    acc.x += f * o.x; acc.y += f * o.y; acc.z += f * o.z; acc.w += f * o.w;
  }
  const float inv = 1.0f / ll;
  int m;
  const int64_t e = row_at<DH>(a, kvbh, r0 + r, &m) + c4 * 4;
  store_row4(a.out, BF16, e, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
}

// ---------------------------------------------------------------- bf16

// 64 pieces of 16 bytes from memory to LDS: piece `lane` from rsrc's base + off to lds + 16 lane.
__device__ __forceinline__ void to_lds(u32x4 rsrc, uint32_t off, uint32_t lds) {
  // (the wait states between a scalar register's last write and a vector memory instruction that reads it are in here: the
  // compiler does not look inside)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(rsrc) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }   // reads and writes of LDS are done
template <int N>
__device__ __forceinline__ void wait_loads() {      // until at most N of this wave's are in flight
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ u32x4 buffer_at(uint64_t base) {
  return u32x4{(uint32_t)base, (uint32_t)(base >> 32) & 0xFFFFu, 0x7FFFFFFFu, 0x00020000u};
}

// Which 16-byte piece of row `row` piece c of it lies at: c ^ swizzle.  Rows of 128 bytes (8 pieces) and of 256 (16): eight
// rows that follow each other are at eight places for the first product's reads, and the 64 bytes that the second one reads of
// each of eight rows fill the banks evenly.
template <int DH>
__device__ __forceinline__ constexpr int swizzle(int row) {
  return DH == 64 ? ((row >> 1 & 1) << 2) | ((row >> 2 & 1) << 1) | (row >> 3 & 1) : ((row & 3) << 2) | (row >> 2 & 3);
}

// 32 rows a wave, WR waves along the rows (they share the tiles of keys), WK along the keys (each has its own tiles), ST places for a
// tile.
template <int DH, int WR, int WK, int KT, int ST>
__global__ __launch_bounds__(WR * WK * 64) void paged_attn_bf16_kernel(PagedAttnArgs a) {
  constexpr int W = WR * WK, ROWS = WR * 32;
  constexpr int KS = DH / 16, DT = DH / 32, SUB = KT / 32;
  constexpr int CPR = DH / 8;                        // pieces of a row
  constexpr int PITCH = DH * 2;
  constexpr int TILE = KT * PITCH;                   // bytes of K, and of V, of a tile
  constexpr int RPI = 64 / CPR;                      // rows of a load
  constexpr int NI = TILE / 1024 / WR;               // loads of K, and of V, of a tile and wave
  constexpr int RG = NI * RPI < 16 ? NI * RPI : 16;  // ... in groups of so many rows: of one page
  constexpr int GROUPS = NI * RPI / RG;
  static_assert(WR > 1 || KT == 32, "a wave by itself takes a tile at once");
  static_assert(NI >= 1 && NI * RPI % RG == 0 && 16 % RG == 0, "whole groups of rows, none over a page's end");
  constexpr int OPITCH = DH + 4;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float s_m[WK][ROWS], s_l[WK][ROWS];
  __shared__ int s_odd;

  const Cell c(a, KT, WK);
  const int R = c.rows * a.gq, r0 = c.rb * ROWS;
  if (r0 >= R) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
  const int wr = wave % WR, kw = wave / WR;
  const int m_first = (int)div_or_rc((uint32_t)r0, (uint32_t)a.gq, a.rc_gq);
  const int m_last = (int)div_or_rc((uint32_t)(min(r0 + ROWS, R) - 1), (uint32_t)a.gq, a.rc_gq);
  const int fresh = m_last + 1;                      // new keys that the block's rows can see: [0, fresh) (a tree's ancestors come first)
  const int seq = c.seq;
  const int TC = (seq + KT - 1) / KT, T = TC + (fresh + KT - 1) / KT;
  const int ns = (T + c.range - 1) / c.range;
  if (c.split >= ns) return;
  const int tbeg = c.split * c.range, tend = min(tbeg + c.range, T);
  if (threadIdx.x == 0) s_odd = 0;

  // Q as the B operand: column = row, 8 consecutive Dh a lane and step
  bf16x8 qb[KS];
  int mrow;
  {
    const int64_t e = row_at<DH>(a, c.kvbh, min(r0 + wr * 32 + l32, R - 1), &mrow);
    const uint16_t* p = reinterpret_cast<const uint16_t*>(a.q) + e + half * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qb[ks] = *reinterpret_cast<const bf16x8*>(p + ks * 16);
  }

  // loads: my piece of a group's rows; the row's part of the swizzle that a load's number decides comes on top
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int lrow = lane / CPR;
  const uint32_t loff = (uint32_t)(((lane % CPR) ^ swizzle<DH>(lrow)) * 16);
  const uint64_t page_bytes = (uint64_t)PITCH << a.page_shift;
  const uint64_t kn = (uint64_t)(uintptr_t)a.kn + (uint64_t)c.kvbh * a.M * PITCH, vn = (uint64_t)(uintptr_t)a.vn + (uint64_t)c.kvbh * a.M * PITCH;
  int entry[GROUPS], ahead[GROUPS];                  // table entries of the next tile to load, and of the one behind it
  auto look_up = [&](int (&e)[GROUPS], int tile) {
    if (tile >= TC || tile >= tend) return;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) e[g] = entry_of(a, c.b, tile * KT + (wr * GROUPS + g) * RG, seq);
  };
  auto load_tile = [&](int tile, int stage, bool keys, bool values) {
    const uint32_t dst = lds0 + (uint32_t)((stage * WK + kw) * 2 * TILE + wr * NI * 1024);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int row0 = (wr * GROUPS + g) * RG;       // inside the tile
      uint64_t k0 = kn, v0 = vn;
      if (tile < TC) {
        const uint64_t at = ((uint64_t)page_of(a, entry[g]) * a.Hkv + c.kvh) * page_bytes +
                            (uint64_t)(((tile * KT + row0) & ((1 << a.page_shift) - 1)) * PITCH);
        k0 = (uint64_t)(uintptr_t)a.kp + at;
        v0 = (uint64_t)(uintptr_t)a.vp + at;
      }
      const u32x4 kr = buffer_at(k0), vr = buffer_at(v0);
#pragma unroll
      for (int i = 0; i < RG / RPI; ++i) {
        const uint32_t piece = loff ^ (uint32_t)(swizzle<DH>((RG < 16 ? row0 & 15 : 0) + i * RPI) * 16);
        const uint32_t off = piece + (uint32_t)((tile < TC ? i * RPI + lrow : min((tile - TC) * KT + row0 + i * RPI + lrow, a.M - 1)) * PITCH);
        const uint32_t to = dst + (uint32_t)((g * (RG / RPI) + i) * 1024);
        if (keys) to_lds(kr, off, to);
        if (values) to_lds(vr, off, to + TILE);
      }
    }
  };

  f32x16 oacc[DT];
  float m_ref = kMasked, l_sum = 0.f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[dt][r] = 0.f;
  // where I read K: my row, piece 2 ks + half; and V: four numbers of the row that the transposing read wants of me
  const uint32_t kread = (uint32_t)(l32 * PITCH + ((half ^ swizzle<DH>(l32)) * 16));
  const int vrow = 4 * half + (l16 >> 2), vpiece = 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1);
  const uint32_t vread = (uint32_t)(vrow * PITCH + ((vpiece ^ swizzle<DH>(vrow)) * 16) + (l16 & 1) * 8);
  const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
  bool odd = false;

  auto scores = [&](const unsigned char* base, int kt) {
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
    bf16x8 ka[KS];                                   // (all asked for before the first product: left to the compiler, two at a time)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) ka[ks] = *reinterpret_cast<const bf16x8*>(base + kt * 32 * PITCH + (kread ^ (uint32_t)(ks * 32)));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[ks], qb[ks], s, 0, 0, 0);
    return s;
  };
  // Weights of 32 keys: I hold keys 8 (r / 4) + 4 half + r % 4 of column l32.  (One copy of this code for whole tiles and
  // others: with two, the accumulators were moved from one's registers to the other's, 396 us instead of 378 for two chunks of
  // 2048 rows.)
  auto weights = [&](int tile, int kt, bool full, f32x16 s, bf16x8 (&pb)[2]) {
    if (!full) {
      const bool is_new = tile >= TC;
      const int key0 = (is_new ? tile - TC : tile) * KT + kt * 32, left = (is_new ? fresh : seq) - key0;
      uint32_t bits = left >= 32 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << left) - 1u;
      if (is_new && left > 0) bits &= sees32(a, mrow, key0);
      bits >>= 4 * half;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = (bits >> (8 * (r >> 2) + (r & 3))) & 1u ? s[r] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
    mx = fmaxf(mx * a.scale, kMasked);               // (scale > 0: the maximum commutes with it; the product alone may lie far below)
    if (__ballot(mx > m_ref + kLazy)) {              // some row's reference moves: rare behind the first tile
      const float v = fmaxf(mx, __shfl_xor(mx, 32));
      const float nm = v > m_ref + kLazy ? v : m_ref;
      const float alpha = __builtin_amdgcn_exp2f(m_ref - nm);
      m_ref = nm;
      l_sum *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) oacc[dt] *= alpha;
    }
    uint32_t pk[8];
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.scale, -m_ref));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r + 1], a.scale, -m_ref));
      pk[r / 2] = pack_bf16(p0, p1);
      l_sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk[r / 2]), ones, l_sum, false);
    }
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) pb[s2] = __builtin_bit_cast(bf16x8, make_uint4(pk[4 * s2], pk[4 * s2 + 1], pk[4 * s2 + 2], pk[4 * s2 + 3]));
  };
  auto read_values = [&](const unsigned char* base, int kt, bf16x8 (&va)[2][DT]) {
    typedef s16x4 __attribute__((address_space(3))) * lds_t;
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const __attribute__((address_space(3))) unsigned char* src =
            (const __attribute__((address_space(3))) unsigned char*)(base + TILE + (kt * 32 + 16 * s2) * PITCH);
        const uint32_t at = vread ^ (uint32_t)(dt * 64);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(src + at));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(src + 8 * PITCH + (at ^ (uint32_t)(swizzle<DH>(8) * 16))));
        const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
        va[s2][dt] = __builtin_bit_cast(bf16x8, make_uint4(l2.x, l2.y, h2.x, h2.y));
      }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto add_values = [&](const bf16x8 (&va)[2][DT], const bf16x8 (&pb)[2]) {
    // contraction slot (half, j) of step s2 is key 16 s2 + (j < 4 ? 0 : 8) + 4 half + j % 4 on both sides
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[s2][dt], pb[s2], oacc[dt], 0, 0, 0);
  };
  // A tile with keys that are not there, or that some row does not see: values of the former become zeros (their slots may hold
  // anything), and so do infinities and NaN among new ones (see add_odd).
  auto clean = [&](int tile, unsigned char* values) {
    const bool is_new = tile >= TC;
    const int here = (is_new ? fresh - (tile - TC) * KT : seq - tile * KT);
    for (int p = wr * 64 + lane; p < KT * CPR; p += WR * 64) {
      uint4* at = reinterpret_cast<uint4*>(values + p * 16);
      if (p / CPR >= here) {
        *at = make_uint4(0, 0, 0, 0);
      } else if (is_new) {
        uint32_t w[4] = {at->x, at->y, at->z, at->w};
        bool found = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if ((w[e] & 0x7F80u) == 0x7F80u) { w[e] &= 0xFFFF0000u; found = true; }
          if ((w[e] & 0x7F800000u) == 0x7F800000u) { w[e] &= 0xFFFFu; found = true; }
        }
        if (found) { *at = make_uint4(w[0], w[1], w[2], w[3]); odd = true; }
      }
    }
  };
  // (only the last tile of the cache, where it is not whole, and new ones: all of a tree's, of a chunk's those that some row of
  // the block is ahead of)
  const int part_tile = seq % KT != 0 ? TC - 1 : T, masked0 = TC + (a.anc ? 0 : (m_first + 1) / KT);
  auto is_full = [&](int tile) { return tile != part_tile && tile < masked0; };

  __syncthreads();                                   // (s_odd is cleared before any wave sets it)
  // Q has arrived before the first load to LDS is issued: a wait for it inside the loop would wait for those as well
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) entry[g] = ahead[g] = 0;
  look_up(entry, tbeg + kw);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qb[ks]));
  if (tbeg + kw < tend) {                            // (the keys' loads first: they are waited for by their number)
    load_tile(tbeg + kw, 0, true, false);
    load_tile(tbeg + kw, 0, false, true);
  }
  look_up(entry, tbeg + kw + WK);
  if (WR == 1) {
    // A wave by itself, one place for its tile: the next tile's keys go where this one's were as soon as the scores are formed,
    // the values likewise.  (Two places would halve the waves that a compute unit holds; one wave waits where another works.)
    unsigned char* base = smem + kw * 2 * TILE;
    for (int tile = tbeg + kw; tile < tend; tile += WK) {
      const bool more = tile + WK < tend, full = is_full(tile);
      look_up(ahead, tile + 2 * WK);                 // (they arrive while the tile is waited for)
      wait_loads<NI>();                              // the keys; the values may be on their way
      bf16x8 pb[2], va[2][DT];
      const f32x16 s = scores(base, 0);
      wait_lds();
      if (more) load_tile(tile + WK, 0, true, false);
      weights(tile, 0, full, s, pb);
      if (more) wait_loads<NI>();                    // the values
      else wait_loads<0>();
      if (!full) {
        clean(tile, base + TILE);
        wave_lds_sync();
      }
      read_values(base, 0, va);
      add_values(va, pb);
      wait_lds();
      if (more) load_tile(tile + WK, 0, false, true);
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) entry[g] = ahead[g];
    }
  } else {
    int stage = 0;
#pragma unroll
    for (int d = 1; d < ST - 1; ++d) {
      if (tbeg + kw + d * WK < tend) load_tile(tbeg + kw + d * WK, d, true, true);
      look_up(entry, tbeg + kw + (d + 1) * WK);
    }
    for (int first = tbeg; first < tend; first += WK) { // (the same rounds for all waves: they meet in them)
      const int tile = first + kw;
      look_up(ahead, tile + ST * WK);
      if (tile + (ST - 2) * WK < tend) wait_loads<(ST - 2) * 2 * NI>();
      else wait_loads<0>();
      __syncthreads();                               // the tile is there, and everybody is done with the one before it
      if (tile + (ST - 1) * WK < tend) load_tile(tile + (ST - 1) * WK, (stage + ST - 1) % ST, true, true);
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) entry[g] = ahead[g];
      unsigned char* base = smem + (stage * WK + kw) * 2 * TILE;
      const int last = min(first + WK, tend) - 1;
      const bool all_full = (part_tile < first || part_tile > last) && last < masked0;
      const bool full = is_full(tile);
      if (!all_full) {
        if (tile < tend && !full) clean(tile, base + TILE);
        __syncthreads();
      }
      if (tile < tend && r0 + wr * 32 < R) {         // (a wave behind the last row only loads)
#pragma unroll
        for (int kt = 0; kt < SUB; ++kt) {
          bf16x8 pb[2], va[2][DT];
          const f32x16 s = scores(base, kt);
          read_values(base, kt, va);
          weights(tile, kt, full, s, pb);
          add_values(va, pb);
        }
      }
      stage = stage + 1 == ST ? 0 : stage + 1;
    }
  }
  l_sum += __shfl_xor(l_sum, 32);
  if (odd) s_odd = 1;

  const int new0 = max(tbeg - TC, 0) * KT, new1 = min(max(tend - TC, 0) * KT, fresh);    // new keys of this range
  const uint16_t* vnew = reinterpret_cast<const uint16_t*>(a.vn) + (int64_t)c.kvbh * a.M * DH;
  const __amdgpu_buffer_rsrc_t dev_o = device_buffer(a.ws_o, a.ws_o_bytes), dev_ml = device_buffer(a.ws_ml, a.ws_ml_bytes);
  const uint32_t part = (c.part + (uint32_t)c.split) * ROWS;
  if (WK == 1) {
    __syncthreads();
    const bool fix = s_odd != 0;
    const int r = wr * 32 + l32;
    if (r0 + r < R) {
      int m;
      const int64_t e = row_at<DH>(a, c.kvbh, r0 + r, &m);
      const float inv = ns == 1 ? 1.0f / l_sum : 1.0f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int d = dt * 32 + g * 8 + half * 4;
          float4 v = make_float4(oacc[dt][4 * g] * inv, oacc[dt][4 * g + 1] * inv, oacc[dt][4 * g + 2] * inv, oacc[dt][4 * g + 3] * inv);
          if (fix) add_odd(a, vnew, DH, m, d, new0, new1, v);
          if (ns == 1) store_row4(a.out, true, e + d, v);
          else store_dev(dev_o, ((part + r) * DH + d) * 4, v);
        }
      if (ns > 1 && half == 0) store_dev(dev_ml, (part + r) * 8, make_float2(m_ref, l_sum));
    }
  } else {
    // the waves' parts of the rows are added in their order
    const int col = wr * 32 + l32;
    if (half == 0) { s_m[kw][col] = m_ref; s_l[kw][col] = l_sum; }
    __syncthreads();                                 // every wave is done with its tiles too
    float* s_o = reinterpret_cast<float*>(smem);     // [WK][ROWS][OPITCH]
    float top = kMasked;
#pragma unroll
    for (int w = 0; w < WK; ++w) top = fmaxf(top, s_m[w][col]);
    const float f = __builtin_amdgcn_exp2f(m_ref - top);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(&s_o[(kw * ROWS + col) * OPITCH + dt * 32 + g * 8 + half * 4]) =
            make_float4(oacc[dt][4 * g] * f, oacc[dt][4 * g + 1] * f, oacc[dt][4 * g + 2] * f, oacc[dt][4 * g + 3] * f);
    __syncthreads();
    const bool fix = s_odd != 0;
    constexpr int C4 = DH / 4;
    for (int idx = threadIdx.x; idx < ROWS * C4; idx += W * 64) {
      const int r = idx / C4, c4 = idx % C4;
      if (r0 + r >= R) continue;
      float mm = kMasked, ll = 0.f;
#pragma unroll
      for (int w = 0; w < WK; ++w) mm = fmaxf(mm, s_m[w][r]);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < WK; ++w) {
        ll += __builtin_amdgcn_exp2f(s_m[w][r] - mm) * s_l[w][r];
        const float4 o = *reinterpret_cast<const float4*>(&s_o[(w * ROWS + r) * OPITCH + c4 * 4]);
        v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
      }
      int m;
      const int64_t e = row_at<DH>(a, c.kvbh, r0 + r, &m) + c4 * 4;
      if (fix) add_odd(a, vnew, DH, m, c4 * 4, new0, new1, v);
      if (ns == 1) {
        const float inv = 1.0f / ll;
        store_row4(a.out, true, e, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
      } else {
        store_dev(dev_o, ((part + r) * DH + c4 * 4) * 4, v);
        if (c4 == 0) store_dev(dev_ml, (part + r) * 8, make_float2(mm, ll));
      }
    }
  }
  if (ns == 1 || a.join_later) return;
  join_ranges<DH, ROWS, W * 64, true>(a, c, r0, R, ns);
}

// ---------------------------------------------------------------- float32

// A block is NT tiles of 16 rows; its W waves take the 16-key tiles of its range in turn.  Lane (i, g) of a wave holds of key i
// the dimensions 16 t + 4 g .. + 3, and of keys 4 g + r the values of dimensions 64 h + 4 i .. + 3: what its 16-byte loads
// bring is what both products want.  Single tokens over long caches are bound by memory (16 items of 2048 to 32768 keys, 32 heads
// over 8 of 128: 413 us, 5.5 TB/s), small calls by latency (a token over 2400 keys: 15 us), rows enough for two tiles, which share what
// is loaded, by matrix and vector instructions that follow each other and loads that are waited for at once (busy 60 % and 28 %
// of the cycles with 32 heads over 8 of 128, 1526 rows over 1380 keys: 604 us, 89 TFLOP/s of the 154 that a large product reaches).
template <int DH, int NT, int W>
__global__ __launch_bounds__(W * 64) void paged_attn_f32_kernel(PagedAttnArgs a) {
  constexpr int ROWS = 16 * NT, HT = DH / 64, P4 = DH / 4 + 1;
  extern __shared__ __align__(16) unsigned char smem[];
  float4* const s_o = reinterpret_cast<float4*>(smem);      // [W][ROWS][P4]
  __shared__ float s_m[W][ROWS], s_l[W][ROWS];
  __shared__ int s_odd;
  const Cell c(a, 16, W);
  const int R = c.rows * a.gq, r0 = c.rb * ROWS;
  if (r0 >= R) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  const int fresh = (int)div_or_rc((uint32_t)(min(r0 + ROWS, R) - 1), (uint32_t)a.gq, a.rc_gq) + 1;
  const int seq = c.seq, TC = (seq + 15) / 16, T = TC + (fresh + 15) / 16;
  const int ns = (T + c.range - 1) / c.range;
  if (c.split >= ns) return;
  const int tbeg = c.split * c.range, tend = min(tbeg + c.range, T);
  if (threadIdx.x == 0) s_odd = 0;
  int row[NT];
  f32x4 q[NT][DH / 16], acc[NT][4 * HT];
  float m[NT], l[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float* qp = reinterpret_cast<const float*>(a.q) + row_at<DH>(a, c.kvbh, min(r0 + nt * 16 + i, R - 1), &row[nt]);
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) q[nt][t] = *reinterpret_cast<const f32x4*>(qp + 16 * t + 4 * g);
#pragma unroll
    for (int d = 0; d < 4 * HT; ++d) acc[nt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[nt] = kMasked;
    l[nt] = 0.f;
  }
  __syncthreads();                                   // (s_odd is cleared before any wave sets it)
  const int64_t page_size = (int64_t)DH << a.page_shift;
  const int64_t new_at = (int64_t)c.kvbh * a.M * DH;
  bool odd = false;
  for (int tile = tbeg + wave; tile < tend; tile += W) {
    const bool is_new = tile >= TC;
    const int key0 = (is_new ? tile - TC : tile) * 16, limit = is_new ? fresh : seq;
    const float *kp, *vp;                              // of key key0
    if (is_new) {
      kp = reinterpret_cast<const float*>(a.kn) + new_at + (int64_t)key0 * DH;
      vp = reinterpret_cast<const float*>(a.vn) + new_at + (int64_t)key0 * DH;
    } else {
      const int64_t at = ((int64_t)page_of(a, entry_of(a, c.b, key0, seq)) * a.Hkv + c.kvh) * page_size + (int64_t)(key0 & ((1 << a.page_shift) - 1)) * DH;
      kp = reinterpret_cast<const float*>(a.kp) + at;
      vp = reinterpret_cast<const float*>(a.vp) + at;
    }
    const int last = min(15, limit - 1 - key0);        // (behind the last key: the last again, masked below)
    f32x4 k[DH / 16], v[4][HT];
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) k[t] = *reinterpret_cast<const f32x4*>(kp + min(i, last) * DH + 16 * t + 4 * g);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int h = 0; h < HT; ++h) v[r][h] = *reinterpret_cast<const f32x4*>(vp + min(4 * g + r, last) * DH + 64 * h + 4 * i);
    const uint32_t there = (limit - key0 >= 16 ? 0xFFFFu : (1u << (limit - key0)) - 1u) >> (4 * g);
    if (is_new || last < 15) {                         // what is not there counts as zeros, and so do infinities and NaN among new values (see add_odd)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int h = 0; h < HT; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool here = (there >> r) & 1u, off = is_new && here && !isfinite(v[r][h][e]);
            odd = odd || off;
            v[r][h][e] = here && !off ? v[r][h][e] : 0.f;
          }
    }
    float sc[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};                  // chains of Dh / 4 products, two at a time
#pragma unroll
      for (int t0 = 0; t0 < DH / 16; t0 += DH / 32) {
        f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = t0; t < t0 + DH / 32; t += 2)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t][e], q[nt][t][e], s0, 0, 0, 0);
            s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t + 1][e], q[nt][t + 1][e], s1, 0, 0, 0);
          }
        s += s0 + s1;
      }
      const uint32_t bits = is_new ? there & (sees32(a, row[nt], key0 & ~31) >> ((key0 & 31) + 4 * g)) : there;
      float mn = kMasked;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sc[nt][r] = (bits >> r) & 1u ? s[r] * a.scale : -INFINITY;
        mn = fmaxf(mn, sc[nt][r]);
      }
      mn = fmaxf(mn, __shfl_xor(mn, 16));
      mn = fmaxf(mn, __shfl_xor(mn, 32));
      mn = fmaxf(mn, m[nt]);
      if (__any(mn != m[nt])) {
        const float f = mn == m[nt] ? 1.f : exp_neg(m[nt] - mn);
        l[nt] *= f;
#pragma unroll
        for (int d = 0; d < 4 * HT; ++d) acc[nt][d] *= f;
        m[nt] = mn;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sc[nt][r] = sc[nt][r] == -INFINITY ? 0.f : exp_neg(sc[nt][r] - m[nt]);
        l[nt] += sc[nt][r];
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int h = 0; h < HT; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            acc[nt][4 * h + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][h][e], sc[nt][r], acc[nt][4 * h + e], 0, 0, 0);
  }
  if (odd) s_odd = 1;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    l[nt] += __shfl_xor(l[nt], 16);
    l[nt] += __shfl_xor(l[nt], 32);
    if (lane < 16) { s_m[wave][nt * 16 + lane] = m[nt]; s_l[wave][nt * 16 + lane] = l[nt]; }
#pragma unroll
    for (int h = 0; h < HT; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        s_o[(wave * ROWS + nt * 16 + i) * P4 + 16 * h + 4 * g + r] =
            make_float4(acc[nt][4 * h][r], acc[nt][4 * h + 1][r], acc[nt][4 * h + 2][r], acc[nt][4 * h + 3][r]);
  }
  __syncthreads();

  const __amdgpu_buffer_rsrc_t dev_o = device_buffer(a.ws_o, a.ws_o_bytes), dev_ml = device_buffer(a.ws_ml, a.ws_ml_bytes);
  const uint32_t part = (c.part + (uint32_t)c.split) * ROWS;
  for (int idx = threadIdx.x; idx < ROWS * DH / 4; idx += W * 64) {
    const int r = idx / (DH / 4), c4 = idx % (DH / 4);
    if (r0 + r >= R) continue;
    float mm = kMasked, ll = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) mm = fmaxf(mm, s_m[w][r]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = exp_neg(s_m[w][r] - mm);
      const float4 x = s_o[(w * ROWS + r) * P4 + c4];
      ll = __builtin_fmaf(f, s_l[w][r], ll);
      o.x = __builtin_fmaf(f, x.x, o.x); o.y = __builtin_fmaf(f, x.y, o.y); o.z = __builtin_fmaf(f, x.z, o.z); o.w = __builtin_fmaf(f, x.w, o.w);
    }
    int mr;
    const int64_t e = row_at<DH>(a, c.kvbh, r0 + r, &mr) + c4 * 4;
    if (s_odd) {
      const int new0 = max(tbeg - TC, 0) * 16, new1 = min(max(tend - TC, 0) * 16, fresh);
      add_odd(a, reinterpret_cast<const uint32_t*>(a.vn) + new_at, DH, mr, c4 * 4, new0, new1, o);
    }
    if (ns == 1) {
      store_row4(a.out, false, e, make_float4(o.x / ll, o.y / ll, o.z / ll, o.w / ll));
    } else {
      store_dev(dev_o, ((part + r) * DH + c4 * 4) * 4, o);
      if (c4 == 0) store_dev(dev_ml, (part + r) * 8, make_float2(mm, ll));
    }
  }
  if (ns == 1 || a.join_later) return;
  join_ranges<DH, ROWS, W * 64, false>(a, c, r0, R, ns);
}

// ---------------------------------------------------------------- host

template <typename K>
int32_t launch(K kern, LppLdsLimit& limit, const PagedAttnArgs& a, int threads, const PagedPlan& p, hipStream_t s) {
  const int32_t st = lpp_ensure_lds(reinterpret_cast<const void*>(kern), limit, p.lds, 48 * 1024);
  if (st != LPP_OK) return st;
  hipLaunchKernelGGL(kern, dim3(a.units * (uint32_t)a.row_blocks), dim3(threads), p.lds, s, a);
  LPP_HIP_TRY(hipGetLastError());
  return LPP_OK;
}
template <int DH, int ROWS, bool BF16>
int32_t launch_join(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  if (!a.join_later) return LPP_OK;
  const uint32_t tiles = a.units / (uint32_t)a.nsplit * (uint32_t)a.row_blocks;
  constexpr int C4 = DH / 4;
  if (a.nsplit <= 8) hipLaunchKernelGGL((paged_attn_join_kernel<DH, ROWS, 2, BF16>), dim3(tiles * (ROWS * C4 * 2 / 256)), dim3(256), 0, s, a, p.kt, p.wk);
  else hipLaunchKernelGGL((paged_attn_join_kernel<DH, ROWS, 256 / C4, BF16>), dim3(tiles * ROWS), dim3(256), 0, s, a, p.kt, p.wk);
  LPP_HIP_TRY(hipGetLastError());
  return LPP_OK;
}
template <int DH, int SHAPE>
int32_t launch_bf16(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  static LppLdsLimit limit;
  constexpr Shape h = kShapes[SHAPE];
  const int32_t st = launch(paged_attn_bf16_kernel<DH, h.wr, h.wk, h.kt, h.st>, limit, a, h.wr * h.wk * 64, p, s);
  return st != LPP_OK ? st : launch_join<DH, h.wr * 32, true>(a, p, s);
}
template <int DH, int NT>
int32_t launch_f32(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  static LppLdsLimit limit;
  constexpr int W = DH == 64 && NT == 1 ? 16 : 8;
  const int32_t st = launch(paged_attn_f32_kernel<DH, NT, W>, limit, a, W * 64, p, s);
  return st != LPP_OK ? st : launch_join<DH, NT * 16, false>(a, p, s);
}
template <int DH>
int32_t launch_paged(const lpp_paged* cache, const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  if (cache->dtype == LPP_F32) return p.shape == 0 ? launch_f32<DH, 1>(a, p, s) : launch_f32<DH, 2>(a, p, s);
  switch (p.shape) {
    case 0: return launch_bf16<DH, 0>(a, p, s);
    case 1: return launch_bf16<DH, 1>(a, p, s);
    case 2: return launch_bf16<DH, 2>(a, p, s);
    case 3: return launch_bf16<DH, 3>(a, p, s);
    default: return launch_bf16<DH, 4>(a, p, s);
  }
}

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

int32_t paged_attention(const lpp_paged* cache, const lpp_tree* tree, const void* q, const void* k_pages, const void* v_pages,
                        const int32_t* page_table, int32_t table_stride, const void* k_new, const void* v_new,
                        const int32_t* seq_len, const int32_t* row_len, int32_t B, int32_t H, int32_t M, int32_t S, float scale,
                        void* out, void* ws, size_t ws_bytes, void* stream) {
  if (!cache || !q || !k_new || !v_new || !out) return LPP_EINVAL;
  if (out == q || out == k_new || out == v_new || out == k_pages || out == v_pages) return LPP_EINVAL;      // (and see below)
  if (B < 1 || H < 1 || M < 1 || S < 0) return LPP_EINVAL;
  if (S > 0 && (!k_pages || !v_pages || !page_table || table_stride < 1)) return LPP_EINVAL;
  if (H % cache->Hkv != 0) return LPP_EINVAL;
  if (S > 0 && ((int64_t)table_stride << cache->page_shift) < S) return LPP_EINVAL;
  if (!(scale >= 0.f && scale <= 2e38f)) return LPP_EINVAL;                 // NaN, negative, infinite in base two
  if (misaligned(q) || misaligned(k_new) || misaligned(v_new) || misaligned(out) || misaligned(k_pages) || misaligned(v_pages)) return LPP_EINVAL;
  const int esz = cache->dtype == LPP_F32 ? 4 : 2, gq = H / cache->Hkv;
  // 32-bit offsets inside one head's new rows, row and key numbers, units and blocks
  if ((int64_t)M * cache->Dh * esz >= (1ll << 31) || (int64_t)M * gq >= (1ll << 30) || (int64_t)S + M >= (1ll << 30)) return LPP_EUNSUPPORTED;
  if ((int64_t)B * cache->Hkv >= (1ll << 24)) return LPP_EUNSUPPORTED;
  const PagedPlan p = plan_paged(cache, B, gq, M, S);
  const int64_t units = (int64_t)B * cache->Hkv * p.nsplit;
  const int waves = cache->dtype == LPP_BF16 ? p.rows / 32 * p.wk : p.wk;
  if (!lpp_launch_fits(units * p.row_blocks, waves * 64)) return LPP_EUNSUPPORTED;
  if (p.o_bytes > 0 && (!ws || misaligned(ws) || ws_bytes < paged_room(cache, B, gq, M, S))) return LPP_ENOWORKSPACE;
  if (!cache->d_counters || (tree && !tree->d_anc)) return LPP_EHIP;     // host-only handle: no device
  if (!lpp_is_current(cache->device) || (tree && tree->device != cache->device)) return LPP_EINVAL;
  // blocks read what others have finished, and parts that others have left: neither lies in an input or in the other
  const uint64_t row_bytes = (uint64_t)cache->Dh * esz, n_q = (uint64_t)B * H * M * row_bytes, n_new = (uint64_t)B * cache->Hkv * M * row_bytes;
  const uint64_t n_pool = S > 0 ? ((uint64_t)cache->n_pages * cache->Hkv << cache->page_shift) * row_bytes : 0;
  const uint64_t n_table = S > 0 ? (uint64_t)B * table_stride * 4 : 0, n_lens = (uint64_t)B * 4, n_parts = p.o_bytes + p.ml_bytes;
  const auto meets_input = [&](const void* x, uint64_t n) {
    return ranges_meet(x, n, q, n_q) || ranges_meet(x, n, k_new, n_new) || ranges_meet(x, n, v_new, n_new) || ranges_meet(x, n, k_pages, n_pool) ||
           ranges_meet(x, n, v_pages, n_pool) || ranges_meet(x, n, page_table, n_table) || ranges_meet(x, n, seq_len, n_lens) ||
           ranges_meet(x, n, row_len, n_lens);
  };
  if (meets_input(out, n_q) || meets_input(ws, n_parts) || ranges_meet(out, n_q, ws, n_parts)) return LPP_EINVAL;
  if (scale == 0.f) scale = 1.0f / sqrtf((float)cache->Dh);
  PagedAttnArgs a;
  a.q = q; a.kp = k_pages; a.vp = v_pages; a.kn = k_new; a.vn = v_new; a.out = out;
  a.table = page_table; a.seq_len = seq_len; a.row_len = row_len;
  a.anc = tree ? tree->d_anc : nullptr; a.words = tree ? tree->words : 0;
  a.Hkv = cache->Hkv; a.gq = gq; a.M = M; a.S = S;
  a.rc_gq = reciprocal((uint32_t)gq, (uint64_t)M * gq);
  a.table_stride = table_stride; a.page_shift = cache->page_shift; a.n_pages = cache->n_pages;
  a.row_blocks = p.row_blocks; a.nsplit = p.nsplit; a.range = p.range;
  a.share = (seq_len || row_len) && looks_at_lengths(cache, B, p) ? B : 0;
  a.units = (uint32_t)units; a.whole = (uint32_t)(units & ~7ll);
  a.scale = cache->dtype == LPP_F32 ? scale : scale * kLog2e;
  a.ws_o = reinterpret_cast<float*>(ws);
  a.ws_ml = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(ws) + p.o_bytes);
  a.ws_o_bytes = (uint32_t)p.o_bytes; a.ws_ml_bytes = (uint32_t)p.ml_bytes;
  a.counters = cache->d_counters;
  a.join_later = p.join_later;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return cache->Dh == 64 ? launch_paged<64>(cache, a, p, s) : launch_paged<128>(cache, a, p, s);
}

}  // namespace

extern "C" size_t lpp_paged_attention_workspace(const lpp_paged* cache, int32_t B, int32_t H, int32_t M, int32_t S) {
  if (!cache || B < 1 || H < 1 || M < 1 || S < 0 || H % cache->Hkv != 0) return 0;
  return std::max<size_t>(paged_room(cache, B, H / cache->Hkv, M, S), 256);
}

extern "C" int32_t lpp_paged_tree_attention(const lpp_paged* cache, const lpp_tree* tree, const void* q, const void* k_pages,
                                            const void* v_pages, const int32_t* page_table, int32_t table_stride,
                                            const void* k_tree, const void* v_tree, const int32_t* seq_len, int32_t B, int32_t H,
                                            int32_t S, float scale, void* out, void* ws, size_t ws_bytes, void* stream) {
  if (!tree) return LPP_EINVAL;
  return paged_attention(cache, tree, q, k_pages, v_pages, page_table, table_stride, k_tree, v_tree, seq_len, nullptr, B, H, tree->M, S,
                         scale, out, ws, ws_bytes, stream);
}

extern "C" int32_t lpp_paged_chunk_attention(const lpp_paged* cache, const void* q, const void* k_pages, const void* v_pages,
                                             const int32_t* page_table, int32_t table_stride, const void* k_new,
                                             const void* v_new, const int32_t* seq_len, const int32_t* row_len, int32_t B,
                                             int32_t H, int32_t M, int32_t S, float scale, void* out, void* ws, size_t ws_bytes,
                                             void* stream) {
  return paged_attention(cache, nullptr, q, k_pages, v_pages, page_table, table_stride, k_new, v_new, seq_len, row_len, B, H, M, S, scale,
                         out, ws, ws_bytes, stream);
}
