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
// Sums, maxima and accumulators are float32.  P is rounded to bf16 for the second product, as its inputs are; a row's sum is
// taken of the rounded weights.
//
// float32.  16 rows a block, its waves take 16-key tiles in turn, both products on the float32 matrix cores straight from the loads.
//
// A (item, key/value head)'s keys are cut into ranges where the launch would leave compute units idle; the block of a row tile
// that finishes last adds the ranges' parts up in their order.
#include <math.h>

#include <algorithm>

#include "lpp_device.h"
#include "lpp_internal.h"
#include "lpp_reciprocal.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kMasked = -1.0e30f;  // finite stand-in for -inf
constexpr float kLazy = 8.0f;        // log2 of the largest weight before a rescale

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
  uint32_t units, whole;             // (item, head, range), and how many of them in eights
  float scale;                       // bf16: times log2 e
  float* ws_o;                       // [item, head, row block][nsplit][ROWS][Dh] unnormalised parts
  float* ws_ml;                      // [item, head, row block][nsplit][ROWS][2]  reference maximum and sum
  uint32_t ws_o_bytes, ws_ml_bytes;
  int32_t* counters;                 // [item, head, row block] zero between calls
};

// What a block works on.  The row blocks of a (item, head, range) read the same keys and sit on one XCD (block index mod 8) one
// behind the other, as long as there are eight such units; the rest spread over the XCDs.
struct Cell {
  int b, kvh, kvbh, rb, split;
  int seq, rows;                     // cached keys, new rows of the item
  bool live;
  __device__ __forceinline__ explicit Cell(const PagedAttnArgs& a) {
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
    kvbh = (int)(u / (uint32_t)a.nsplit);
    split = (int)(u - (uint32_t)kvbh * (uint32_t)a.nsplit);
    b = kvbh / a.Hkv;
    kvh = kvbh - b * a.Hkv;
    seq = a.seq_len ? min(max(a.seq_len[b], 0), a.S) : a.S;
    rows = a.row_len ? min(max(a.row_len[b], 0), a.M) : a.M;
    if (!a.anc) rb = a.row_blocks - 1 - rb;          // a chunk's last rows see most: first
  }
};

__device__ __forceinline__ int page_of(const PagedAttnArgs& a, int b, int pos, int seq) {
  // (scalar loads, whatever is written meanwhile; positions past the last: its page again)
  typedef const __attribute__((address_space(4))) int32_t* table_t;
  const int page = ((table_t)(uintptr_t)a.table)[(int64_t)b * a.table_stride + (min(pos, seq - 1) >> a.page_shift)];
  return min(max(page, 0), a.n_pages - 1);
}

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

// The parts of a row tile's key ranges, added up in their order by the block that finishes last (`weight` of a difference of
// references, at most 0): every wave waits until its own stores have completed, the barrier gathers the waves, then
// the ticket is taken; stores, ticket and loads are device-scope, so no cache is written back.
template <int DH, int ROWS, int THREADS, bool BF16, typename W>
__device__ __forceinline__ void join_ranges(const PagedAttnArgs& a, const Cell& c, int r0, int R, int ns, W weight) {
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
  const uint32_t part0 = (uint32_t)tile * (uint32_t)a.nsplit * ROWS;
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
      const float keep = weight(mm - nm);
      acc.x *= keep; acc.y *= keep; acc.z *= keep; acc.w *= keep; ll *= keep;
      mm = nm;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (s0 + u < ns) {
          const float f = weight(ml[u].x - mm);
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

// ---------------------------------------------------------------- bf16

// 64 pieces of 16 bytes from memory to LDS: piece `lane` from rsrc's base + off to lds + 16 lane.
__device__ __forceinline__ void to_lds(u32x4 rsrc, uint32_t off, uint32_t lds) {
  // (the wait states between a scalar register's last write and a vector memory instruction that reads it are in here: the
  // compiler does not look inside)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(rsrc) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() {      // until at most N of this wave's are in flight
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ u32x4 buffer_at(uint64_t base) {
  return u32x4{(uint32_t)base, (uint32_t)(base >> 32) & 0xFFFFu, 0x7FFFFFFFu, 0x00020000u};
}

// Which 16-byte piece of row `row` piece c of it lies at: c ^ swizzle.  Rows of 128 bytes (8 pieces) and of 256 (16): eight rows
// that follow each other are at eight places for the first product's reads, and the 64 bytes that the second one reads of each of eight rows fill
// the banks evenly.
template <int DH>
__device__ __forceinline__ constexpr int swizzle(int row) {
  return DH == 64 ? ((row >> 1 & 1) << 2) | ((row >> 2 & 1) << 1) | (row >> 3 & 1) : ((row & 7) << 1) | (row >> 3 & 1);
}

// NT tiles of 32 rows a wave, WR waves along the rows (they share the tiles of keys), WK along the keys (each has its own tiles).
template <int DH, int NT, int WR, int WK, int KT>
__global__ __launch_bounds__(WR * WK * 64) void paged_attn_bf16_kernel(PagedAttnArgs a) {
  static_assert(WR == 1 || WK == 1, "barriers inside the loop over the keys");
  constexpr int W = WR * WK, ROWS = NT * WR * 32;
  constexpr int KS = DH / 16, DT = DH / 32, SUB = KT / 32;
  constexpr int CPR = DH / 8;                        // pieces of a row
  constexpr int PITCH = DH * 2;
  constexpr int TILE = KT * PITCH;                   // bytes of K, and of V, of a tile
  constexpr int RPI = 64 / CPR;                      // rows of a load
  constexpr int NI = TILE / 1024 / WR;               // loads of K, and of V, of a tile and wave
  constexpr int GROUPS = NI * RPI / 16;              // ... in groups of 16 rows: a page each at least
  static_assert(GROUPS >= 1 && NI * RPI % 16 == 0, "a wave loads whole groups of 16 rows");
  constexpr int OPITCH = DH + 4;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float s_m[W][NT * 32], s_l[W][NT * 32];
  __shared__ int s_odd;

  const Cell c(a);
  const int R = c.rows * a.gq, r0 = c.rb * ROWS;
  if (r0 >= R) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
  const int wr = WR > 1 ? wave : 0, kw = WK > 1 ? wave : 0;
  const int m_first = (int)div_or_rc((uint32_t)r0, (uint32_t)a.gq, a.rc_gq);
  const int m_last = (int)div_or_rc((uint32_t)(min(r0 + ROWS, R) - 1), (uint32_t)a.gq, a.rc_gq);
  const int fresh = m_last + 1;                      // new keys that the block's rows can see: [0, fresh) (a tree's ancestors come first)
  const int seq = c.seq;
  const int TC = (seq + KT - 1) / KT, T = TC + (fresh + KT - 1) / KT;
  const int ns = (T + a.range - 1) / a.range;
  if (c.split >= ns) return;
  const int tbeg = c.split * a.range, tend = min(tbeg + a.range, T);
  if (threadIdx.x == 0) s_odd = 0;

  // Q as the B operand: column = row, 8 consecutive Dh a lane and step
  bf16x8 qb[NT][KS];
  int mrow[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int64_t e = row_at<DH>(a, c.kvbh, min(r0 + (wr * NT + nt) * 32 + l32, R - 1), &mrow[nt]);
    const uint16_t* p = reinterpret_cast<const uint16_t*>(a.q) + e + half * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qb[nt][ks] = *reinterpret_cast<const bf16x8*>(p + ks * 16);
  }

  // loads: my piece of a group's rows; the row's part of the swizzle that a load's number decides comes on top
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int lrow = lane / CPR;
  const uint32_t loff = (uint32_t)(((lane % CPR) ^ swizzle<DH>(lrow)) * 16);
  const uint64_t page_bytes = (uint64_t)PITCH << a.page_shift;
  const uint64_t kn = (uint64_t)(uintptr_t)a.kn + (uint64_t)c.kvbh * a.M * PITCH, vn = (uint64_t)(uintptr_t)a.vn + (uint64_t)c.kvbh * a.M * PITCH;
  int page[GROUPS];                                  // of the next tile to load
  auto look_up = [&](int tile) {
    if (tile >= TC || tile >= tend) return;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) page[g] = page_of(a, c.b, tile * KT + (wr * GROUPS + g) * 16, seq);
  };
  auto load_tile = [&](int tile, int stage) {
    const uint32_t dst = lds0 + (uint32_t)((stage * WK + kw) * 2 * TILE + wr * NI * 1024);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int row0 = (wr * GROUPS + g) * 16;       // inside the tile
      u32x4 kr, vr;
      if (tile < TC) {
        const uint64_t at = ((uint64_t)page[g] * a.Hkv + c.kvh) * page_bytes +
                            (uint64_t)(((tile * KT + row0) & ((1 << a.page_shift) - 1)) * PITCH);
        kr = buffer_at((uint64_t)(uintptr_t)a.kp + at);
        vr = buffer_at((uint64_t)(uintptr_t)a.vp + at);
      } else {
        kr = buffer_at(kn);
        vr = buffer_at(vn);
      }
#pragma unroll
      for (int i = 0; i < 16 / RPI; ++i) {
        const uint32_t piece = loff ^ (uint32_t)(swizzle<DH>(i * RPI) * 16);
        const uint32_t off = piece + (uint32_t)((tile < TC ? i * RPI + lrow : min((tile - TC) * KT + row0 + i * RPI + lrow, a.M - 1)) * PITCH);
        const uint32_t to = dst + (uint32_t)((g * (16 / RPI) + i) * 1024);
        to_lds(kr, off, to);
        to_lds(vr, off, to + TILE);
      }
    }
  };

  f32x16 oacc[NT][DT];
  float m_ref[NT], l_sum[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m_ref[nt] = kMasked;
    l_sum[nt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[nt][dt][r] = 0.f;
  }
  // where I read K: my row, piece 2 ks + half; and V: four numbers of the row that the transposing read wants of me
  const uint32_t kread = (uint32_t)(l32 * PITCH + ((half ^ swizzle<DH>(l32)) * 16));
  const int vrow = 4 * half + (l16 >> 2), vpiece = 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1);
  const uint32_t vread = (uint32_t)(vrow * PITCH + ((vpiece ^ swizzle<DH>(vrow)) * 16) + (l16 & 1) * 8);
  const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
  bool odd = false;

  auto work = [&](int tile, const unsigned char* base, auto full_tag) {
    constexpr bool FULL = decltype(full_tag)::value;
    const bool is_new = tile >= TC;
    const int key0 = (is_new ? tile - TC : tile) * KT, limit = is_new ? fresh : seq;
#pragma unroll
    for (int kt = 0; kt < SUB; ++kt) {
      f32x16 s[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[nt][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 ka = *reinterpret_cast<const bf16x8*>(base + kt * 32 * PITCH + (kread ^ (uint32_t)(ks * 32)));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qb[nt][ks], s[nt], 0, 0, 0);
      }
      // weights: I hold keys 8 (r / 4) + 4 half + r % 4 of column l32
      uint32_t bits[NT];
      float mx[NT];
      bool need = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        bits[nt] = 0xFFFFFFFFu;
        if (!FULL) {
          const int left = limit - key0 - kt * 32;
          bits[nt] = left >= 32 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << left) - 1u;
          if (is_new && left > 0) bits[nt] &= sees32(a, mrow[nt], key0 + kt * 32);
          bits[nt] >>= 4 * half;
        }
        float v = kMasked;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float x = s[nt][r];
          if (!FULL && !((bits[nt] >> (8 * (r >> 2) + (r & 3))) & 1u)) x = kMasked;
          v = fmaxf(v, x);
        }
        mx[nt] = v > 0.5f * kMasked ? v * a.scale : kMasked;       // (scale > 0: the maximum commutes with it)
        need = need || mx[nt] > m_ref[nt] + kLazy;
      }
      if (__ballot(need)) {                          // some row's reference moves: rare behind the first tile
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float v = fmaxf(mx[nt], __shfl_xor(mx[nt], 32));
          const float nm = v > m_ref[nt] + kLazy ? v : m_ref[nt];
          const float alpha = __builtin_amdgcn_exp2f(m_ref[nt] - nm);
          m_ref[nt] = nm;
          l_sum[nt] *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) oacc[nt][dt] *= alpha;
        }
      }
      bf16x8 pb[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        uint32_t pk[8];
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nt][r], a.scale, -m_ref[nt]));
          float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nt][r + 1], a.scale, -m_ref[nt]));
          if (!FULL) {
            if (!((bits[nt] >> (8 * (r >> 2) + (r & 3))) & 1u)) p0 = 0.f;
            if (!((bits[nt] >> (8 * (r >> 2) + (r & 3) + 1)) & 1u)) p1 = 0.f;
          }
          pk[r / 2] = pack_bf16(p0, p1);
          l_sum[nt] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk[r / 2]), ones, l_sum[nt], false);
        }
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) pb[nt][s2] = __builtin_bit_cast(bf16x8, make_uint4(pk[4 * s2], pk[4 * s2 + 1], pk[4 * s2 + 2], pk[4 * s2 + 3]));
      }
      // contraction slot (half, j) of step s2 is key 16 s2 + (j < 4 ? 0 : 8) + 4 half + j % 4 on both sides
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const unsigned char* src = base + TILE + (kt * 32 + 16 * s2) * PITCH;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (s16x4 __attribute__((address_space(3)))*)(const __attribute__((address_space(3))) unsigned char*)(src + (vread ^ (uint32_t)(dt * 64))));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (s16x4 __attribute__((address_space(3)))*)(const __attribute__((address_space(3))) unsigned char*)(
                  src + 8 * PITCH + (vread ^ (uint32_t)(dt * 64) ^ (uint32_t)(swizzle<DH>(8) * 16))));
          const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
          const bf16x8 va = __builtin_bit_cast(bf16x8, make_uint4(l2.x, l2.y, h2.x, h2.y));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) oacc[nt][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pb[nt][s2], oacc[nt][dt], 0, 0, 0);
        }
    }
  };
  // A tile with keys that are not there, or that some row does not see: values of the former become zeros (their slots may hold
  // anything), and so do infinities and NaN among new ones (see add_odd).
  auto clean = [&](int tile, unsigned char* values) {
    const bool is_new = tile >= TC;
    const int here = (is_new ? fresh - (tile - TC) * KT : seq - tile * KT);
    for (int p = WR > 1 ? (int)threadIdx.x : lane; p < KT * CPR; p += WR * 64) {
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
    if (WR > 1) __syncthreads();
    else wave_lds_sync();
  };

  __syncthreads();                                   // (s_odd is cleared before any wave sets it)
  // Q has arrived before the first load to LDS is issued: a wait for it inside the loop would wait for those as well
  look_up(tbeg + kw);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qb[nt][ks]));
  if (tbeg + kw < tend) load_tile(tbeg + kw, 0);
  look_up(tbeg + kw + WK);
  int stage = 0;
  for (int tile = tbeg + kw; tile < tend; tile += WK) {
    const bool more = tile + WK < tend;
    if (WR > 1) {
      wait_loads<0>();
      __syncthreads();                               // the tile is there, and everybody is done with the one before it
      if (more) load_tile(tile + WK, stage ^ 1);
    } else if (more) {
      __builtin_amdgcn_s_waitcnt(0xC07F);            // lgkmcnt(0): what was read of that stage has been read
      load_tile(tile + WK, stage ^ 1);
      wait_loads<2 * NI>();
    } else {
      wait_loads<0>();
    }
    if (more) look_up(tile + 2 * WK);
    unsigned char* base = smem + (stage * WK + kw) * 2 * TILE;
    const bool full = tile < TC ? (tile + 1) * KT <= seq : !a.anc && (tile - TC + 1) * KT <= m_first + 1;
    if (full) {
      work(tile, base, std::integral_constant<bool, true>());
    } else {
      clean(tile, base + TILE);
      work(tile, base, std::integral_constant<bool, false>());
    }
    stage ^= 1;
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) l_sum[nt] += __shfl_xor(l_sum[nt], 32);
  if (odd) s_odd = 1;

  const int new0 = max(tbeg - TC, 0) * KT, new1 = min(max(tend - TC, 0) * KT, fresh);    // new keys of this range
  const uint16_t* vnew = reinterpret_cast<const uint16_t*>(a.vn) + (int64_t)c.kvbh * a.M * DH;
  const __amdgpu_buffer_rsrc_t dev_o = device_buffer(a.ws_o, a.ws_o_bytes), dev_ml = device_buffer(a.ws_ml, a.ws_ml_bytes);
  const uint32_t part = (uint32_t)((c.kvbh * a.row_blocks + c.rb) * a.nsplit + c.split) * ROWS;
  if (WK == 1) {
    __syncthreads();
    const bool fix = s_odd != 0;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = (wr * NT + nt) * 32 + l32;
      if (r0 + r >= R) continue;
      int m;
      const int64_t e = row_at<DH>(a, c.kvbh, r0 + r, &m);
      const float inv = ns == 1 ? 1.0f / l_sum[nt] : 1.0f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int d = dt * 32 + g * 8 + half * 4;
          float4 v = make_float4(oacc[nt][dt][4 * g] * inv, oacc[nt][dt][4 * g + 1] * inv, oacc[nt][dt][4 * g + 2] * inv, oacc[nt][dt][4 * g + 3] * inv);
          if (fix) add_odd(a, vnew, DH, m, d, new0, new1, v);
          if (ns == 1) store_row4(a.out, true, e + d, v);
          else store_dev(dev_o, ((part + r) * DH + d) * 4, v);
        }
      if (ns > 1 && half == 0) store_dev(dev_ml, (part + r) * 8, make_float2(m_ref[nt], l_sum[nt]));
    }
  } else {
    // the waves' parts of the rows are added in their order
    if (half == 0) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) { s_m[wave][nt * 32 + l32] = m_ref[nt]; s_l[wave][nt * 32 + l32] = l_sum[nt]; }
    }
    __syncthreads();                                 // every wave is done with its tiles too
    float* s_o = reinterpret_cast<float*>(smem);     // [W][ROWS][OPITCH]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int col = nt * 32 + l32;
      float mm = kMasked;
#pragma unroll
      for (int w = 0; w < W; ++w) mm = fmaxf(mm, s_m[w][col]);
      const float f = __builtin_amdgcn_exp2f(m_ref[nt] - mm);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<float4*>(&s_o[(wave * ROWS + col) * OPITCH + dt * 32 + g * 8 + half * 4]) =
              make_float4(oacc[nt][dt][4 * g] * f, oacc[nt][dt][4 * g + 1] * f, oacc[nt][dt][4 * g + 2] * f, oacc[nt][dt][4 * g + 3] * f);
    }
    __syncthreads();
    const bool fix = s_odd != 0;
    constexpr int C4 = DH / 4;
    for (int idx = threadIdx.x; idx < ROWS * C4; idx += W * 64) {
      const int r = idx / C4, c4 = idx % C4;
      if (r0 + r >= R) continue;
      float mm = kMasked, ll = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) mm = fmaxf(mm, s_m[w][r]);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < W; ++w) {
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
  if (ns == 1) return;
  join_ranges<DH, ROWS, W * 64, true>(a, c, r0, R, ns, [](float t) { return __builtin_amdgcn_exp2f(t); });
}

// ---------------------------------------------------------------- float32

// A block is 16 rows; its W waves take the 16-key tiles of its range in turn.  Lane (i, g) of a wave holds of key i the dimensions 16 t + 4 g .. + 3, and of
// keys 4 g + r the values of dimensions 64 h + 4 i .. + 3: what its 16-byte loads bring is what both products want.
template <int DH, int W>
__global__ __launch_bounds__(W * 64) void paged_attn_f32_kernel(PagedAttnArgs a) {
  constexpr int ROWS = 16, HT = DH / 64, P4 = DH / 4 + 1;
  extern __shared__ __align__(16) unsigned char smem[];
  float4* const s_o = reinterpret_cast<float4*>(smem);      // [W][16][P4]
  __shared__ float s_m[W][16], s_l[W][16];
  __shared__ int s_odd;
  const Cell c(a);
  const int R = c.rows * a.gq, r0 = c.rb * ROWS;
  if (r0 >= R) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  const int fresh = (int)div_or_rc((uint32_t)(min(r0 + ROWS, R) - 1), (uint32_t)a.gq, a.rc_gq) + 1;
  const int seq = c.seq, TC = (seq + 15) / 16, T = TC + (fresh + 15) / 16;
  const int ns = (T + a.range - 1) / a.range;
  if (c.split >= ns) return;
  const int tbeg = c.split * a.range, tend = min(tbeg + a.range, T);
  if (threadIdx.x == 0) s_odd = 0;
  int row;
  const float* qp = reinterpret_cast<const float*>(a.q) + row_at<DH>(a, c.kvbh, min(r0 + i, R - 1), &row);
  f32x4 q[DH / 16], acc[4 * HT];
#pragma unroll
  for (int t = 0; t < DH / 16; ++t) q[t] = *reinterpret_cast<const f32x4*>(qp + 16 * t + 4 * g);
#pragma unroll
  for (int d = 0; d < 4 * HT; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  __syncthreads();                                   // (s_odd is cleared before any wave sets it)
  const int64_t page_size = (int64_t)DH << a.page_shift;
  const int64_t new_at = (int64_t)c.kvbh * a.M * DH;
  float m = kMasked, l = 0.f;
  bool odd = false;
  for (int tile = tbeg + wave; tile < tend; tile += W) {
    const bool is_new = tile >= TC;
    const int key0 = (is_new ? tile - TC : tile) * 16, limit = is_new ? fresh : seq;
    const float *kp, *vp;                              // of key key0
    if (is_new) {
      kp = reinterpret_cast<const float*>(a.kn) + new_at + (int64_t)key0 * DH;
      vp = reinterpret_cast<const float*>(a.vn) + new_at + (int64_t)key0 * DH;
    } else {
      const int64_t at = ((int64_t)page_of(a, c.b, key0, seq) * a.Hkv + c.kvh) * page_size + (int64_t)(key0 & ((1 << a.page_shift) - 1)) * DH;
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
    f32x4 s = {0.f, 0.f, 0.f, 0.f};                    // chains of Dh / 4 products, two at a time
#pragma unroll
    for (int t0 = 0; t0 < DH / 16; t0 += DH / 32) {
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = t0; t < t0 + DH / 32; t += 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t][e], q[t][e], s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t + 1][e], q[t + 1][e], s1, 0, 0, 0);
        }
      s += s0 + s1;
    }
    uint32_t bits = limit - key0 >= 16 ? 0xFFFFu : (1u << (limit - key0)) - 1u;
    if (is_new) {
      bits &= sees32(a, row, key0 & ~31) >> (key0 & 31);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int h = 0; h < HT; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!isfinite(v[r][h][e])) { v[r][h][e] = 0.f; odd = true; }
    }
    bits >>= 4 * g;
    float mn = kMasked, sc[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      sc[r] = (bits >> r) & 1u ? s[r] * a.scale : kMasked;
      mn = fmaxf(mn, sc[r]);
    }
    mn = fmaxf(mn, __shfl_xor(mn, 16));
    mn = fmaxf(mn, __shfl_xor(mn, 32));
    mn = fmaxf(mn, m);
    if (__any(mn != m)) {
      const float f = mn == m ? 1.f : exp_neg(m - mn);
      l *= f;
#pragma unroll
      for (int d = 0; d < 4 * HT; ++d) acc[d] *= f;
      m = mn;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      sc[r] = (bits >> r) & 1u ? exp_neg(sc[r] - m) : 0.f;
      l += sc[r];
      const bool there = key0 + 4 * g + r < limit;      // (values that are not there: the last's, weight 0)
#pragma unroll
      for (int h = 0; h < HT; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[4 * h + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(there ? v[r][h][e] : 0.f, sc[r], acc[4 * h + e], 0, 0, 0);
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (lane < 16) { s_m[wave][lane] = m; s_l[wave][lane] = l; }
  if (odd) s_odd = 1;
#pragma unroll
  for (int h = 0; h < HT; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      s_o[(wave * 16 + i) * P4 + 16 * h + 4 * g + r] = make_float4(acc[4 * h][r], acc[4 * h + 1][r], acc[4 * h + 2][r], acc[4 * h + 3][r]);
  __syncthreads();

  const __amdgpu_buffer_rsrc_t dev_o = device_buffer(a.ws_o, a.ws_o_bytes), dev_ml = device_buffer(a.ws_ml, a.ws_ml_bytes);
  const uint32_t part = (uint32_t)((c.kvbh * a.row_blocks + c.rb) * a.nsplit + c.split) * ROWS;
  for (int idx = threadIdx.x; idx < 16 * DH / 4; idx += W * 64) {
    const int r = idx / (DH / 4), c4 = idx % (DH / 4);
    if (r0 + r >= R) continue;
    float mm = kMasked, ll = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) mm = fmaxf(mm, s_m[w][r]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = exp_neg(s_m[w][r] - mm);
      const float4 x = s_o[(w * 16 + r) * P4 + c4];
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
  if (ns == 1) return;
  join_ranges<DH, ROWS, W * 64, false>(a, c, r0, R, ns, [](float t) { return exp_neg(t); });
}

// ---------------------------------------------------------------- host

struct PagedPlan {
  int nt, wr, wk, kt, rows;          // shape of a block
  int row_blocks, nsplit, range;
  size_t lds;
  size_t o_bytes, ml_bytes;          // partials
};

PagedPlan plan_paged(const lpp_paged* cache, int64_t B, int gq, int64_t M, int64_t S) {
  PagedPlan p;
  const int64_t R = M * gq;
  const int Dh = cache->Dh;
  int resident;                      // blocks that a compute unit holds
  if (cache->dtype == LPP_F32) {
    p.nt = 1; p.wr = 1; p.wk = Dh == 64 ? 16 : 8; p.kt = 16; p.rows = 16;
    p.lds = (size_t)p.wk * 16 * (Dh + 4) * sizeof(float);
    resident = 2;
  } else {
    if (R <= 32) { p.nt = 1; p.wr = 1; p.wk = 4; p.kt = 32; }
    else if (R <= 64) { p.nt = 2; p.wr = 1; p.wk = 4; p.kt = 32; }
    else { p.nt = 1; p.wr = 4; p.wk = 1; p.kt = 64; }
    p.rows = p.nt * p.wr * 32;
    const size_t tiles = (size_t)2 * p.wk * 2 * p.kt * Dh * 2;
    const size_t merge = p.wk > 1 ? (size_t)p.wk * p.rows * (Dh + 4) * sizeof(float) : 0;
    p.lds = std::max(tiles, merge);
    resident = std::max<int>(1, std::min<int>(2, (int)(150 * 1024 / p.lds)));
  }
  p.row_blocks = (int)((R + p.rows - 1) / p.rows);
  const int64_t units = B * cache->Hkv * p.row_blocks;
  const int64_t tiles = (S + p.kt - 1) / p.kt + (M + p.kt - 1) / p.kt, rounds = (tiles + p.wk - 1) / p.wk;
  // key ranges only while compute units would idle, of two rounds of the block's waves at least
  int64_t ranges = std::min<int64_t>((int64_t)cache->n_cu * resident / std::max<int64_t>(units, 1), rounds / 2);
  if (units > LPP_COUNTER_SLOTS) ranges = 1;
  ranges = std::max<int64_t>(1, std::min<int64_t>(ranges, ((int64_t)1 << 31) / (units * p.rows * (Dh + 2) * 4) - 1));
  const int64_t per = (rounds + ranges - 1) / ranges;
  p.range = (int)(per * p.wk);
  p.nsplit = (int)((tiles + p.range - 1) / p.range);
  const size_t parts = p.nsplit > 1 ? (size_t)units * p.nsplit * p.rows : 0;
  p.o_bytes = lpp_align_up(parts * Dh * sizeof(float), 256);
  p.ml_bytes = lpp_align_up(parts * 2 * sizeof(float), 256);
  return p;
}

template <typename K>
int32_t launch(K kern, LppLdsLimit& limit, const PagedAttnArgs& a, int threads, const PagedPlan& p, hipStream_t s) {
  const int32_t st = lpp_ensure_lds(reinterpret_cast<const void*>(kern), limit, p.lds, 48 * 1024);
  if (st != LPP_OK) return st;
  hipLaunchKernelGGL(kern, dim3(a.units * (uint32_t)a.row_blocks), dim3(threads), p.lds, s, a);
  LPP_HIP_TRY(hipGetLastError());
  return LPP_OK;
}
template <int DH, int NT, int WR, int WK, int KT>
int32_t launch_bf16(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  static LppLdsLimit limit;
  return launch(paged_attn_bf16_kernel<DH, NT, WR, WK, KT>, limit, a, WR * WK * 64, p, s);
}
template <int DH, int W>
int32_t launch_f32(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  static LppLdsLimit limit;
  return launch(paged_attn_f32_kernel<DH, W>, limit, a, W * 64, p, s);
}
template <int DH>
int32_t launch_paged(const lpp_paged* cache, const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  if (cache->dtype == LPP_F32) return launch_f32<DH, DH == 64 ? 16 : 8>(a, p, s);
  if (p.wr == 4) return launch_bf16<DH, 1, 4, 1, 64>(a, p, s);
  return p.nt == 1 ? launch_bf16<DH, 1, 1, 4, 32>(a, p, s) : launch_bf16<DH, 2, 1, 4, 32>(a, p, s);
}

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

int32_t paged_attention(const lpp_paged* cache, const lpp_tree* tree, const void* q, const void* k_pages, const void* v_pages,
                        const int32_t* page_table, int32_t table_stride, const void* k_new, const void* v_new,
                        const int32_t* seq_len, const int32_t* row_len, int32_t B, int32_t H, int32_t M, int32_t S, float scale,
                        void* out, void* ws, size_t ws_bytes, void* stream) {
  if (!cache || !q || !k_new || !v_new || !out) return LPP_EINVAL;
  if (B < 1 || H < 1 || M < 1 || S < 0) return LPP_EINVAL;
  if (S > 0 && (!k_pages || !v_pages || !page_table || table_stride < 1)) return LPP_EINVAL;
  if (H % cache->Hkv != 0) return LPP_EINVAL;
  if (S > 0 && ((int64_t)table_stride << cache->page_shift) < S) return LPP_EINVAL;
  if (!(scale >= 0.f) || scale == INFINITY) return LPP_EINVAL;           // NaN, negative, infinite
  if (misaligned(q) || misaligned(k_new) || misaligned(v_new) || misaligned(out) || misaligned(k_pages) || misaligned(v_pages)) return LPP_EINVAL;
  const int esz = cache->dtype == LPP_F32 ? 4 : 2, gq = H / cache->Hkv;
  // 32-bit offsets inside one head's new rows, row and key numbers, units and blocks
  if ((int64_t)M * cache->Dh * esz >= (1ll << 31) || (int64_t)M * gq >= (1ll << 30) || (int64_t)S + M >= (1ll << 30)) return LPP_EUNSUPPORTED;
  if ((int64_t)B * cache->Hkv >= (1ll << 24)) return LPP_EUNSUPPORTED;
  const PagedPlan p = plan_paged(cache, B, gq, M, S);
  const int64_t units = (int64_t)B * cache->Hkv * p.nsplit;
  if (units * p.row_blocks >= (1ll << 31)) return LPP_EUNSUPPORTED;
  if (p.o_bytes + p.ml_bytes > 0 && (!ws || misaligned(ws) || ws_bytes < p.o_bytes + p.ml_bytes)) return LPP_ENOWORKSPACE;
  if (!cache->d_counters || (tree && !tree->d_anc)) return LPP_EHIP;     // host-only handle: no device
  if (!lpp_is_current(cache->device) || (tree && tree->device != cache->device)) return LPP_EINVAL;
  if (scale == 0.f) scale = 1.0f / sqrtf((float)cache->Dh);
  PagedAttnArgs a;
  a.q = q; a.kp = k_pages; a.vp = v_pages; a.kn = k_new; a.vn = v_new; a.out = out;
  a.table = page_table; a.seq_len = seq_len; a.row_len = row_len;
  a.anc = tree ? tree->d_anc : nullptr; a.words = tree ? tree->words : 0;
  a.Hkv = cache->Hkv; a.gq = gq; a.M = M; a.S = S;
  a.rc_gq = reciprocal((uint32_t)gq, (uint64_t)M * gq);
  a.table_stride = table_stride; a.page_shift = cache->page_shift; a.n_pages = cache->n_pages;
  a.row_blocks = p.row_blocks; a.nsplit = p.nsplit; a.range = p.range;
  a.units = (uint32_t)units; a.whole = (uint32_t)(units & ~7ll);
  a.scale = cache->dtype == LPP_F32 ? scale : scale * 1.44269504088896340736f;
  a.ws_o = reinterpret_cast<float*>(ws);
  a.ws_ml = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(ws) + p.o_bytes);
  a.ws_o_bytes = (uint32_t)p.o_bytes; a.ws_ml_bytes = (uint32_t)p.ml_bytes;
  a.counters = cache->d_counters;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return cache->Dh == 64 ? launch_paged<64>(cache, a, p, s) : launch_paged<128>(cache, a, p, s);
}

}  // namespace

extern "C" size_t lpp_paged_attention_workspace(const lpp_paged* cache, int32_t B, int32_t H, int32_t M, int32_t S) {
  if (!cache || B < 1 || H < 1 || M < 1 || S < 0 || H % cache->Hkv != 0) return 0;
  const PagedPlan p = plan_paged(cache, B, H / cache->Hkv, M, S);
  return std::max<size_t>(p.o_bytes + p.ml_bytes, 256);
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
