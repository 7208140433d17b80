// The target's logits on their way to verification: guidance, penalties for tokens seen, biases and a grammar's mask.
//
// A row of the tree is scored in the context of its own path: what counts for row i of item b is the item's history
// (counts) and the drafted tokens on the way from the root to row i, row i's own included, the root's not (it is history).
//   l = u + cfg_scale (c - u)                    where unconditional logits are given
//   n = counts[b][x] + occurrences of x on the path;  n > 0:  l = (l > 0 ? l / repetition : l repetition) - frequency n - presence
//   l += bias[x];  a token that the mask does not allow: -inf, whatever l is
//
// Bound by memory: a logit is read once and written once.  A block is a piece of one row; its lanes ask for their logits
// first, and while these are on their way the path's tokens are counted into a byte for every token of the piece in LDS (a path
// has at most 255 tokens), so that the pass over the piece needs no second look and may write where it read.
#include <math.h>

#include "lpp_device.h"
#include "lpp_internal.h"

namespace {

struct LogitsArgs {
  const void* cond;
  const void* uncond;
  float* out;
  const uint64_t* anc;
  const int32_t* tokens;
  const int32_t* counts;
  const float* repetition;
  const float* frequency;
  const float* presence;
  const float* bias;
  const uint32_t* mask;
  int64_t ldv, bias_stride, mask_item, mask_row;
  int32_t V, M, words, parts;
  float cfg_scale;
};

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));       // rows may start on any element
typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ void load4(float (&x)[4], const float* p) {
  const f32x4_any v = *reinterpret_cast<const f32x4_any*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = v[e];
}
__device__ __forceinline__ void load4(float (&x)[4], const uint16_t* p) {
  const u16x4_any v = *reinterpret_cast<const u16x4_any*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = __uint_as_float((uint32_t)v[e] << 16);
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

// CELLS: groups of four tokens a lane.  Two, or one where blocks of two would be fewer than four a compute unit: 61 guided rows
// of 8192 4.2 -> 3.5 us; 2064 rows of 16384 62.9 us with two, 68.3 with one, 67.4 with four (4.4 TB/s of the 4.95 that a copy
// reaches).
template <typename T, bool GUIDED, int CELLS>
__global__ __launch_bounds__(256) void adjust_logits_kernel(LogitsArgs a) {
  constexpr int kCells = CELLS, kPiece = 256 * 4 * CELLS;
  __shared__ __align__(16) uint32_t s_had[kPiece / 4];       // occurrences on the path, a byte a token
  const int tid = threadIdx.x;
  const int row = (int)(blockIdx.x / (unsigned)a.parts), part = (int)(blockIdx.x - (unsigned)row * a.parts);   // row: b M + i
  const int b = row / a.M, i = row - b * a.M;
  const int x0 = part * kPiece, V = a.V;
  const T* cond = reinterpret_cast<const T*>(a.cond) + row * a.ldv;
  const T* uncond = GUIDED ? reinterpret_cast<const T*>(a.uncond) + row * a.ldv : nullptr;
  float* out = a.out + row * a.ldv;

  float c[kCells][4], u[kCells][4];
#pragma unroll
  for (int k = 0; k < kCells; ++k) {
    const int x = x0 + (k * 256 + tid) * 4;
    if (x + 4 <= V) {
      load4(c[k], cond + x);
      if (GUIDED) load4(u[k], uncond + x);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[k][e] = x + e < V ? load1(cond + x + e) : 0.f;
        if (GUIDED) u[k][e] = x + e < V ? load1(uncond + x + e) : 0.f;
      }
    }
  }
  const float rep = a.repetition ? a.repetition[b] : 1.f, freq = a.frequency ? a.frequency[b] : 0.f;
  const float pres = a.presence ? a.presence[b] : 0.f;
  const bool path = a.tokens && i > 0;
  if (path) {
#pragma unroll
    for (int k = 0; k < kCells; ++k) s_had[k * 256 + tid] = 0;
    __syncthreads();
    if (tid > 0 && tid < a.M && ((a.anc[(int64_t)i * a.words + (tid >> 6)] >> (tid & 63)) & 1)) {
      const int x = min(max(a.tokens[(int64_t)b * a.M + tid], 0), V - 1) - x0;
      if (x >= 0 && x < kPiece) atomicAdd(&s_had[x >> 2], 1u << (8 * (x & 3)));
    }
    __syncthreads();
  }
#pragma unroll
  for (int k = 0; k < kCells; ++k) {
    const int x = x0 + (k * 256 + tid) * 4;
    if (x >= V) continue;
    const bool whole = x + 4 <= V;
    int n[4] = {0, 0, 0, 0};
    if (a.counts) {
      const int32_t* p = a.counts + (int64_t)b * V + x;
      if (whole) {
        const i32x4_any v = *reinterpret_cast<const i32x4_any*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) n[e] = v[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) n[e] = x + e < V ? p[e] : 0;
      }
    }
    if (path) {
      const uint32_t had = s_had[k * 256 + tid];
#pragma unroll
      for (int e = 0; e < 4; ++e) n[e] += (int)((had >> (8 * e)) & 255u);
    }
    float bias[4] = {0.f, 0.f, 0.f, 0.f};
    if (a.bias) {
      const float* p = a.bias + b * a.bias_stride + x;
      if (whole) load4(bias, p);
      else
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[e] = x + e < V ? p[e] : 0.f;
    }
    const uint32_t allowed = a.mask ? a.mask[b * a.mask_item + i * a.mask_row + (x >> 5)] >> (x & 31) : 0xFu;
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float l = GUIDED ? u[k][e] + a.cfg_scale * (c[k][e] - u[k][e]) : c[k][e];
      if (n[e] > 0) l = (l > 0.f ? l / rep : l * rep) - freq * (float)n[e] - pres;
      l += bias[e];
      y[e] = (allowed >> e) & 1u ? l : -INFINITY;
    }
    if (whole) {
      *reinterpret_cast<f32x4_any*>(out + x) = f32x4_any{y[0], y[1], y[2], y[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (x + e < V) out[x + e] = y[e];
    }
  }
}

// How often every token occurs among an item's: a block counts one piece of the vocabulary in LDS, 4 us for 4096 tokens of an item,
// 8.7 for 32768: few blocks, each as long as its lanes take for the item's tokens.
constexpr int kCounted = 32768;
__global__ __launch_bounds__(1024) void token_counts_kernel(const int32_t* tokens, const int32_t* len, int32_t T, int32_t V,
                                                            int32_t pieces, int32_t* counts) {
  extern __shared__ int32_t s_n[];
  const int b = (int)(blockIdx.x / (unsigned)pieces), x0 = (int)(blockIdx.x - (unsigned)b * pieces) * kCounted;
  const int here = min(V - x0, kCounted), n = len ? min(max(len[b], 0), T) : T;
  for (int x = threadIdx.x; x < here; x += 1024) s_n[x] = 0;
  __syncthreads();
  const int32_t* t = tokens + (int64_t)b * T;
  for (int j = threadIdx.x; j < n; j += 1024) {
    const int x = t[j];
    if (x >= x0 && x - x0 < here) atomicAdd(&s_n[x - x0], 1);
  }
  __syncthreads();
  int32_t* out = counts + (int64_t)b * V + x0;
  for (int x = threadIdx.x; x < here; x += 1024) out[x] = s_n[x];
}

// One wave an item: the accepted path's tokens, then the emitted one.  (Whole numbers: the order of the adds is no matter.)
__global__ __launch_bounds__(64) void commit_counts_kernel(const int32_t* tokens, const int32_t* path, const int32_t* accept_len,
                                                           const int32_t* final_token, int32_t M, int32_t depth, int32_t V,
                                                           int32_t* counts) {
  const int b = blockIdx.x, n = min(accept_len[b], depth);
  for (int j = threadIdx.x; j <= n; j += 64) {               // (a walk that gave up: accept_len and final_token -1, nothing to add)
    int x = final_token[b];
    if (j < n) {
      const int node = path[(int64_t)b * depth + j];
      x = node >= 0 && node < M ? min(max(tokens[(int64_t)b * M + node], 0), V - 1) : -1;
    }
    if (x >= 0 && x < V) atomicAdd(&counts[(int64_t)b * V + x], 1);
  }
}

template <typename T, bool GUIDED>
int32_t launch_adjust(LogitsArgs& a, int64_t rows, int32_t n_cu, hipStream_t s) {
  const int64_t wide = ((int64_t)a.V + 2047) / 2048, narrow = ((int64_t)a.V + 1023) / 1024;
  const bool two = rows * wide >= (int64_t)n_cu * 4;
  a.parts = (int32_t)(two ? wide : narrow);
  const int64_t blocks = rows * a.parts;
  if (two) hipLaunchKernelGGL((adjust_logits_kernel<T, GUIDED, 2>), dim3((unsigned)blocks), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((adjust_logits_kernel<T, GUIDED, 1>), dim3((unsigned)blocks), dim3(256), 0, s, a);
  LPP_HIP_TRY(hipGetLastError());
  return LPP_OK;
}

}  // namespace

extern "C" int32_t lpp_adjust_logits(const lpp_tree* tree, int32_t dtype, const void* logits, int64_t ldv, int32_t vocab_offset,
                                     int32_t V, int32_t B, const lpp_logits_options* opts, float* out, void* stream) {
  if (!tree || !logits || !opts || !out) return LPP_EINVAL;
  if (B < 1 || V < 1 || vocab_offset < 0 || (int64_t)vocab_offset + V > ldv) return LPP_EINVAL;
  if (opts->cfg_scale != opts->cfg_scale) return LPP_EINVAL;
  if (opts->bias_stride < 0 || opts->mask_item_stride < 0 || opts->mask_row_stride < 0) return LPP_EINVAL;
  if (dtype != LPP_F32 && dtype != LPP_BF16) return LPP_EUNSUPPORTED;
  if (V >= 1 << 30) return LPP_EUNSUPPORTED;                 // (a lane's tokens are numbered past V)
  // what is written must not be read by another lane: in place with float32 logits only
  if (dtype != LPP_F32 && (out == logits || out == opts->uncond_logits)) return LPP_EINVAL;
  LogitsArgs a;
  const int esz = dtype == LPP_F32 ? 4 : 2;
  a.cond = (const unsigned char*)logits + (int64_t)vocab_offset * esz;
  a.uncond = opts->uncond_logits ? (const unsigned char*)opts->uncond_logits + (int64_t)vocab_offset * esz : nullptr;
  a.out = out + vocab_offset;
  a.anc = tree->d_anc; a.tokens = opts->tokens; a.counts = opts->counts;
  a.repetition = opts->repetition; a.frequency = opts->frequency; a.presence = opts->presence;
  a.bias = opts->bias; a.bias_stride = opts->bias_stride;
  a.mask = opts->mask; a.mask_item = opts->mask_item_stride; a.mask_row = opts->mask_row_stride;
  a.ldv = ldv; a.V = V; a.M = tree->M; a.words = tree->words; a.cfg_scale = opts->cfg_scale;
  const int64_t rows = (int64_t)B * tree->M;
  if (!lpp_launch_fits(rows * (((int64_t)V + 2047) / 2048), 256)) return LPP_EUNSUPPORTED;     // (narrower blocks: few)
  if (!tree->d_anc) return LPP_EHIP;                         // host-only handle: no device
  if (!lpp_is_current(tree->device)) return LPP_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == LPP_F32) return a.uncond ? launch_adjust<float, true>(a, rows, tree->n_cu, s) : launch_adjust<float, false>(a, rows, tree->n_cu, s);
  return a.uncond ? launch_adjust<uint16_t, true>(a, rows, tree->n_cu, s) : launch_adjust<uint16_t, false>(a, rows, tree->n_cu, s);
}

extern "C" int32_t lpp_token_counts(const int32_t* tokens, const int32_t* len, int32_t B, int32_t T, int32_t V, int32_t* counts,
                                    void* stream) {
  if (!counts || B < 1 || T < 0 || V < 1 || (T > 0 && !tokens)) return LPP_EINVAL;
  if (T >= 1 << 30 || V >= 1 << 30) return LPP_EUNSUPPORTED; // (lanes step past the last token)
  const int64_t pieces = ((int64_t)V + kCounted - 1) / kCounted, blocks = B * pieces;
  if (!lpp_launch_fits(blocks, 1024)) return LPP_EUNSUPPORTED;
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || ndev < 1) {
    (void)hipGetLastError();
    return LPP_EHIP;
  }
  static LppLdsLimit limit;
  const size_t lds = (size_t)(V < kCounted ? V : kCounted) * sizeof(int32_t);
  const int32_t st = lpp_ensure_lds(reinterpret_cast<const void*>(token_counts_kernel), limit, lds, 64 * 1024);
  if (st != LPP_OK) return st;
  hipLaunchKernelGGL(token_counts_kernel, dim3((unsigned)blocks), dim3(1024), lds, reinterpret_cast<hipStream_t>(stream), tokens, len,
                     T, V, (int32_t)pieces, counts);
  LPP_HIP_TRY(hipGetLastError());
  return LPP_OK;
}

extern "C" int32_t lpp_commit_counts(const lpp_tree* tree, const int32_t* tokens, const int32_t* path, const int32_t* accept_len,
                                     const int32_t* final_token, int32_t B, int32_t V, int32_t* counts, void* stream) {
  if (!tree || !tokens || !path || !accept_len || !final_token || !counts) return LPP_EINVAL;
  if (B < 1 || V < 1) return LPP_EINVAL;
  if (!lpp_launch_fits(B, 64)) return LPP_EUNSUPPORTED;
  if (!tree->d_anc) return LPP_EHIP;
  if (!lpp_is_current(tree->device)) return LPP_EINVAL;
  hipLaunchKernelGGL(commit_counts_kernel, dim3((unsigned)B), dim3(64), 0, reinterpret_cast<hipStream_t>(stream), tokens, path,
                     accept_len, final_token, tree->M, tree->depth, V, counts);
  LPP_HIP_TRY(hipGetLastError());
  return LPP_OK;
}
