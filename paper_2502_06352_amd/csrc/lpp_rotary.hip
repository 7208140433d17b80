// Rotary positions of a step's rows: what the projections give becomes the queries, keys and values that attention reads.
//
//   row (b, i) stands at position p = first_pos[b] + (tree: depth of row i; chunk: i)
//   pair j of a head's first `dim` numbers turns by p theta_j:  y1 = m (x1 cos - x2 sin), y2 = m (x2 cos + x1 sin)
//   the rest of the head, and the values, are copied
//
// theta_j comes from the handle in turns per position, float64: p theta_j is formed in float64 and only its fraction of a
// turn is rounded to float32, so that far positions (2^20 and more) turn as exactly as near ones.
//
// Bound by memory: every number is read and written once, and the layout changes from rows of heads to heads of rows on the
// way. A lane has 8 pairs of one row (two 16-byte pieces of bf16) and goes through a group of heads with the same cosines and
// sines.  (4 chunks of up to 2048 rows, 32 heads and 8 of 128 in bf16: 29.4 us, 4.3 TB/s of the 4.95 that a copy reaches;
// groups of all heads, fewer blocks than the chip holds, 36.7 us; one of a verification step's 61 rows, 72 heads in all: 4.1 us
// and 5.9.)
#include <math.h>

#include <algorithm>
#include <new>

#include "lpp_device.h"
#include "lpp_internal.h"
#include "lpp_overlap.h"

struct lpp_rotary {
  int32_t dim = 0, layout = 0;
  float magnitude = 1.f;
  double turns[LPP_ROTARY_MAX_DIM / 2] = {};        // turns per position of every pair
};

extern "C" int32_t lpp_rotary_create(const lpp_rotary_config* c, lpp_rotary** out) {
  if (!c || !out) return LPP_EINVAL;
  *out = nullptr;
  if (c->dim < 1) return LPP_EINVAL;
  if (c->layout != LPP_ROTARY_HALF && c->layout != LPP_ROTARY_INTERLEAVED) return LPP_EINVAL;
  if (c->scaling < LPP_ROTARY_NONE || c->scaling > LPP_ROTARY_YARN) return LPP_EINVAL;
  const double base = c->base == 0. ? 10000. : c->base, fast = c->fast == 0. ? 32. : c->fast, slow = c->slow == 0. ? 1. : c->slow;
  if (!(base > 1.) || !std::isfinite(base) || !(c->magnitude >= 0.)) return LPP_EINVAL;
  if (!std::isfinite((float)c->magnitude) || (c->magnitude > 0. && (float)c->magnitude == 0.f)) return LPP_EINVAL;      // (m is a float32)
  if (c->scaling != LPP_ROTARY_NONE && (!(c->factor >= 1.) || !std::isfinite(c->factor))) return LPP_EINVAL;
  if (c->scaling == LPP_ROTARY_YARN && (c->original_len < 1 || !(slow > 0.) || !(fast > slow) || !std::isfinite(fast))) return LPP_EINVAL;
  if (c->dim % 16 != 0 || c->dim > LPP_ROTARY_MAX_DIM) return LPP_EUNSUPPORTED;
  lpp_rotary* r = new (std::nothrow) lpp_rotary();
  if (!r) return LPP_EHIP;
  constexpr double kTwoPi = 6.283185307179586476925286766559;
  const double s = c->scaling == LPP_ROTARY_NONE ? 1. : c->factor, d = c->dim;
  r->dim = c->dim; r->layout = c->layout;
  const double b = c->scaling == LPP_ROTARY_NTK ? base * pow(s, d / (d - 2.)) : base;
  for (int32_t j = 0; j < c->dim / 2; ++j) {
    double theta = pow(b, -2. * j / d);
    if (c->scaling == LPP_ROTARY_LINEAR) theta /= s;
    if (c->scaling == LPP_ROTARY_YARN) {             // pairs that turn often within the original length keep their angle
      const double g = std::min(1., std::max(0., (c->original_len * theta / kTwoPi - slow) / (fast - slow)));
      theta = (1. - g) * theta / s + g * theta;
    }
    r->turns[j] = theta / kTwoPi;
  }
  r->magnitude = (float)(c->magnitude > 0. ? c->magnitude : c->scaling == LPP_ROTARY_YARN ? 0.1 * log(s) + 1. : 1.);
  *out = r;
  return LPP_OK;
}

extern "C" int32_t lpp_rotary_destroy(lpp_rotary* r) {
  delete r;
  return LPP_OK;
}

namespace {

struct RotaryArgs {
  const unsigned char* in[3];        // q, k, v
  unsigned char* out[3];
  int64_t item[3], row[3], head[3];  // strides of `in`, in elements
  const int32_t* first_pos;
  const int32_t* row_len;
  const uint64_t* anc;               // tree, or null
  int32_t words, M, Dh, dim;
  int32_t rows, units, row_blocks;   // rows of a block, lanes of a row, blocks of an item
  int32_t heads_q, heads_qk, heads;  // H, H + Hkv, H + 2 Hkv (what is missing counts none)
  int32_t group, groups;             // heads of a block; blocks of some rows
  int32_t n_heads[3];
  float magnitude;
  double turns[LPP_ROTARY_MAX_DIM / 2];
};

template <typename T> struct Eight;
template <> struct Eight<uint16_t> {
  uint4 x;
  __device__ __forceinline__ void load(const uint16_t* p) { x = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<uint4*>(p) = x; }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    x = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  }
};
template <> struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
  __device__ __forceinline__ void store(float* p) const { reinterpret_cast<float4*>(p)[0] = a; reinterpret_cast<float4*>(p)[1] = b; }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ __forceinline__ void set(const float (&f)[8]) { a = make_float4(f[0], f[1], f[2], f[3]); b = make_float4(f[4], f[5], f[6], f[7]); }
};

template <typename T, bool HALF>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  const int id = (int)(blockIdx.x / (unsigned)a.groups), group = (int)(blockIdx.x - (unsigned)id * a.groups);
  const int b = id / a.row_blocks, rb = id - b * a.row_blocks;
  const int r = (int)threadIdx.x / a.units, u = (int)threadIdx.x - r * a.units;
  const int i = rb * a.rows + r;
  const int n = a.row_len ? min(max(a.row_len[b], 0), a.M) : a.M;
  if (r >= a.rows || i >= n) return;
  const bool turned = u * 16 < a.dim;
  const int e0 = HALF && turned ? 8 * u : 16 * u, e1 = HALF && turned ? a.dim / 2 + 8 * u : 16 * u + 8;
  const int h0 = group * a.group, h1 = min(h0 + a.group, a.heads);
  float cs[8], sn[8];
  if (turned && h0 < a.heads_qk) {
    int64_t pos = a.first_pos ? a.first_pos[b] : 0;
    if (a.anc) {
      int depth = -1;
      for (int w = 0; w < a.words; ++w) depth += __popcll(a.anc[(int64_t)i * a.words + w]);
      pos += depth;
    } else {
      pos += i;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const double t = (double)pos * a.turns[8 * u + j];
      float s, c;
      sincospif(2.f * (float)(t - rint(t)), &s, &c);
      cs[j] = a.magnitude * c;
      sn[j] = a.magnitude * s;
    }
  }
  constexpr int UN = 2;                              // heads in flight
  for (int h = h0; h < h1; h += UN) {
    Eight<T> x[UN][2];
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      const int hh = min(h + k, h1 - 1);             // (past the group: its last again, not written)
      const int which = hh < a.heads_q ? 0 : hh < a.heads_qk ? 1 : 2;
      const int hl = hh - (which == 0 ? 0 : which == 1 ? a.heads_q : a.heads_qk);
      const T* src = reinterpret_cast<const T*>(a.in[which]) + (b * a.item[which] + i * a.row[which] + hl * a.head[which]);
      x[k][0].load(src + e0);
      x[k][1].load(src + e1);
    }
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      const int hh = h + k;
      if (hh >= h1) break;
      const int which = hh < a.heads_q ? 0 : hh < a.heads_qk ? 1 : 2;
      const int hl = hh - (which == 0 ? 0 : which == 1 ? a.heads_q : a.heads_qk);
      T* dst = reinterpret_cast<T*>(a.out[which]) + (((int64_t)b * a.n_heads[which] + hl) * a.M + i) * a.Dh;
      if (turned && which < 2) {
        float p[8], q[8];
        x[k][0].get(p);
        x[k][1].get(q);
        if (HALF) {                                  // pair j = (p[j], q[j])
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float y1 = __builtin_fmaf(p[j], cs[j], -(q[j] * sn[j])), y2 = __builtin_fmaf(q[j], cs[j], p[j] * sn[j]);
            p[j] = y1; q[j] = y2;
          }
        } else {                                     // pair j = two neighbours of the sixteen
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float y1 = __builtin_fmaf(p[2 * j], cs[j], -(p[2 * j + 1] * sn[j])), y2 = __builtin_fmaf(p[2 * j + 1], cs[j], p[2 * j] * sn[j]);
            p[2 * j] = y1; p[2 * j + 1] = y2;
            const float z1 = __builtin_fmaf(q[2 * j], cs[4 + j], -(q[2 * j + 1] * sn[4 + j])), z2 = __builtin_fmaf(q[2 * j + 1], cs[4 + j], q[2 * j] * sn[4 + j]);
            q[2 * j] = z1; q[2 * j + 1] = z2;
          }
        }
        x[k][0].set(p);
        x[k][1].set(q);
      }
      x[k][0].store(dst + e0);
      x[k][1].store(dst + e1);
    }
  }
}

}  // namespace

extern "C" int32_t lpp_rotary_qkv(const lpp_rotary* rotary, const lpp_tree* tree, int32_t dtype, const lpp_rows* q,
                                  const lpp_rows* k, const lpp_rows* v, const int32_t* first_pos, const int32_t* row_len,
                                  int32_t B, int32_t H, int32_t Hkv, int32_t M, int32_t Dh, void* q_out, void* k_out,
                                  void* v_out, void* stream) {
  if (!rotary || (!q && !k && !v)) return LPP_EINVAL;
  if (B < 1 || H < 1 || Hkv < 1 || M < 1 || Dh < 1) return LPP_EINVAL;
  if (tree && tree->M != M) return LPP_EINVAL;
  if (rotary->dim > Dh) return LPP_EINVAL;
  if (dtype != LPP_F32 && dtype != LPP_BF16) return LPP_EUNSUPPORTED;
  if (Dh % 16 != 0 || Dh > LPP_ROTARY_MAX_DIM) return LPP_EUNSUPPORTED;
  if (M >= 1 << 30) return LPP_EUNSUPPORTED;                 // (a block's rows are numbered past M)
  const int esz = dtype == LPP_F32 ? 4 : 2;
  const lpp_rows* in[3] = {q, k, v};
  void* out[3] = {q_out, k_out, v_out};
  RotaryArgs a;
  a.heads = 0;
  for (int t = 0; t < 3; ++t) {
    const int32_t heads = !in[t] ? 0 : t == 0 ? H : Hkv;
    if (!in[t] != !out[t]) return LPP_EINVAL;
    a.in[t] = nullptr; a.out[t] = nullptr; a.item[t] = a.row[t] = a.head[t] = 0;
    if (in[t]) {
      const lpp_rows& y = *in[t];
      if (!y.data || y.item < 0 || y.row < 0 || y.head < 0) return LPP_EINVAL;
      if (((reinterpret_cast<uintptr_t>(y.data) | reinterpret_cast<uintptr_t>(out[t])) & 15) != 0) return LPP_EINVAL;
      if ((y.item * esz) % 16 != 0 || (y.row * esz) % 16 != 0 || (y.head * esz) % 16 != 0) return LPP_EUNSUPPORTED;
      // in place only where every number stays where it is
      if (y.data == out[t] && ((B > 1 && y.item != (int64_t)heads * M * Dh) || (heads > 1 && y.head != (int64_t)M * Dh) || (M > 1 && y.row != Dh)))
        return LPP_EINVAL;
      a.in[t] = (const unsigned char*)y.data; a.out[t] = (unsigned char*)out[t];
      a.item[t] = y.item; a.row[t] = y.row; a.head[t] = y.head;
    }
    a.n_heads[t] = heads;
    a.heads += heads;
    if (t == 0) a.heads_q = a.heads;
    if (t == 1) a.heads_qk = a.heads;
  }
  if (tree && !tree->d_anc) return LPP_EHIP;                 // host-only handle: no device
  if (tree && !lpp_is_current(tree->device)) return LPP_EINVAL;
  a.first_pos = first_pos; a.row_len = row_len;
  a.anc = tree ? tree->d_anc : nullptr; a.words = tree ? tree->words : 0;
  a.M = M; a.Dh = Dh; a.dim = rotary->dim; a.magnitude = rotary->magnitude;
  a.units = Dh / 16; a.rows = std::min(256 / a.units, M);
  a.row_blocks = (M + a.rows - 1) / a.rows;
  // (two heads a block, blocks of some rows one behind the other, so that what lies together is read together)
  a.group = 2;
  a.groups = (a.heads + a.group - 1) / a.group;
  std::copy(rotary->turns, rotary->turns + LPP_ROTARY_MAX_DIM / 2, a.turns);
  const int64_t blocks = (int64_t)B * a.row_blocks * a.groups;
  if (!lpp_launch_fits(blocks, 256)) return LPP_EUNSUPPORTED;
  // blocks read what others have written: outputs lie in no input (but in place, see above) and in no other output
  for (int t = 0; t < 3; ++t)
    for (int u = 0; u < 3 && out[t]; ++u) {
      const int64_t width = (int64_t)Dh * esz, n = (int64_t)B * a.n_heads[t] * M * width;
      if (in[u] && !(u == t && in[u]->data == out[t]) &&
          rows_meet(in[u]->data, in[u]->item * esz, in[u]->row * esz, in[u]->head * esz, B, M, a.n_heads[u], width, out[t], n)) return LPP_EINVAL;
      if (u > t && ranges_meet(out[t], (uint64_t)n, out[u], (uint64_t)B * a.n_heads[u] * M * width)) return LPP_EINVAL;
    }
  const dim3 grid((unsigned)blocks);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool half = rotary->layout == LPP_ROTARY_HALF;
  if (dtype == LPP_BF16) {
    if (half) hipLaunchKernelGGL((rotary_kernel<uint16_t, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((rotary_kernel<uint16_t, false>), grid, dim3(256), 0, s, a);
  } else {
    if (half) hipLaunchKernelGGL((rotary_kernel<float, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((rotary_kernel<float, false>), grid, dim3(256), 0, s, a);
  }
  LPP_HIP_TRY(hipGetLastError());
  return LPP_OK;
}
