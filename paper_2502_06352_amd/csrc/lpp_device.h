// Device code that the attention kernels share.
#ifndef LPP_DEVICE_H_
#define LPP_DEVICE_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {   // round to nearest even (hardware convert)
  const bf16x2 v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

// 16- and 8-byte accesses that are visible device-wide once they have completed (the cache policy
// of a device-scope atomic, on whole vectors): what the blocks of one head exchange their partial
// results with inside one launch.  `off` is a byte offset into the buffer behind `rsrc`.
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
constexpr int kDeviceScope = 16;     // sc1
__device__ __forceinline__ __amdgpu_buffer_rsrc_t device_buffer(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ void store_dev(__amdgpu_buffer_rsrc_t r, uint32_t off, float4 v) {
  const u32x4 x = {__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)};
  __builtin_amdgcn_raw_buffer_store_b128(x, r, (int)off, 0, kDeviceScope);
}
__device__ __forceinline__ void store_dev(__amdgpu_buffer_rsrc_t r, uint32_t off, float2 v) {
  const u32x2 x = {__float_as_uint(v.x), __float_as_uint(v.y)};
  __builtin_amdgcn_raw_buffer_store_b64(x, r, (int)off, 0, kDeviceScope);
}
__device__ __forceinline__ float4 load_dev4(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, kDeviceScope);
  return make_float4(__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w));
}
__device__ __forceinline__ float2 load_dev2(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(r, (int)off, 0, kDeviceScope);
  return make_float2(__uint_as_float(x.x), __uint_as_float(x.y));
}

// e^t for t <= 0 (0 below -200, NaN stays): the hardware's 2^x on t log2 e, whose rounding is taken back to first
// order.  Without that, scores of a few units cost a fifth of the accuracy; expf keeps it, but its registers
// spill in the kernel (12 bytes a lane at rows of 64).
__device__ __forceinline__ float exp_neg(float t) {
  constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
  t = t < -200.f ? -200.f : t;
  const float x = t * kLog2e, r = __builtin_amdgcn_exp2f(x);
  return __builtin_fmaf(r, __builtin_fmaf(t, kLog2e, -x) * kLn2, r);
}

}  // namespace

#endif  // LPP_DEVICE_H_
