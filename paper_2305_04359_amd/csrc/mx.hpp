// Microscaled 4-bit rows: what the kernels on them share.
#pragma once
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "driver_internal.hpp"

namespace annmi {

constexpr u32 MX_STEP = 128;        // elements of a step: what one scaled matrix instruction takes of a row
constexpr u32 MX_STEP_BYTES = 64;   // their codes
constexpr u32 MX_STEP_SCALES = 4;   // their scale bytes
constexpr u32 MX_MOST_D = 65536;
constexpr u64 MX_MOST_ROWS = (1ull << 31) - 1;

constexpr u32 mx_steps(u32 d) { return (d + MX_STEP - 1) / MX_STEP; }

// 4-bit rows as the kernels take them
struct MxRows {
  const uint8_t* codes;
  const uint8_t* scales;
  u32 n;
  u32 steps;
};

using v4i = int __attribute__((ext_vector_type(4)));
using v8i = int __attribute__((ext_vector_type(8)));
using v4f = float __attribute__((ext_vector_type(4)));
using v8bf = __bf16 __attribute__((ext_vector_type(8)));
using v2bf = __bf16 __attribute__((ext_vector_type(2)));

// D = C + A B over 128 elements of 4 bits: lane l holds row (A) or column (B) l & 15, elements 32 (l >> 4) and
// on, and the scale byte of that block; D's column is l & 15 too, its rows 4 (l >> 4) and the three after.
__device__ __forceinline__ v4f mx_mfma(v4i a, v4i b, v4f c, int scale_a, int scale_b) {
  const v8i x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, scale_a, 0, scale_b);
}

// 2^(b - 127) of a scale byte; NaN for 255 (and 2^-127, a subnormal number, for 0)
__device__ __forceinline__ float mx_scale(u32 b) {
  return __uint_as_float(b == 0 ? 1u << 22 : b == 255 ? 0x7FC00000u : b << 23);
}

template <typename T>
__device__ __forceinline__ float mx_float(T v) {
  return static_cast<float>(v);
}
template <>
__device__ __forceinline__ float mx_float<__half>(__half v) {
  return __half2float(v);
}
template <typename T>
__device__ __forceinline__ T mx_round(float v);
template <>
__device__ __forceinline__ float mx_round<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ __half mx_round<__half>(float v) {
  return __float2half_rn(v);
}
template <>
__device__ __forceinline__ __bf16 mx_round<__bf16>(float v) {
  return static_cast<__bf16>(v);
}

// N elements that follow each other, for one load or store where the address allows
template <typename T, int N>
struct alignas(sizeof(T) * N) Pack {
  T v[N];
};
// N elements wherever they begin, for one load or store of all
template <typename T, int N>
struct __attribute__((packed, aligned(alignof(T)))) AnyPack {
  T v[N];
};

// a larger key for a larger float; 0 for NaN
__device__ __forceinline__ u32 float_key(float f) {
  const u32 b = __float_as_uint(f + 0.0f);
  return f != f ? 0u : (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_float(u32 k) { return __uint_as_float((k >> 31) ? k & 0x7FFFFFFFu : ~k); }

// Stands where lanes of one wave read from LDS what others of it wrote, and before they write there again.  The hardware
// keeps a wave's accesses to LDS in order; this has the compiler keep them too, and takes no instruction.
__device__ __forceinline__ void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

inline bool aligned_to(const void* p, u64 bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
constexpr u64 dtype_bytes(int t) { return t == ANN_F32 ? 4 : t == ANN_F16 || t == ANN_BF16 ? 2 : t == ANN_U8 || t == ANN_I8 ? 1 : 0; }

// the checks that all calls on 4-bit rows make of one set of them
int check_mx_rows(const char* what, const uint8_t* codes, const uint8_t* scales, u64 n, u32 d);

}  // namespace annmi
