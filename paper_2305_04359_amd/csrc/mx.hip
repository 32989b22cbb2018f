// Rows to microscaled 4-bit codes and back.
#include "mx.hpp"

namespace annmi {

int check_mx_rows(const char* what, const uint8_t* codes, const uint8_t* scales, u64 n, u32 d) {
  if (n > MX_MOST_ROWS) return fail(ANN_EINVAL, "%s: rows must stay below 2^31", what);
  if (d < 1 || d > MX_MOST_D) return fail(ANN_EINVAL, "%s: d must be 1 to %u", what, MX_MOST_D);
  if (n == 0) return ANN_OK;
  if (!codes || !scales) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(codes, 16)) return fail(ANN_EINVAL, "%s: codes must be 16-byte aligned", what);
  if (!aligned_to(scales, 4)) return fail(ANN_EINVAL, "%s: scales must be 4-byte aligned", what);
  return ANN_OK;
}

struct QuantizeArgs {
  const char* x;
  u64 ldx;
  u32 n, d, steps;
  u32 wide;  // every row can be read eight elements at a time
  uint8_t* codes;
  uint8_t* scales;
  float* norms;
};

// Four lanes take 32 elements, eight each: their largest magnitude by two exchanges, then the codes.  LPR lanes
// (16, 32 or 64: one, two or four steps) take a row, longer rows in turns; whole waves then read and write
// runs of memory.  Bound by memory: a byte in for each element at least, 17 bytes out for 32.
template <typename T, int LPR>
__global__ __launch_bounds__(256) void mx_quantize_kernel(QuantizeArgs a) {
  const u32 lane = threadIdx.x % LPR;
  const u32 per_block = 256 / LPR;
  for (u64 r = (u64)blockIdx.x * per_block + threadIdx.x / LPR; r < a.n; r += (u64)gridDim.x * per_block) {
    const T* row = reinterpret_cast<const T*>(a.x) + r * a.ldx;
    float norm = 0.0f;
    for (u32 s = 0; s < a.steps; s += LPR / 16) {
      const u32 at = s * MX_STEP + lane * 8;  // the lane's first element
      float v[8];
      if (a.wide && at + 8 <= a.d) {
        const Pack<T, 8> p = *reinterpret_cast<const Pack<T, 8>*>(row + at);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = mx_float(p.v[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = at + i < a.d ? mx_float(row[at + i]) : 0.0f;
      }
      // magnitudes compare like their bits, and so do NaN and infinity
      u32 most = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
      most = max(most, (u32)__shfl_xor((int)most, 1));
      most = max(most, (u32)__shfl_xor((int)most, 2));
      const bool fine = most < 0x7F800000u;
      const u32 exponent = most >> 23;
      const u32 byte = !fine ? 255u : exponent > 2 ? exponent - 2 : 0u;
      const float inverse = __uint_as_float((254u - byte) << 23);  // 2^(127 - byte); of no use where byte is 255
      u32 code = 0;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        // (the scale is in the factor: the instruction gets 1)
        const float lo = v[i] * inverse, hi = v[i + 1] * inverse;
        if (i == 0) code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, lo, hi, 1.0f, 0);
        if (i == 2) code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, lo, hi, 1.0f, 1);
        if (i == 4) code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, lo, hi, 1.0f, 2);
        if (i == 6) code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, lo, hi, 1.0f, 3);
      }
      if (!fine) code = 0;
      if (a.norms) {
        using v2f = float __attribute__((ext_vector_type(2)));
        const v2f p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 3)};
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = __builtin_fmaf(p[i].x, p[i].x, __builtin_fmaf(p[i].y, p[i].y, sum));
        const float scale = mx_scale(byte);
        norm = __builtin_fmaf(sum * scale, scale, norm);
      }
      const u32 step = s + lane / 16;
      if (step < a.steps) {
        reinterpret_cast<u32*>(a.codes)[(r * a.steps + step) * 16 + lane % 16] = code;
        if (lane % 4 == 0) a.scales[(r * a.steps + step) * 4 + lane % 16 / 4] = (uint8_t)(at < a.d ? byte : 0u);
      }
    }
    if (a.norms) {
#pragma unroll
      for (int w = 1; w < LPR; w *= 2) norm += __shfl_xor(norm, w);
      if (lane == 0) a.norms[r] = norm;
    }
  }
}

template <typename T>
hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t s) {
  const u32 lpr = a.steps == 1 ? 16 : a.steps == 2 ? 32 : 64;
  const u64 blocks = ((u64)a.n * lpr + 255) / 256;
  const u32 grid = (u32)(blocks < (1u << 20) ? blocks : (1u << 20));
  if (lpr == 16)
    hipLaunchKernelGGL((mx_quantize_kernel<T, 16>), dim3(grid), dim3(256), 0, s, a);
  else if (lpr == 32)
    hipLaunchKernelGGL((mx_quantize_kernel<T, 32>), dim3(grid), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((mx_quantize_kernel<T, 64>), dim3(grid), dim3(256), 0, s, a);
  return hipGetLastError();
}

struct DequantizeArgs {
  const uint8_t* codes;
  const uint8_t* scales;
  u64 pieces;  // of eight elements, in all rows (padding included)
  u32 steps, d;
  char* out;
  u64 ldo;
  u32 wide;
};

// A lane per eight elements.  Bound by memory.
template <typename T>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(DequantizeArgs a) {
  for (u64 i = (u64)blockIdx.x * 256 + threadIdx.x; i < a.pieces; i += (u64)gridDim.x * 256) {
    const u64 r = i / (a.steps * 16);
    const u32 at = (u32)(i - r * (a.steps * 16)) * 8;
    if (at >= a.d) continue;
    const u32 code = reinterpret_cast<const u32*>(a.codes)[i];
    const float scale = mx_scale(a.scales[i / 4]);
    using v2f = float __attribute__((ext_vector_type(2)));
    const v2f p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 1),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 3)};
    Pack<T, 8> o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o.v[2 * j] = mx_round<T>(p[j].x * scale);
      o.v[2 * j + 1] = mx_round<T>(p[j].y * scale);
    }
    T* to = reinterpret_cast<T*>(a.out) + r * a.ldo + at;
    if (a.wide && at + 8 <= a.d) {
      *reinterpret_cast<Pack<T, 8>*>(to) = o;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (at + j < a.d) to[j] = o.v[j];
    }
  }
}

template <typename T>
hipError_t launch_dequantize(const DequantizeArgs& a, hipStream_t s) {
  const u64 blocks = (a.pieces + 255) / 256;
  hipLaunchKernelGGL(mx_dequantize_kernel<T>, dim3((u32)(blocks < (1u << 20) ? blocks : (1u << 20))), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace annmi

using namespace annmi;

extern "C" {

int ann_mx_quantize(const void* x_dev, uint64_t n, uint32_t d, ann_dtype dtype, uint64_t ldx, uint8_t* codes_dev,
                    uint8_t* scales_dev, float* norms_dev, void* stream) try {
  const u64 esz = dtype_bytes(dtype);
  if (esz == 0) return fail(ANN_EINVAL, "unknown dtype");
  int rc = check_mx_rows("ann_mx_quantize", codes_dev, scales_dev, n, d);
  if (rc) return rc;
  if (ldx < d) return fail(ANN_EINVAL, "ldx must be at least d");
  if (n == 0) return ANN_OK;
  if (!x_dev) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(x_dev, esz) || !aligned_to(norms_dev, 4)) return fail(ANN_EINVAL, "x or norms not aligned to their elements");
  QuantizeArgs a{static_cast<const char*>(x_dev), ldx, (u32)n, d, mx_steps(d), 0, codes_dev, scales_dev, norms_dev};
  a.wide = aligned_to(x_dev, 8 * esz) && ldx % 8 == 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (dtype) {
    case ANN_U8: HIP_TRY(launch_quantize<uint8_t>(a, st)); break;
    case ANN_I8: HIP_TRY(launch_quantize<int8_t>(a, st)); break;
    case ANN_F16: HIP_TRY(launch_quantize<__half>(a, st)); break;
    case ANN_BF16: HIP_TRY(launch_quantize<__bf16>(a, st)); break;
    default: HIP_TRY(launch_quantize<float>(a, st)); break;
  }
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

int ann_mx_dequantize(const uint8_t* codes_dev, const uint8_t* scales_dev, uint64_t n, uint32_t d, void* out_dev,
                      ann_dtype dtype, uint64_t ldo, void* stream) try {
  const u64 esz = dtype_bytes(dtype);
  if (esz < 2) return fail(ANN_EINVAL, "the values come as ANN_F32, ANN_F16 or ANN_BF16");
  int rc = check_mx_rows("ann_mx_dequantize", codes_dev, scales_dev, n, d);
  if (rc) return rc;
  if (ldo < d) return fail(ANN_EINVAL, "ldo must be at least d");
  if (n == 0) return ANN_OK;
  if (!out_dev) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(out_dev, esz)) return fail(ANN_EINVAL, "out not aligned to its elements");
  DequantizeArgs a{codes_dev, scales_dev, n * mx_steps(d) * 16, mx_steps(d), d, static_cast<char*>(out_dev), ldo, 0};
  a.wide = aligned_to(out_dev, 8 * esz) && ldo % 8 == 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (dtype) {
    case ANN_F16: HIP_TRY(launch_dequantize<__half>(a, st)); break;
    case ANN_BF16: HIP_TRY(launch_dequantize<__bf16>(a, st)); break;
    default: HIP_TRY(launch_dequantize<float>(a, st)); break;
  }
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

}  // extern "C"
