// Rows to microscaled 4-bit codes and back.
#include <type_traits>

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
  uint8_t* codes;
  uint8_t* scales;
  float* norms;
};

// exchanges inside 16 lanes, by one instruction each
template <int CTRL>
__device__ __forceinline__ u32 dpp(u32 v) {
  return (u32)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true);
}
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_ROT4 = 0x124, DPP_ROT8 = 0x128;
template <int CTRL>
__device__ __forceinline__ float dpp_sum(float v) {
  return v + __uint_as_float(dpp<CTRL>(__float_as_uint(v)));
}

// Four lanes take 32 elements, eight each: their largest magnitude by two exchanges, then the codes.  LPR lanes
// (16, 32 or 64: one, two or four steps) take a row, longer rows in turns; a wave asks for four such pieces of rows
// at once.  A million int8 rows of 100 take 55 us, 3.1 TB/s of the 4.9 that a copy reaches: rows of bytes are bound by
// vector instructions (1.1 a cycle and compute unit), wider types by memory: fp16 60 us, 4.5 TB/s, and fp32 92 us, 5.1 TB/s
// (250,000 rows of 1,024: bytes 131 us, 3.0 TB/s, fp16 144 us, 4.5 TB/s, fp32 211 us, 5.5 TB/s).
// WIDE: every row has eight elements at least; eight are then read at once, past d too, but in the last row, whose
// last eight are read where these reach its end.
template <typename T, int LPR, bool WIDE>
__global__ __launch_bounds__(256) void mx_quantize_kernel(QuantizeArgs a) {
  constexpr u32 AHEAD = 4, PER_BLOCK = 256 / LPR;
  const u32 lane = threadIdx.x % LPR;
  const u32 turns = (a.steps + LPR / 16 - 1) / (LPR / 16);  // 1 but for rows of more than four steps
  // the rows of a pass: of AHEAD turns of one row where rows are long, else of AHEAD rows
  const bool rows_ahead = turns == 1;
  const u64 stride = (u64)gridDim.x * PER_BLOCK;
  for (u64 r0 = (u64)blockIdx.x * PER_BLOCK + threadIdx.x / LPR; r0 < a.n; r0 += rows_ahead ? stride * AHEAD : stride) {
    float norm[AHEAD] = {};
    for (u32 s0 = 0; s0 < turns; s0 += AHEAD) {
      AnyPack<T, 8> in[AHEAD];
      u64 row[AHEAD];
      u32 at[AHEAD];
      bool on[AHEAD];
      u32 early[AHEAD];
#pragma unroll
      for (u32 u = 0; u < AHEAD; ++u) {
        row[u] = rows_ahead ? r0 + stride * u : r0;
        at[u] = (rows_ahead ? 0 : s0 + u) * (LPR / 16 * MX_STEP) + lane * 8;  // the lane's first element
        on[u] = row[u] < a.n && at[u] < a.steps * MX_STEP;
        const u64 r = min(row[u], (u64)a.n - 1);
        const T* from = reinterpret_cast<const T*>(a.x) + r * a.ldx;
        if (WIDE) {
          const u32 first = at[u] < a.d ? at[u] : 0;
          early[u] = (a.n - 1 - r) * a.ldx < 7 && first + 8 > a.d ? first + 8 - a.d : 0;
          in[u] = *reinterpret_cast<const AnyPack<T, 8>*>(from + (first - early[u]));
        } else {
#pragma unroll
          for (u32 e = 0; e < 8; ++e) in[u].v[e] = from[min(at[u] + e, a.d - 1)];
        }
      }
#pragma unroll
      for (u32 u = 0; u < AHEAD; ++u) {
        if (!on[u]) continue;  // (whole rows or steps at a time: 16 lanes alike)
        float v[8];
        u32 most = 0;
        if constexpr (WIDE && sizeof(T) == 1) {  // bytes: eight at once where they can be (0 is a byte of 0)
          u64 bytes = __builtin_bit_cast(u64, in[u]) >> (8 * early[u]);
          const u32 there = at[u] < a.d ? min(a.d - at[u], 8u) : 0;
          bytes &= there ? ~0ull >> (64 - 8 * there) : 0ull;
          float m = 0.0f;
#pragma unroll
          for (u32 e = 0; e < 8; ++e) {
            v[e] = mx_float(static_cast<T>(bytes >> (8 * e)));
            m = __builtin_fmaxf(m, __builtin_fabsf(v[e]));
          }
          most = __float_as_uint(m);
        } else {
#pragma unroll
          for (u32 e = 0; e < 8; ++e) v[e] = mx_float(static_cast<T>(in[u].v[e]));
          if (WIDE && early[u])
            for (u32 k = 0; k < early[u]; ++k)
#pragma unroll
              for (u32 e = 0; e < 7; ++e) v[e] = v[e + 1];
#pragma unroll
          for (u32 e = 0; e < 8; ++e) v[e] = at[u] + e < a.d ? v[e] : 0.0f;
          // magnitudes compare like their bits, and so do NaN and infinity
#pragma unroll
          for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
        }
        most = max(most, dpp<DPP_XOR1>(most));
        most = max(most, dpp<DPP_XOR2>(most));
        const bool fine = most < 0x7F800000u;
        const u32 exponent = most >> 23;
        const u32 byte = !fine ? 255u : exponent > 2 ? exponent - 2 : 0u;
        const float inverse = __uint_as_float((254u - byte) << 23);  // 2^(127 - byte); of no use where byte is 255
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= inverse;
        // (the scale is in the factor: the instruction gets 1)
        u32 code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], 1.0f, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], 1.0f, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], 1.0f, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], 1.0f, 3);
        if (!fine) code = 0;
        if (a.norms) {
          using v2f = float __attribute__((ext_vector_type(2)));
          const v2f p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 3)};
          float sum = 0.0f;
#pragma unroll
          for (int i = 0; i < 4; ++i) sum = __builtin_fmaf(p[i].x, p[i].x, __builtin_fmaf(p[i].y, p[i].y, sum));
          const float scale = mx_scale(byte);
          float& to = norm[rows_ahead ? u : 0];
          to = __builtin_fmaf(sum * scale, scale, to);
        }
        // a step's four scale bytes meet in one word
        u32 word = (at[u] < a.d ? byte : 0u) << (lane % 16 / 4 * 8);
        word |= dpp<DPP_ROT4>(word);
        word |= dpp<DPP_ROT8>(word);
        const u64 step = row[u] * a.steps + at[u] / MX_STEP;
        reinterpret_cast<u32*>(a.codes)[step * 16 + lane % 16] = code;
        if (lane % 16 == 0) reinterpret_cast<u32*>(a.scales)[step] = word;
      }
    }
    if (a.norms) {
#pragma unroll
      for (u32 u = 0; u < AHEAD; ++u) {
        float sum = dpp_sum<DPP_XOR1>(norm[u]);
        sum = dpp_sum<DPP_XOR2>(sum);
        sum = dpp_sum<DPP_ROT4>(sum);
        sum = dpp_sum<DPP_ROT8>(sum);
#pragma unroll
        for (int w = 16; w < LPR; w *= 2) sum += __shfl_xor(sum, w);
        const u64 r = r0 + stride * u;
        if (lane == 0 && (u == 0 || rows_ahead) && r < a.n) a.norms[r] = sum;
        if (!rows_ahead) break;
      }
    }
  }
}

template <typename T, bool WIDE>
hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t s) {
  const u32 lpr = a.steps == 1 ? 16 : a.steps == 2 ? 32 : 64;
  // four rows for each place, where a turn takes a row
  const u64 per = 256 / lpr * (a.steps <= 4 ? 4 : 1), blocks = ((u64)a.n + per - 1) / per;
  const u32 grid = (u32)(blocks < (1u << 20) ? blocks : (1u << 20));
  auto kernel = mx_quantize_kernel<T, 16, WIDE>;
  if constexpr (WIDE) {  // (others have one step)
    if (lpr == 32) kernel = mx_quantize_kernel<T, 32, WIDE>;
    if (lpr == 64) kernel = mx_quantize_kernel<T, 64, WIDE>;
  }
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t s) {
  return a.d >= 8 ? launch_quantize<T, true>(a, s) : launch_quantize<T, false>(a, s);
}

struct DequantizeArgs {
  const uint8_t* codes;
  const uint8_t* scales;
  u64 n;
  u32 steps, d;
  char* out;
  u64 ldo;
};

// A thread takes 16 bytes of a row of `out`, and the same ones of other rows in turn.  Bound by memory: a million rows of
// 100 to fp32 take 114 us, 4.1 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(DequantizeArgs a) {
  constexpr u32 E = 16 / sizeof(T), AHEAD = 4;  // elements; rows at a time
  using Codes = std::conditional_t<E == 4, unsigned short, u32>;
  using v2f = float __attribute__((ext_vector_type(2)));
  const u32 pieces = (a.d + E - 1) / E;
  const u32 across = pieces < 256 ? pieces : 256, rows = 256 / across;  // of a block
  const u32 sub = threadIdx.x / across;
  if (sub >= rows) return;
  const u64 stride = (u64)gridDim.x * rows;
  for (u64 r0 = (u64)blockIdx.x * rows + sub; r0 < a.n; r0 += stride * AHEAD) {
    for (u32 c = threadIdx.x % across; c < pieces; c += across) {
      u32 code[AHEAD];
      float scale[AHEAD];
#pragma unroll
      for (u32 u = 0; u < AHEAD; ++u) {
        const u64 r = min(r0 + stride * u, a.n - 1) * a.steps;
        code[u] = reinterpret_cast<const Codes*>(a.codes + r * MX_STEP_BYTES)[c];
        scale[u] = mx_scale(a.scales[r * MX_STEP_SCALES + c * E / 32]);
      }
#pragma unroll
      for (u32 u = 0; u < AHEAD; ++u) {
        if (r0 + stride * u >= a.n) break;
        v2f p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], 1.0f, 1)};
        if (E == 8) p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], 1.0f, 2), p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], 1.0f, 3);
        AnyPack<T, E> o;
#pragma unroll
        for (u32 j = 0; j < E / 2; ++j) {
          o.v[2 * j] = mx_round<T>(p[j].x * scale[u]);
          o.v[2 * j + 1] = mx_round<T>(p[j].y * scale[u]);
        }
        T* to = reinterpret_cast<T*>(a.out) + (r0 + stride * u) * a.ldo + c * E;
        if (c * E + E <= a.d) {
          *reinterpret_cast<AnyPack<T, E>*>(to) = o;
        } else {
#pragma unroll
          for (u32 j = 0; j < E; ++j)
            if (c * E + j < a.d) to[j] = o.v[j];
        }
      }
    }
  }
}

template <typename T>
hipError_t launch_dequantize(const DequantizeArgs& a, hipStream_t s) {
  const u32 pieces = (u32)((a.d + 16 / sizeof(T) - 1) / (16 / sizeof(T))), rows = pieces < 256 ? 256 / pieces : 1;
  const u64 blocks = (a.n + 4 * rows - 1) / (4 * rows);
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
  QuantizeArgs a{static_cast<const char*>(x_dev), ldx, (u32)n, d, mx_steps(d), codes_dev, scales_dev, norms_dev};
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
  DequantizeArgs a{codes_dev, scales_dev, n, mx_steps(d), d, static_cast<char*>(out_dev), ldo};
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
