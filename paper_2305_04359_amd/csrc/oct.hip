// Rows or columns to 8-bit floating point with a scale for each 128 elements, and back.
#include <algorithm>
#include <type_traits>

#include "oct.hpp"

namespace annmi {

int check_oct_rows(const char* what, const uint8_t* codes, const uint8_t* scales, u64 n, u32 d) {
  if (n > OCT_MOST_ROWS) return fail(ANN_EINVAL, "%s: rows must stay below 2^30", what);
  if (d < 1 || d > OCT_MOST_D) return fail(ANN_EINVAL, "%s: d must be 1 to %u", what, OCT_MOST_D);
  if (n * oct_steps(d) >> 32) return fail(ANN_EINVAL, "%s: rows * ceil(d / 128) must stay below 2^32", what);
  if (n == 0) return ANN_OK;
  if (!codes || !scales) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(codes, 16)) return fail(ANN_EINVAL, "%s: codes must be 16-byte aligned", what);
  if (!aligned_to(scales, 4)) return fail(ANN_EINVAL, "%s: scales must be 4-byte aligned", what);
  return ANN_OK;
}

struct OctQuantizeArgs {
  const char* x;
  u64 ldx;
  u32 n, d, steps;
  uint8_t* codes;
  u32* scales;
};

// The scale byte of 128 elements whose largest magnitude has the bits `most`: e + 127 for the least e of at least
// -127 with most <= 448 * 2^e.  448 is 1.75 * 2^8, so that the mantissa decides whether the exponent less 8 is enough.
__device__ __forceinline__ u32 oct_scale_byte(u32 most) {
  if (most >= 0x7F800000u) return 255u;  // infinite or NaN
  const u32 e = (most >> 23) + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return e > 8 ? e - 8 : 0u;
}
// 2^(127 - byte), exact; of no use where byte is 255
__device__ __forceinline__ float oct_inverse(u32 byte) { return __uint_as_float((254u - byte) << 23); }
// four elements as four codes, to the nearest, ties to even; none is above 448
__device__ __forceinline__ u32 oct_codes(float a, float b, float c, float d) {
  const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (u32)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true);
}

// exchanges inside 16 lanes, by one instruction each
template <int CTRL>
__device__ __forceinline__ u32 row_max(u32 v) {
  return max(v, (u32)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ u32 max_of_16(u32 v) {
  v = row_max<0xB1>(v);   // the neighbour
  v = row_max<0x4E>(v);   // two away
  v = row_max<0x124>(v);  // four and eight around
  return row_max<0x128>(v);
}

// Rows.  Sixteen lanes take a step, eight elements each, whichever row it is of: steps without gaps are where their codes lie.
// A row a wave, four turns ahead, takes 291 us for 131,072 x 4,096 bf16, 55 for 100,000 x 640 bytes (half of its lanes have nothing),
// 242 for 64 x 200,000 fp32 and 5 for 1 x 4,096 bf16; so 268 (5.9 TB/s), 25, 14 and 2 (200,000 x 1,000 fp32 176 and 185).
// Stores past the caches take 260 for the first, but the products that read the codes next lose more.
// WIDE: every row has eight elements at least; eight are then read at once, past d too, but in the last rows, whose
// last eight are read where these would reach past the end of the last row.
constexpr u32 ROW_STEPS = 16;
template <typename T>
constexpr u32 row_ahead = sizeof(T) == 1 ? 4 : 2;  // steps that a thread asks for at once (of bytes 25 us, with two 28; bf16 268, with four 287)
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void oct_quantize_kernel(OctQuantizeArgs a, u64 items, u32 reciprocal) {
  constexpr u32 ROW_AHEAD = row_ahead<T>, ROW_TILE = ROW_STEPS * ROW_AHEAD;
  const u32 lane = threadIdx.x % 16, group = threadIdx.x / 16;
  const u32 words = oct_words(a.steps);
  for (u64 base = (u64)blockIdx.x * ROW_TILE; base < items; base += (u64)gridDim.x * ROW_TILE) {
    const u64 row0 = (u32)base / a.steps;
    const u32 step0 = (u32)(base - row0 * a.steps);
    AnyPack<T, 8> in[ROW_AHEAD];
    u64 row[ROW_AHEAD];
    u32 step[ROW_AHEAD], early[ROW_AHEAD];
#pragma unroll
    for (u32 u = 0; u < ROW_AHEAD; ++u) {
      const u32 from0 = step0 + u * ROW_STEPS + group;
      const u32 rows = a.steps == 1 ? from0 : __umulhi(from0, reciprocal);
      step[u] = from0 - rows * a.steps;
      row[u] = row0 + rows;
      const u64 r = min(row[u], (u64)a.n - 1);
      const T* from = reinterpret_cast<const T*>(a.x) + r * a.ldx;
      const u32 at = step[u] * OCT_STEP + lane * 8;  // the lane's first element
      early[u] = 0;
      if (WIDE) {
        const u32 first = at < a.d ? at : 0;
        early[u] = (a.n - 1 - r) * a.ldx < 7 && first + 8 > a.d ? first + 8 - a.d : 0;
        in[u] = *reinterpret_cast<const AnyPack<T, 8>*>(from + (first - early[u]));
      } else {
#pragma unroll
        for (u32 e = 0; e < 8; ++e) in[u].v[e] = from[min(at + e, a.d - 1)];
      }
    }
#pragma unroll
    for (u32 u = 0; u < ROW_AHEAD; ++u) {
      const u64 item = base + u * ROW_STEPS + group;
      if (item >= items) break;  // (all lanes of a step alike)
      const u32 at = step[u] * OCT_STEP + lane * 8;
      float v[8];
#pragma unroll
      for (u32 e = 0; e < 8; ++e) v[e] = mx_float(static_cast<T>(in[u].v[e]));
      if (at + 8 > a.d) {  // the row's end
        if (WIDE && early[u])
          for (u32 k = 0; k < early[u]; ++k)
#pragma unroll
            for (u32 e = 0; e < 7; ++e) v[e] = v[e + 1];
#pragma unroll
        for (u32 e = 0; e < 8; ++e) v[e] = at + e < a.d ? v[e] : 0.0f;
      }
      u32 most = 0;  // magnitudes compare like their bits, and so do NaN and infinity
#pragma unroll
      for (u32 e = 0; e < 8; ++e) most = max(most, __float_as_uint(v[e]) & 0x7FFFFFFFu);
      const u32 byte = oct_scale_byte(max_of_16(most));
      const float inverse = oct_inverse(byte);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= inverse;
      Pack<u32, 2> code = {{oct_codes(v[0], v[1], v[2], v[3]), oct_codes(v[4], v[5], v[6], v[7])}};
      if (byte == 255) code = {{0, 0}};
      *reinterpret_cast<Pack<u32, 2>*>(a.codes + item * OCT_STEP + lane * 8) = code;
      // the step's byte, and the rest of the last word
      const u32 scale = step[u] + lane;
      if (lane == 0 || (step[u] + 1 == a.steps && scale < words * 4))
        reinterpret_cast<uint8_t*>(a.scales)[row[u] * words * 4 + scale] = lane == 0 ? (uint8_t)byte : 0;
    }
  }
}

// Columns: row i of the result is column i of x, which has d rows.  A workgroup takes a step of COLS columns: a thread EACH
// elements of four neighbouring columns, whose maxima meet in LDS; through LDS the codes get into whole rows of 128 bytes.
// Inputs stay the words that they are in memory until they are codes, with maxima of two 16-bit ones at once: held as fp32 they
// take 188 registers, two waves a SIMD, and 67 us from memory for 4,096 columns of 16,384 bf16, so 97 and 43, 4.6 TB/s.
// 16,384 columns of 4,096 fp32 come past the caches in 65 us, 5.2 TB/s, and through them in 81, also from a cache that has them
// (67 MB 15 and 21); to 16-bit ones it makes no difference.
constexpr u32 COLS = 128;
constexpr u32 COLUMN_EACH = 16, COLUMN_PARTS = OCT_STEP / COLUMN_EACH, COLUMN_THREADS = COLS / 4 * COLUMN_PARTS;
// four neighbouring elements of a row, as they are in memory
template <typename T>
using Four = Pack<u32, sizeof(T)>;
template <typename T>
__device__ __forceinline__ Four<T> four_at(const T* from) {
  if constexpr (sizeof(T) == 4) {
    using Streamed = v4i __attribute__((aligned(4)));
    return __builtin_bit_cast(Four<T>, v4i(__builtin_nontemporal_load(reinterpret_cast<const Streamed*>(from))));
  } else {
    return __builtin_bit_cast(Four<T>, *reinterpret_cast<const AnyPack<T, 4>*>(from));
  }
}
template <typename T>
__device__ __forceinline__ float four_get(const Four<T>& four, u32 k) {
  if constexpr (sizeof(T) == 4)
    return __uint_as_float(four.v[k]);
  else if constexpr (std::is_same_v<T, __bf16>)
    return __uint_as_float(k % 2 ? four.v[k / 2] & 0xFFFF0000u : four.v[k / 2] << 16);
  else if constexpr (sizeof(T) == 2)
    return mx_float(__builtin_bit_cast(__half, (uint16_t)(four.v[k / 2] >> (k % 2 * 16))));
  else if constexpr (std::is_same_v<T, int8_t>)
    return (float)(int8_t)(four.v[0] >> (8 * k));
  else
    return (float)(uint8_t)(four.v[0] >> (8 * k));
}
// the largest magnitudes of EACH elements of four columns, as fp32's bits
template <typename T>
__device__ __forceinline__ Pack<u32, 4> four_most(const Four<T> (&in)[COLUMN_EACH]) {
  Pack<u32, 4> most = {{0, 0, 0, 0}};
  if constexpr (sizeof(T) == 2) {  // magnitudes compare like their bits: two at once
    using v2h = uint16_t __attribute__((ext_vector_type(2)));
    v2h low = {0, 0}, high = {0, 0};
#pragma unroll
    for (u32 e = 0; e < COLUMN_EACH; ++e) {
      low = __builtin_elementwise_max(low, __builtin_bit_cast(v2h, in[e].v[0] & 0x7FFF7FFFu));
      high = __builtin_elementwise_max(high, __builtin_bit_cast(v2h, in[e].v[1] & 0x7FFF7FFFu));
    }
    const Four<T> all = {{__builtin_bit_cast(u32, low), __builtin_bit_cast(u32, high)}};
#pragma unroll
    for (u32 k = 0; k < 4; ++k) most.v[k] = __float_as_uint(four_get<T>(all, k));
  } else if constexpr (sizeof(T) == 1) {  // as whole numbers of 16 bits, two at once: columns 0 and 2, 1 and 3
    using v2s = std::conditional_t<std::is_same_v<T, int8_t>, int16_t, uint16_t> __attribute__((ext_vector_type(2)));
    v2s top[2] = {}, low[2] = {};
#pragma unroll
    for (u32 e = 0; e < COLUMN_EACH; ++e) {
      const v2s both = __builtin_bit_cast(v2s, in[e].v[0]), part[2] = {(v2s)(both << 8) >> 8, both >> 8};
#pragma unroll
      for (u32 o = 0; o < 2; ++o) {
        top[o] = __builtin_elementwise_max(top[o], part[o]);
        low[o] = __builtin_elementwise_min(low[o], part[o]);
      }
    }
#pragma unroll
    for (u32 k = 0; k < 4; ++k) most.v[k] = __float_as_uint((float)max((int)top[k % 2][k / 2], -(int)low[k % 2][k / 2]));
  } else {
#pragma unroll
    for (u32 e = 0; e < COLUMN_EACH; ++e)
#pragma unroll
      for (u32 k = 0; k < 4; ++k) most.v[k] = max(most.v[k], __float_as_uint(four_get<T>(in[e], k)) & 0x7FFFFFFFu);
  }
  return most;
}
template <typename T>
__global__ __launch_bounds__(COLUMN_THREADS, 4) void oct_columns_kernel(OctQuantizeArgs a, u32 across, u64 tiles) {
  using Part = Pack<u32, COLUMN_EACH / 4>;  // a thread's codes of a column
  __shared__ u32 most_of[COLUMN_PARTS][COLS];
  __shared__ __align__(16) char codes[COLS * OCT_STEP];
  const u32 c = threadIdx.x % (COLS / 4) * 4, g = threadIdx.x / (COLS / 4);
  const u32 words = oct_words(a.steps);
  for (u64 t = blockIdx.x; t < tiles; t += gridDim.x) {
    const u64 i0 = t % across * COLS;        // the first column
    const u32 step = (u32)(t / across);
    const u32 e0 = step * OCT_STEP + g * COLUMN_EACH;
    const u32 there = (u32)min((u64)COLS, a.n - i0);
    const T* x = reinterpret_cast<const T*>(a.x) + i0;
    Four<T> in[COLUMN_EACH];
    if (there == COLS && step * OCT_STEP + OCT_STEP <= a.d) {
      const T* from = x + (u64)e0 * a.ldx + c;
#pragma unroll
      for (u32 e = 0; e < COLUMN_EACH; ++e) in[e] = four_at<T>(from + e * a.ldx);
    } else {
#pragma unroll
      for (u32 e = 0; e < COLUMN_EACH; ++e) {
        const T* from = x + (u64)min(e0 + e, a.d - 1) * a.ldx;
        if (c + 4 <= there) {
          in[e] = four_at<T>(from + c);
        } else {
          AnyPack<T, 4> four;
#pragma unroll
          for (u32 k = 0; k < 4; ++k) four.v[k] = from[min(c + k, there - 1)];
          in[e] = __builtin_bit_cast(Four<T>, four);
        }
        if (e0 + e >= a.d)
#pragma unroll
          for (u32 w = 0; w < sizeof(T); ++w) in[e].v[w] = 0;
      }
    }
    *reinterpret_cast<Pack<u32, 4>*>(&most_of[g][c]) = four_most<T>(in);
    __syncthreads();
    // a column's maximum: each thread's four, of all parts
    u32 m[4] = {};
#pragma unroll
    for (u32 o = 0; o < COLUMN_PARTS; ++o) {
      const Pack<u32, 4> other = *reinterpret_cast<const Pack<u32, 4>*>(&most_of[o][c]);
#pragma unroll
      for (u32 k = 0; k < 4; ++k) m[k] = max(m[k], other.v[k]);
    }
#pragma unroll
    for (u32 k = 0; k < 4; ++k) {
      const u32 byte = oct_scale_byte(m[k]);
      const float inverse = oct_inverse(byte);
      Part code;
#pragma unroll
      for (u32 q = 0; q < COLUMN_EACH / 4; ++q)
        code.v[q] = oct_codes(four_get<T>(in[4 * q], k) * inverse, four_get<T>(in[4 * q + 1], k) * inverse, four_get<T>(in[4 * q + 2], k) * inverse,
                              four_get<T>(in[4 * q + 3], k) * inverse);
      if (byte == 255) code = {};
      // pieces of 16 bytes change places by the column's number
      const u32 r = c + k, at = g * COLUMN_EACH;
      *reinterpret_cast<Part*>(codes + r * OCT_STEP + ((at / 16 ^ (r / 4 + r) % 8) * 16 | at % 16)) = code;
      if (g == 0 && r < there) {
        uint8_t* to = reinterpret_cast<uint8_t*>(a.scales) + (i0 + r) * words * 4;
        to[step] = (uint8_t)byte;
        if (step + 1 == a.steps)  // the rest of the last word
          for (u32 o = a.steps; o < words * 4; ++o) to[o] = 0;
      }
    }
    __syncthreads();
    for (u32 r = threadIdx.x / 8; r < there; r += COLUMN_THREADS / 8) {
      const u32 u = threadIdx.x % 8;
      *reinterpret_cast<v4i*>(a.codes + ((i0 + r) * a.steps + step) * OCT_STEP + u * 16) =
          *reinterpret_cast<const v4i*>(codes + r * OCT_STEP + (u ^ (r / 4 + r) % 8) * 16);
    }
    // (the next turn's maxima go where none are read any more; its codes come behind its own barrier)
  }
}

template <typename T, bool WIDE>
hipError_t launch_oct_rows(const OctQuantizeArgs& a, hipStream_t s) {
  constexpr u32 ROW_TILE = ROW_STEPS * row_ahead<T>;
  const u64 items = (u64)a.n * a.steps, blocks = (items + ROW_TILE - 1) / ROW_TILE;
  // 2^32 / steps rounded up: from 2 to 2^13 steps and places below 2^13 + 64 their product's upper half is the quotient
  const u32 reciprocal = (u32)(((1ull << 32) + a.steps - 1) / a.steps);
  hipLaunchKernelGGL((oct_quantize_kernel<T, WIDE>), dim3((u32)std::min<u64>(blocks, 1u << 20)), dim3(256), 0, s, a, items, reciprocal);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_oct_quantize(const OctQuantizeArgs& a, bool columns, hipStream_t s) {
  if (!columns) return a.d >= 8 ? launch_oct_rows<T, true>(a, s) : launch_oct_rows<T, false>(a, s);
  const u32 across = (u32)(((u64)a.n + COLS - 1) / COLS);
  const u64 tiles = (u64)across * a.steps;
  hipLaunchKernelGGL(oct_columns_kernel<T>, dim3((u32)(tiles < (1u << 20) ? tiles : (1u << 20))), dim3(COLUMN_THREADS), 0, s, a, across, tiles);
  return hipGetLastError();
}

struct OctDequantizeArgs {
  const uint8_t* codes;
  const uint8_t* scales;
  u64 n;
  u32 steps, d;
  char* out;
  u64 ldo;
};

// Pieces of 16 bytes of `out`, its rows one after another, two for a thread.  They go past the caches, which also serves who
// reads them next: 4,096 x 16,384 bf16 and a copy of them 87 us from memory, with plain stores 107 (67 MB that a cache holds 41
// and 40).  A row's pieces in turn by one workgroup with plain stores: 131,072 x 4,096 bf16 442 us, so 251 (6.4 TB/s);
// 64 x 200,000 fp32 263 and 14.
constexpr u32 DEQUANTIZE_AHEAD = 2, DEQUANTIZE_TILE = 256 * DEQUANTIZE_AHEAD;
template <typename T>
__global__ __launch_bounds__(256) void oct_dequantize_kernel(OctDequantizeArgs a, u32 pieces, u64 items) {
  constexpr u32 E = 16 / sizeof(T), AHEAD = DEQUANTIZE_AHEAD;
  using v2f = float __attribute__((ext_vector_type(2)));
  using Streamed = v4i __attribute__((aligned(2)));
  const u32 words = oct_words(a.steps);
  for (u64 base = (u64)blockIdx.x * DEQUANTIZE_TILE; base < items; base += (u64)gridDim.x * DEQUANTIZE_TILE) {
    const u64 row0 = items >> 32 ? base / pieces : (u32)base / pieces;
    const u32 p0 = (u32)(base - row0 * pieces);
    Pack<u32, E / 4> code[AHEAD];
    float scale[AHEAD];
    u64 row[AHEAD];
    u32 c[AHEAD];
#pragma unroll
    for (u32 u = 0; u < AHEAD; ++u) {
      const u32 p = p0 + u * 256 + threadIdx.x, rows = p / pieces;
      c[u] = p - rows * pieces;
      row[u] = row0 + rows;
      const u64 r = min(row[u], a.n - 1);
      code[u] = *reinterpret_cast<const Pack<u32, E / 4>*>(a.codes + r * a.steps * OCT_STEP + c[u] * E);
      scale[u] = mx_scale(a.scales[r * words * 4 + c[u] * E / OCT_STEP]);
    }
#pragma unroll
    for (u32 u = 0; u < AHEAD; ++u) {
      if (row[u] >= a.n) break;
      AnyPack<T, E> o;
#pragma unroll
      for (u32 q = 0; q < E / 4; ++q) {
        const v2f low = __builtin_amdgcn_cvt_pk_f32_fp8((int)code[u].v[q], false), high = __builtin_amdgcn_cvt_pk_f32_fp8((int)code[u].v[q], true);
        o.v[4 * q] = mx_round<T>(low.x * scale[u]);
        o.v[4 * q + 1] = mx_round<T>(low.y * scale[u]);
        o.v[4 * q + 2] = mx_round<T>(high.x * scale[u]);
        o.v[4 * q + 3] = mx_round<T>(high.y * scale[u]);
      }
      T* to = reinterpret_cast<T*>(a.out) + row[u] * a.ldo + c[u] * E;
      if (c[u] * E + E <= a.d) {
        __builtin_nontemporal_store(__builtin_bit_cast(v4i, o), reinterpret_cast<Streamed*>(to));
      } else {
#pragma unroll
        for (u32 k = 0; k < E; ++k)
          if (c[u] * E + k < a.d) to[k] = o.v[k];
      }
    }
  }
}

template <typename T>
hipError_t launch_oct_dequantize(const OctDequantizeArgs& a, hipStream_t s) {
  const u32 pieces = (u32)((a.d + 16 / sizeof(T) - 1) / (16 / sizeof(T)));
  const u64 items = a.n * pieces, blocks = (items + DEQUANTIZE_TILE - 1) / DEQUANTIZE_TILE;
  hipLaunchKernelGGL(oct_dequantize_kernel<T>, dim3((u32)std::min<u64>(blocks, 1u << 23)), dim3(256), 0, s, a, pieces, items);
  return hipGetLastError();
}

}  // namespace annmi

using namespace annmi;

extern "C" {

int ann_oct_quantize(const void* x_dev, uint64_t n, uint32_t d, ann_dtype dtype, uint64_t ldx, int columns, uint8_t* codes_dev,
                    uint8_t* scales_dev, void* stream) try {
  const u64 esz = dtype_bytes(dtype);
  if (esz == 0) return fail(ANN_EINVAL, "unknown dtype");
  int rc = check_oct_rows("ann_oct_quantize", codes_dev, scales_dev, n, d);
  if (rc) return rc;
  if (ldx < (columns ? n : d)) return fail(ANN_EINVAL, columns ? "ldx must be at least n" : "ldx must be at least d");
  if (n == 0) return ANN_OK;
  if (!x_dev) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(x_dev, esz)) return fail(ANN_EINVAL, "x not aligned to its elements");
  OctQuantizeArgs a{static_cast<const char*>(x_dev), ldx, (u32)n, d, oct_steps(d), codes_dev, reinterpret_cast<u32*>(scales_dev)};
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (dtype) {
    case ANN_U8: HIP_TRY(launch_oct_quantize<uint8_t>(a, columns, st)); break;
    case ANN_I8: HIP_TRY(launch_oct_quantize<int8_t>(a, columns, st)); break;
    case ANN_F16: HIP_TRY(launch_oct_quantize<__half>(a, columns, st)); break;
    case ANN_BF16: HIP_TRY(launch_oct_quantize<__bf16>(a, columns, st)); break;
    default: HIP_TRY(launch_oct_quantize<float>(a, columns, st)); break;
  }
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

int ann_oct_dequantize(const uint8_t* codes_dev, const uint8_t* scales_dev, uint64_t n, uint32_t d, void* out_dev,
                      ann_dtype dtype, uint64_t ldo, void* stream) try {
  const u64 esz = dtype_bytes(dtype);
  if (esz < 2) return fail(ANN_EINVAL, "the values come as ANN_F32, ANN_F16 or ANN_BF16");
  int rc = check_oct_rows("ann_oct_dequantize", codes_dev, scales_dev, n, d);
  if (rc) return rc;
  if (ldo < d) return fail(ANN_EINVAL, "ldo must be at least d");
  if (n == 0) return ANN_OK;
  if (!out_dev) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(out_dev, esz)) return fail(ANN_EINVAL, "out not aligned to its elements");
  OctDequantizeArgs a{codes_dev, scales_dev, n, oct_steps(d), d, static_cast<char*>(out_dev), ldo};
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (dtype) {
    case ANN_F16: HIP_TRY(launch_oct_dequantize<__half>(a, st)); break;
    case ANN_BF16: HIP_TRY(launch_oct_dequantize<__bf16>(a, st)); break;
    default: HIP_TRY(launch_oct_dequantize<float>(a, st)); break;
  }
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

}  // extern "C"
