// Products of a batch with microscaled 4-bit rows.
#include "mx.hpp"

namespace annmi {

struct ProductArgs {
  MxRows w;  // the 4-bit rows
  MxRows q;  // the batch, where it is 4-bit rows too
  const char* x;  // the batch otherwise
  u64 ldx;
  u32 nx, d;
  char* out;
  u64 ldo;
  u32 wide;  // four results can be written at once
};

// The 64 x 64 results of a wave: rows of `w` in the matrix instruction's rows, so that a lane holds four results
// that follow each other in `out`.
template <typename OUT>
__device__ __forceinline__ void store_results(const ProductArgs& a, const v4f (&acc)[4][4], u64 w0, u64 x0) {
  const u32 lane = threadIdx.x % 64;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const u64 x = x0 + 16 * j + lane % 16;
    if (x >= a.nx) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u64 w = w0 + 16 * i + lane / 16 * 4;
      OUT* to = reinterpret_cast<OUT*>(a.out) + x * a.ldo + w;
      if (a.wide && w + 4 <= a.w.n) {
        Pack<OUT, 4> p;
#pragma unroll
        for (int r = 0; r < 4; ++r) p.v[r] = mx_round<OUT>(acc[i][j][r]);
        *reinterpret_cast<Pack<OUT, 4>*>(to) = p;
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (w + r < a.w.n) to[r] = mx_round<OUT>(acc[i][j][r]);
      }
    }
  }
}

struct Fragment {  // 16 rows x 128 elements of 4 bits, a lane's share
  v4i codes;
  int scale;
};
// rows past the last are read as the last one: their results go nowhere
__device__ __forceinline__ Fragment load_fragment(const MxRows& m, u64 row0, u32 step) {
  const u32 lane = threadIdx.x % 64;
  const u64 row = min(row0 + lane % 16, (u64)m.n - 1);
  Fragment f;
  f.codes = *reinterpret_cast<const v4i*>(m.codes + (row * m.steps + step) * MX_STEP_BYTES + lane / 16 * 16);
  f.scale = m.scales[(row * m.steps + step) * MX_STEP_SCALES + lane / 16];
  return f;
}

// 128 x 128 results a workgroup, 64 x 64 a wave; both sides from memory, step by step.
template <typename OUT>
__global__ __launch_bounds__(256) void mx_product4_kernel(ProductArgs a, u32 tiles_w, u64 tiles) {
  const u32 wave = threadIdx.x / 64;
  for (u64 t = blockIdx.x; t < tiles; t += gridDim.x) {
    const u64 w0 = t % tiles_w * 128 + (wave & 1) * 64, x0 = t / tiles_w * 128 + (wave >> 1) * 64;
    if (w0 >= a.w.n || x0 >= a.nx) continue;
    v4f acc[4][4] = {};
    for (u32 s = 0; s < a.w.steps; ++s) {
      Fragment w[4], x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = load_fragment(a.w, w0 + 16 * i, s);
        x[i] = load_fragment(a.q, x0 + 16 * i, s);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = mx_mfma(w[i].codes, x[j].codes, acc[i][j], w[i].scale, x[j].scale);
    }
    store_results<OUT>(a, acc, w0, x0);
  }
}

// A float as bf16 numbers whose sum it is: the upper halves of what is left, without rounding, so that none
// leaves the range.  Infinities and NaN stay in the first.
template <int PARTS>
__device__ __forceinline__ void split(float v, __bf16 (&part)[PARTS]) {
  if (PARTS == 1) {
    part[0] = static_cast<__bf16>(v);
    return;
  }
  const u32 b = __float_as_uint(v);
  const bool fine = (b & 0x7F800000u) != 0x7F800000u;
#pragma unroll
  for (int i = 0; i < PARTS; ++i) {
    u32 top = __float_as_uint(v) & 0xFFFF0000u;
    if (i == 0 && v != v) top = 0x7FC00000u;
    part[i] = __builtin_bit_cast(__bf16, (unsigned short)(top >> 16));
    v = fine ? v - __uint_as_float(top) : 0.0f;
  }
}
template <typename T>
constexpr int parts_of() {
  return sizeof(T) == 4 ? 3 : __is_same(T, __half) ? 2 : 1;
}

// 4-bit rows against rows of 16 or 32 bits: codes become bf16 numbers times their scale, exactly; the batch is the
// sum of one, two or three bf16 numbers.  Within a step the elements are taken in the order that a lane holds
// them: 8 at a time of the lane's 32, the same ones on both sides.
template <typename T, typename OUT>
__global__ __launch_bounds__(256) void mx_product16_kernel(ProductArgs a, u32 tiles_w, u64 tiles) {
  constexpr int PARTS = parts_of<T>();
  const u32 wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  for (u64 t = blockIdx.x; t < tiles; t += gridDim.x) {
    const u64 w0 = t % tiles_w * 128 + (wave & 1) * 64, x0 = t / tiles_w * 128 + (wave >> 1) * 64;
    if (w0 >= a.w.n || x0 >= a.nx) continue;
    v4f acc[4][4] = {};
    for (u32 s = 0; s < a.w.steps; ++s) {
      Fragment w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = load_fragment(a.w, w0 + 16 * i, s);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        v8bf wv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float scale = mx_scale((u32)w[i].scale);
          const v2bf p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((u32)w[i].codes[c], scale, 0),
                             __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((u32)w[i].codes[c], scale, 1),
                             __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((u32)w[i].codes[c], scale, 2),
                             __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((u32)w[i].codes[c], scale, 3)};
          wv[i] = v8bf{p[0].x, p[0].y, p[1].x, p[1].y, p[2].x, p[2].y, p[3].x, p[3].y};
        }
        const u32 at = s * MX_STEP + lane / 16 * 32 + c * 8;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u64 row = min(x0 + 16 * j + lane % 16, (u64)a.nx - 1);
          const T* from = reinterpret_cast<const T*>(a.x) + row * a.ldx + at;
          v8bf xv[PARTS];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            __bf16 part[PARTS];
            split<PARTS>(at + e < a.d ? mx_float(from[e]) : 0.0f, part);
#pragma unroll
            for (int p = 0; p < PARTS; ++p) xv[p][e] = part[p];
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[i], xv[p], acc[i][j], 0, 0, 0);
        }
      }
    }
    store_results<OUT>(a, acc, w0, x0);
  }
}

template <typename OUT>
hipError_t launch_product(const ProductArgs& a, int xdtype, hipStream_t s) {
  const u32 tiles_w = (u32)(((u64)a.w.n + 127) / 128);
  const u64 tiles = tiles_w * (((u64)a.nx + 127) / 128);
  const dim3 grid((u32)(tiles < (1u << 20) ? tiles : (1u << 20)));
  if (xdtype < 0)
    hipLaunchKernelGGL(mx_product4_kernel<OUT>, grid, dim3(256), 0, s, a, tiles_w, tiles);
  else if (xdtype == ANN_F32)
    hipLaunchKernelGGL((mx_product16_kernel<float, OUT>), grid, dim3(256), 0, s, a, tiles_w, tiles);
  else if (xdtype == ANN_F16)
    hipLaunchKernelGGL((mx_product16_kernel<__half, OUT>), grid, dim3(256), 0, s, a, tiles_w, tiles);
  else
    hipLaunchKernelGGL((mx_product16_kernel<__bf16, OUT>), grid, dim3(256), 0, s, a, tiles_w, tiles);
  return hipGetLastError();
}

// xdtype < 0: the batch is 4-bit rows
int product(ProductArgs a, int xdtype, u64 nx, u64 n, void* out, int odtype, u64 ldo, void* stream) {
  const u64 osz = dtype_bytes(odtype);
  if (osz < 2) return fail(ANN_EINVAL, "out must be ANN_F32, ANN_F16 or ANN_BF16");
  if (ldo < n) return fail(ANN_EINVAL, "ldo must be at least n");
  if (nx == 0 || n == 0) return ANN_OK;
  if (!out) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(out, osz)) return fail(ANN_EINVAL, "out not aligned to its elements");
  a.w.n = (u32)n;
  a.nx = (u32)nx;
  a.out = static_cast<char*>(out);
  a.ldo = ldo;
  a.wide = aligned_to(out, 4 * osz) && ldo % 4 == 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (odtype) {
    case ANN_F16: HIP_TRY(launch_product<__half>(a, xdtype, st)); break;
    case ANN_BF16: HIP_TRY(launch_product<__bf16>(a, xdtype, st)); break;
    default: HIP_TRY(launch_product<float>(a, xdtype, st)); break;
  }
  return ANN_OK;
}

}  // namespace annmi

using namespace annmi;

extern "C" {

int ann_mx_product(const void* x_dev, uint64_t nx, ann_dtype xdtype, uint64_t ldx, const uint8_t* codes_dev,
                   const uint8_t* scales_dev, uint64_t n, uint32_t d, void* out_dev, ann_dtype out_dtype, uint64_t ldo,
                   void* stream) try {
  const u64 esz = dtype_bytes(xdtype);
  if (esz < 2) return fail(ANN_EINVAL, "x must be ANN_F32, ANN_F16 or ANN_BF16 (bytes: ann_mx_quantize, ann_mx_product_mx)");
  int rc = check_mx_rows("ann_mx_product", codes_dev, scales_dev, n, d);
  if (rc) return rc;
  if (nx > MX_MOST_ROWS) return fail(ANN_EINVAL, "nx must stay below 2^31");
  if (ldx < d) return fail(ANN_EINVAL, "ldx must be at least d");
  if (nx && n && !x_dev) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(x_dev, esz)) return fail(ANN_EINVAL, "x not aligned to its elements");
  ProductArgs a{};
  a.w = {codes_dev, scales_dev, 0, mx_steps(d)};
  a.x = static_cast<const char*>(x_dev);
  a.ldx = ldx;
  a.d = d;
  return product(a, xdtype, nx, n, out_dev, out_dtype, ldo, stream);
} catch (...) {
  return annmi::on_exception();
}

int ann_mx_product_mx(const uint8_t* xcodes_dev, const uint8_t* xscales_dev, uint64_t nx, const uint8_t* codes_dev,
                      const uint8_t* scales_dev, uint64_t n, uint32_t d, void* out_dev, ann_dtype out_dtype, uint64_t ldo,
                      void* stream) try {
  int rc = check_mx_rows("ann_mx_product_mx", codes_dev, scales_dev, n, d);
  if (rc) return rc;
  rc = check_mx_rows("ann_mx_product_mx", xcodes_dev, xscales_dev, nx, d);
  if (rc) return rc;
  ProductArgs a{};
  a.w = {codes_dev, scales_dev, 0, mx_steps(d)};
  a.q = {xcodes_dev, xscales_dev, (u32)nx, mx_steps(d)};
  a.d = d;
  return product(a, -1, nx, n, out_dev, out_dtype, ldo, stream);
} catch (...) {
  return annmi::on_exception();
}

}  // extern "C"
