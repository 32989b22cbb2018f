// Products of a batch with microscaled 4-bit rows.
#include <type_traits>
#include <utility>

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
  int odtype;
  u32 wide;  // four results can be written at once
  u32 wide_x;  // the batch's rows have eight elements and more
};

constexpr size_t FEW_LDS = 160 * 1024;    // of a compute unit
// Most of it that a batch may take: the rest is room for eight waves' sums.  By 131,072 rows of bf16, in LDS and by the
// tiles of mx_product_many_kernel: 16 x 2,900 45 us and 81, 32 x 1,400 29 and 39, 48 x 900 32 and 32, 64 x 600 30 and 24;
// 33 x 200 fp32 by 500,001 45 and 59, 64 x 200 bf16 48 and 44.  (More than 48 rows would be served better by the tiles.)
constexpr size_t FEW_BATCH = 96 * 1024;
constexpr u32 LONG_STEPS = 8;             // rows of so many steps are summed in runs
constexpr size_t few_batch(u32 nx, u32 steps, int parts) { return (size_t)nx * (steps * MX_STEP * 2 + 16) * parts; }
static_assert(few_batch(64, 1, 3) <= FEW_BATCH);  // so that 64 rows shorter than a step always fit

// The 16 WF x 16 XF results of a wave.  They lie in the matrix instruction's order (a lane holds four neighbours of a
// row of `out`); through LDS of the wave's own they get into runs of a whole row's part, so that stores fill lines
// wherever a row of `out` begins.
template <int WF>
constexpr u32 store_room() {
  return 16 * (16 * WF + 4) * 4;  // bytes of LDS for a wave: the four floats more keep rows in different banks
}
template <typename OUT, int WF, int XF>
__device__ __forceinline__ void store_as(const ProductArgs& a, const v4f (&acc)[WF][XF], u64 w0, u64 x0, float* room) {
  constexpr u32 ROW = 16 * WF, STRIDE = ROW + 4;
  const u32 lane = threadIdx.x % 64;
#pragma unroll
  for (int j = 0; j < XF; ++j) {
    if (x0 + 16 * j >= a.nx) break;
    wave_exchange();
#pragma unroll
    for (int i = 0; i < WF; ++i) *reinterpret_cast<v4f*>(room + lane % 16 * STRIDE + 16 * i + lane / 16 * 4) = acc[i][j];
    wave_exchange();
    OUT* out = reinterpret_cast<OUT*>(a.out) + (x0 + 16 * j) * a.ldo + w0;
    const u32 xs = (u32)min((u64)16, a.nx - (x0 + 16 * j)), ws = (u32)min((u64)ROW, a.w.n - w0);
    if (a.wide && ws == ROW) {
#pragma unroll
      for (u32 k = 0; k < 16 * ROW / 256; ++k) {
        const u32 r = (k * 256 + lane * 4) / ROW, at = (k * 256 + lane * 4) % ROW;
        const v4f v = *reinterpret_cast<const v4f*>(room + r * STRIDE + at);
        Pack<OUT, 4> p;
#pragma unroll
        for (int e = 0; e < 4; ++e) p.v[e] = mx_round<OUT>(v[e]);
        if (r < xs) *reinterpret_cast<Pack<OUT, 4>*>(out + r * a.ldo + at) = p;
      }
    } else {
#pragma unroll 4
      for (u32 k = 0; k < 16 * ROW / 64; ++k) {
        const u32 r = (k * 64 + lane) / ROW, at = (k * 64 + lane) % ROW;
        const float v = room[r * STRIDE + at];
        if (r < xs && at < ws) out[r * a.ldo + at] = mx_round<OUT>(v);
      }
    }
  }
}
template <int WF, int XF>
__device__ __forceinline__ void store_results(const ProductArgs& a, const v4f (&acc)[WF][XF], u64 w0, u64 x0, char* room) {
  if (a.odtype == ANN_F32)
    store_as<float, WF, XF>(a, acc, w0, x0, reinterpret_cast<float*>(room));
  else if (a.odtype == ANN_F16)
    store_as<__half, WF, XF>(a, acc, w0, x0, reinterpret_cast<float*>(room));
  else
    store_as<__bf16, WF, XF>(a, acc, w0, x0, reinterpret_cast<float*>(room));
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

// 128 x 128 results a workgroup, 64 x 64 a wave; both sides from memory, step by step.  For products whose results are
// most of what moves: 1,000 x 10,000 of 128 elements to fp32 take 13 us, 3.2 TB/s.
__global__ __launch_bounds__(256) void mx_product4_kernel(ProductArgs a, u32 tiles_w, u64 tiles) {
  __shared__ __align__(16) char room[4 * store_room<4>()];
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
    store_results<4, 4>(a, acc, w0, x0, room + wave * store_room<4>());
  }
}

// 4-bit rows on both sides, many: 256 x 256 results a workgroup of eight waves, 128 x 64 a wave.  Pairs of steps (256
// elements) pass through LDS, two at a time: while one is multiplied the next waits in registers for its turn.  The
// scales lie in LDS so that a lane reads those of all its fragments' rows at once; the instruction picks the byte.
// 4,096 x 65,536 of 2,048 elements take 440 us, 2.5 PFLOP/s (490 us once the clock has fallen under a load that lasts):
// the matrix cores work 28 % of that time, and the waves wait for loads, one pair of steps ahead, for which LDS and
// registers have room.  Workgroups that stay for several tiles, with the next one's first pairs asked for before the
// results leave, are no faster (474 to 480 us in the place of 469).
constexpr u32 BOTH_THREADS = 512;
constexpr u32 BOTH_ROWS = 256;  // of either side

template <int... I, typename F>
__device__ __forceinline__ void unroll(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unroll(F f) {
  unroll(std::make_integer_sequence<int, N>(), f);
}
template <int BYTE_A, int BYTE_B>
__device__ __forceinline__ v4f mx_mfma_bytes(v4i a, v4i b, v4f c, int scales_a, int scales_b) {
  const v8i x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, BYTE_A, scales_a, BYTE_B, scales_b);
}

__global__ __launch_bounds__(BOTH_THREADS) void mx_product4_many_kernel(ProductArgs a, u32 tiles_w, u32 tiles) {
  constexpr u32 BYTES = BOTH_ROWS * 128;                // codes of one side of a stage
  constexpr u32 STAGE = 2 * BYTES + 2 * BOTH_ROWS * 8;  // and the scales of both
  extern __shared__ __align__(16) char lds[];
  const u32 tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  // Chiplets take workgroups in turn: each gets a run of tiles that share rows.
  const u32 per = (tiles + 7) / 8, t = blockIdx.x % 8 * per + blockIdx.x / 8;
  if (t >= tiles) return;
  const u32 tiles_x = tiles / tiles_w;
  const u64 w0 = (u64)(t / tiles_x) * BOTH_ROWS, x0 = (u64)(t % tiles_x) * BOTH_ROWS;
  const u32 ww = wave % 2 * 128, wx = wave / 2 * 64;  // the wave's part of the tile
  const u32 steps = a.w.steps, pairs = (steps + 1) / 2;

  // What this thread brings to LDS: 16 bytes of the pair's 128 of four rows of each side, and the scales of one step
  // of a row.  A step past the last is read as the one before, and the 4-bit rows' codes of it count as 0.
  const u32 unit = tid % 8;
  const uint8_t* side_codes[2] = {a.w.codes + w0 * steps * MX_STEP_BYTES, a.q.codes + x0 * steps * MX_STEP_BYTES};
  const u32* side_scales[2] = {reinterpret_cast<const u32*>(a.w.scales) + w0 * steps, reinterpret_cast<const u32*>(a.q.scales) + x0 * steps};
  const u32 last_row[2] = {(u32)min((u64)BOTH_ROWS, a.w.n - w0) - 1, (u32)min((u64)BOTH_ROWS, a.q.n - x0) - 1};
  u32 offset[2][4], scale_at[2];
#pragma unroll
  for (u32 side = 0; side < 2; ++side) {
#pragma unroll
    for (u32 i = 0; i < 4; ++i) offset[side][i] = min(tid / 8 + 64 * i, last_row[side]) * steps * MX_STEP_BYTES + unit % 4 * 16;
    scale_at[side] = min(tid / 2, last_row[side]) * steps;
  }
  v4i next[2][4];
  u32 next_scale[2];
  bool there;
  auto fetch = [&](u32 p) {
    there = p * 2 + unit / 4 < steps;
    const u32 second = there ? unit / 4 * MX_STEP_BYTES : 0, scale = min(p * 2 + tid % 2, steps - 1);
#pragma unroll
    for (u32 side = 0; side < 2; ++side) {
      const uint8_t* from = side_codes[side] + p * (2 * MX_STEP_BYTES);
#pragma unroll
      for (u32 i = 0; i < 4; ++i) next[side][i] = *reinterpret_cast<const v4i*>(from + (offset[side][i] + second));
      next_scale[side] = side_scales[side][scale_at[side] + scale];
    }
  };
  auto keep = [&](u32 p) {
    char* stage = lds + p % 2 * STAGE;
#pragma unroll
    for (u32 side = 0; side < 2; ++side) {
#pragma unroll
      for (u32 i = 0; i < 4; ++i) {
        const u32 r = tid / 8 + 64 * i;
        *reinterpret_cast<v4i*>(stage + side * BYTES + r * 128 + (unit ^ r % 8) * 16) = side || there ? next[side][i] : v4i{};
      }
      // (step, block, row % 16, row / 16): a lane's fragments are 16 rows apart
      const u32 row = tid / 2;
      char* scales = stage + 2 * BYTES + side * BOTH_ROWS * 8 + (tid % 2 * 64 + row % 16) * 16 + row / 16;
#pragma unroll
      for (u32 g = 0; g < 4; ++g) scales[g * 256] = (char)(next_scale[side] >> (8 * g));
    }
  };
  v4f acc[8][4] = {};
  fetch(0);
  keep(0);
  fetch(min(1u, pairs - 1));
  for (u32 p = 0; p < pairs; ++p) {
    __syncthreads();
    const char* stage = lds + p % 2 * STAGE;
#pragma unroll
    for (u32 h = 0; h < 2; ++h) {
      __builtin_amdgcn_sched_barrier(0);  // (or both steps' fragments would be read at once, in too many registers)
      if (h == 1) {
        // Behind the first products: they run while the next pair is put away.  At the end a pair too many is, and
        // not read: at a condition the compiler would move the products behind it.
        keep(p + 1);
        fetch(min(p + 2, pairs - 1));
        __builtin_amdgcn_sched_barrier(0);
      }
      const char* scales = stage + 2 * BYTES + (h * 64 + lane) * 16;
      using v2i = int __attribute__((ext_vector_type(2)));
      const v2i ws = *reinterpret_cast<const v2i*>(scales + ww / 16);
      const int xs = *reinterpret_cast<const int*>(scales + BOTH_ROWS * 8 + wx / 16);
      const u32 at = ((h * 4 + lane / 16) ^ lane % 8) * 16 + lane % 16 * 128;
      v4i x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const v4i*>(stage + BYTES + (wx + 16 * j) * 128 + at);
      unroll<8>([&](auto i) {
        const v4i w = *reinterpret_cast<const v4i*>(stage + (ww + 16 * i) * 128 + at);
        unroll<4>([&](auto j) { acc[i][j] = mx_mfma_bytes<i % 4, j>(w, x[j], acc[i][j], ws[i / 4], xs); });
      });
    }
  }
  __syncthreads();
  if (w0 + ww < a.w.n) store_results<8, 4>(a, acc, w0 + ww, x0 + wx, lds + wave * store_room<8>());
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

// Eight elements of a row of the batch from `at` on; rows past the last are read as it.  WIDE, for rows of eight
// elements and more: in one load wherever they begin, and the row's last eight where they would reach past its end.
// `mask_batch` then brings these to their place and puts zeros behind them, later, so that no branch waits for a load.
// (Rows that begin at any element against rows at multiples of 16 bytes: 98 us and 94 for 1,000 of 200 by 100,000,
// where eight loads of an element each took 166.)
template <typename T, bool WIDE>
__device__ __forceinline__ Pack<T, 8> load_batch(const ProductArgs& a, u64 row, u32 at) {
  const T* from = reinterpret_cast<const T*>(a.x) + min(row, (u64)a.nx - 1) * a.ldx;
  using Whole = Pack<T, 8>;
  if (WIDE) return __builtin_bit_cast(Whole, *reinterpret_cast<const AnyPack<T, 8>*>(from + min(at, a.d - 8)));
  Pack<T, 8> p;
#pragma unroll
  for (int e = 0; e < 8; ++e) p.v[e] = from[min(at + e, a.d - 1)];
  return p;
}
template <typename T, bool WIDE>
__device__ __forceinline__ void mask_batch(const ProductArgs& a, Pack<T, 8>& p, u32 at) {
  if (WIDE) {
    constexpr u32 WORDS = 2 * sizeof(T);
    using Words = Pack<u32, WORDS>;
    // Elements to leave out at the front.  (Written with unsigned numbers, at + 8 > d ? min(at + 8 - d, 8) : 0, the
    // compiler made it 8 for some constant parts of `at`.)
    const u32 past = min(max((int)(at + 8 - a.d), 0), 8);
    Words w = __builtin_bit_cast(Words, p);
#pragma unroll
    for (u32 by = 8; by * sizeof(T) >= 4; by /= 2) {
      const u32 words = by * sizeof(T) / 4;
#pragma unroll
      for (u32 i = 0; i < WORDS; ++i) w.v[i] = past & by ? (i + words < WORDS ? w.v[i + words] : 0u) : w.v[i];
    }
    if (sizeof(T) == 2) {
#pragma unroll
      for (u32 i = 0; i < WORDS; ++i) w.v[i] = __builtin_amdgcn_alignbit(i + 1 < WORDS ? w.v[i + 1] : 0u, w.v[i], past % 2 * 16);
    }
    using Whole = Pack<T, 8>;
    p = __builtin_bit_cast(Whole, w);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (at + e >= a.d) p.v[e] = T(0.0f);
}
template <typename T, int PARTS>
__device__ __forceinline__ void split_pack(const Pack<T, 8>& p, v8bf (&out)[PARTS]) {
  if constexpr (PARTS == 1) {
    out[0] = __builtin_bit_cast(v8bf, p);
    return;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      __bf16 part[PARTS];
      split<PARTS>(mx_float(p.v[e]), part);
#pragma unroll
      for (int i = 0; i < PARTS; ++i) out[i][e] = part[i];
    }
  }
}

// Eight codes as bf16 numbers times their scale, exactly.  The conversion reads the exponent bits of its scale
// alone, so that a scale byte needs no care at its ends: 0 is 2^-127 and 255 is NaN.
__device__ __forceinline__ v8bf unpack(u32 codes, u32 scale_byte) {
  const float scale = __uint_as_float(scale_byte << 23);
  const v2bf p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1),
                     __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3)};
  return v8bf{p[0].x, p[0].y, p[1].x, p[1].y, p[2].x, p[2].y, p[3].x, p[3].y};
}

// Few rows of 16 or 32 bits against all 4-bit rows: the batch stays in LDS, as one, two or three bf16 numbers for
// each element, and the 4-bit rows stream past it, each byte read once.  A wave takes 16 WF of them and always has
// the next AHEAD steps on their way while it multiplies the present ones.  Long rows (LONG) are summed in runs of
// groups of AHEAD steps, which are added up in their order, by one wave or, where 4-bit rows are few, by a wave
// each: the sums do not depend on that.  Within a step the elements are taken in the order that a lane holds
// them (8 at a time of its 32, the same ones on both sides).  One row of 4,096 bf16 by 131,072 is bound by memory: 53 to
// 56 us, 5.1 to 5.4 TB/s.  33 rows of 200 floats by 500,001 take 47 us: three bf16 numbers for each element, the matrix cores at work
// 41 % of the time, 2.8 TB/s.
constexpr u32 FEW_THREADS = 512;

template <int G, int WF>
constexpr u32 few_room(u32 share) {  // bytes of LDS of a wave's own
  return share > 1 && WF * G * 1024 > store_room<WF>() ? WF * G * 1024 : store_room<WF>();
}

template <typename T, int G, int WF, int AHEAD, bool LONG>
__global__ __launch_bounds__(FEW_THREADS) void mx_product_few_kernel(ProductArgs a, u32 tiles, u32 runs, u32 share) {
  constexpr int PARTS = parts_of<T>();
  const u32 room_bytes = few_room<G, WF>(share);
  extern __shared__ __align__(16) char lds[];
  const u32 lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  // 16 bytes more for each row than its elements take: the rows' pieces then lie in different banks
  const u32 row_bytes = a.w.steps * MX_STEP * 2 + 16, part_bytes = a.nx * row_bytes;
  const u32 pieces = a.w.steps * 16;
  for (u32 i = threadIdx.x; i < a.nx * pieces; i += FEW_THREADS) {
    const u32 row = i / pieces, at = i % pieces;
    const bool wide = LONG || a.wide_x;
    Pack<T, 8> piece = wide ? load_batch<T, true>(a, row, at * 8) : load_batch<T, false>(a, row, at * 8);
    if (wide)
      mask_batch<T, true>(a, piece, at * 8);
    else
      mask_batch<T, false>(a, piece, at * 8);
    v8bf x[PARTS];
    split_pack<T, PARTS>(piece, x);
#pragma unroll
    for (int p = 0; p < PARTS; ++p) *reinterpret_cast<v8bf*>(lds + p * part_bytes + row * row_bytes + at * 16) = x[p];
  }
  __syncthreads();
  char* room = lds + PARTS * part_bytes + wave * room_bytes;
  const u32 teams = FEW_THREADS / 64 / share;  // of waves that share rows
  const u32 first_run = LONG ? wave % share * (runs / share) : 0, last_run = LONG ? first_run + runs / share : 1;
  const u32 groups = (a.w.steps + AHEAD - 1) / AHEAD;
  const u32 g_first = LONG ? groups * first_run / runs : 0, g_last = LONG ? groups * last_run / runs : groups;
  const char* xs[G];
#pragma unroll
  for (int j = 0; j < G; ++j) xs[j] = lds + min(16u * j + lane % 16, a.nx - 1) * row_bytes + lane / 16 * 64;

  struct Ahead {
    v4i w[AHEAD][WF];
    u32 b[WF][AHEAD];
  } next;
  auto ask = [&](u32 tile, u32 group) {
    const u32 s0 = group * AHEAD;
#pragma unroll
    for (int i = 0; i < WF; ++i) {
      const u64 row = min((u64)tile * (16 * WF) + 16 * i + lane % 16, (u64)a.w.n - 1) * a.w.steps;
      const u32* scales = reinterpret_cast<const u32*>(a.w.scales) + row;
      const uint8_t* codes = a.w.codes + row * MX_STEP_BYTES + lane / 16 * 16;
      if (LONG) {  // one load for the group; the last one may begin before s0
        const u32 from = min(s0, a.w.steps - AHEAD), skip = s0 - from;
        using Scales = u32 __attribute__((ext_vector_type(AHEAD), aligned(4)));
        const Scales some = *reinterpret_cast<const Scales*>(scales + from);
#pragma unroll
        for (u32 u = 0; u < AHEAD; ++u) {
          next.b[i][u] = some[u];
#pragma unroll
          for (u32 k = 1; k + u < AHEAD; ++k)
            if (skip == k) next.b[i][u] = some[u + k];
        }
      } else {
#pragma unroll
        for (u32 u = 0; u < AHEAD; ++u) next.b[i][u] = scales[min(s0 + u, a.w.steps - 1)];
      }
#pragma unroll
      for (u32 u = 0; u < AHEAD; ++u) next.w[u][i] = *reinterpret_cast<const v4i*>(codes + (u64)min(s0 + u, a.w.steps - 1) * MX_STEP_BYTES);
    }
  };
  u32 t = blockIdx.x * teams + wave / share;
  const u32 stride = gridDim.x * teams;
  if (t < tiles) ask(t, g_first);
  for (; t - wave / share < tiles; t += stride) {  // (all waves of a workgroup alike: they may have to meet)
    v4f sum[WF][G] = {};
    if (t < tiles) {
      v4f acc[WF][G] = {};
      u32 run = first_run, g_run = LONG ? groups * (run + 1) / runs : groups;
      for (u32 g = g_first; g < g_last; ++g) {
        const Ahead now = next;
        const bool more = g + 1 < g_last;  // of this tile
        ask(more ? t : min(t + stride, tiles - 1), more ? g + 1 : g_first);
#pragma unroll
        for (u32 u = 0; u < AHEAD; ++u) {
          const u32 s = g * AHEAD + u;
          if (s >= a.w.steps) break;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            // (or all the batch's pieces of a step would be read at once, into more registers than there are)
            __builtin_amdgcn_sched_barrier(0);
            v8bf wv[WF];
#pragma unroll
            for (int i = 0; i < WF; ++i) wv[i] = unpack((u32)now.w[u][i][c], now.b[i][u] >> (lane / 16 * 8) & 255);
#pragma unroll
            for (int j = 0; j < G; ++j)
#pragma unroll
              for (int p = PARTS - 1; p >= 0; --p) {
                const v8bf x = *reinterpret_cast<const v8bf*>(xs[j] + p * part_bytes + s * (MX_STEP * 2) + c * 16);
#pragma unroll
                for (int i = 0; i < WF; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[i], x, acc[i][j], 0, 0, 0);
              }
          }
        }
        if (LONG && g + 1 == g_run) {
#pragma unroll
          for (int i = 0; i < WF; ++i)
#pragma unroll
            for (int j = 0; j < G; ++j) sum[i][j] += acc[i][j], acc[i][j] = v4f{};
          ++run;
          g_run = groups * (run + 1) / runs;
        }
      }
      if (!LONG)
#pragma unroll
        for (int i = 0; i < WF; ++i)
#pragma unroll
          for (int j = 0; j < G; ++j) sum[i][j] = acc[i][j];
    }
    if (LONG && share > 1) {  // (a run each) they meet in the team's first wave
      char* mine = room + lane * 16;
      if (wave % share)
#pragma unroll
        for (int i = 0; i < WF * G; ++i) *reinterpret_cast<v4f*>(mine + i * 1024) = sum[i / G][i % G];
      __syncthreads();
      if (wave % share == 0)
        for (u32 o = 1; o < share; ++o)
#pragma unroll
          for (int i = 0; i < WF * G; ++i) sum[i / G][i % G] += *reinterpret_cast<const v4f*>(mine + o * room_bytes + i * 1024);
      __syncthreads();
    }
    if (t < tiles && wave % share == 0) store_results<WF, G>(a, sum, (u64)t * (16 * WF), 0, room);
  }
}

// Many rows: 256 4-bit rows x 64 XF rows of the batch a workgroup of eight waves, 128 x 16 XF a wave.  Halves of a
// step (64 elements) pass through LDS, two at a time: while one is multiplied the next waits in registers for
// its turn and the one after is on its way.  The codes become bf16 numbers on their way from LDS to the matrix
// cores, four conversions for each fragment of 16 rows x 32 elements, which serves XF x PARTS products.
// 2,048 x 16,384 of 4,096 bf16 take 240 us as a call among others, 1.15 PFLOP/s, and 261 to 289 under a load that lasts, when
// the clock falls; the library's product of bf16 on both sides takes 219 to 229.  The matrix cores work 53 % of the time.
// fp16, two products for each element, takes 484 us, fp32, three, 645.
constexpr u32 MANY_THREADS = 512;
constexpr u32 MANY_ROWS = 256;

template <typename T, int XF, bool WIDE>
__global__ __launch_bounds__(MANY_THREADS, XF == 1 ? 4 : 2) void mx_product_many_kernel(ProductArgs a, u32 tiles_w, u32 tiles) {
  constexpr int PARTS = parts_of<T>();
  constexpr u32 X_ROWS = 64 * XF;
  constexpr u32 W_BYTES = MANY_ROWS * 32, X_BYTES = X_ROWS * 128, STAGE = W_BYTES + PARTS * X_BYTES;
  extern __shared__ __align__(16) char lds[];  // two stages, then the scales of two steps
  const u32 tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  // Chiplets take workgroups in turn: each gets a run of tiles that share rows.
  const u32 per = (tiles + 7) / 8, t = blockIdx.x % 8 * per + blockIdx.x / 8;
  if (t >= tiles) return;
  const u32 tiles_x = tiles / tiles_w;
  const u64 w0 = (u64)(t / tiles_x) * MANY_ROWS, x0 = (u64)(t % tiles_x) * X_ROWS;
  const u32 ww = wave % 2 * 128, wx = wave / 2 * (16 * XF);  // the wave's part of the tile

  // what this thread brings to LDS: half the codes of a row, XF pieces of eight elements, a row's scales
  const uint8_t* codes = a.w.codes + min(w0 + tid / 2, (u64)a.w.n - 1) * a.w.steps * MX_STEP_BYTES + tid % 2 * 16;
  const u32* scales = reinterpret_cast<const u32*>(a.w.scales) + min(w0 + tid % MANY_ROWS, (u64)a.w.n - 1) * a.w.steps;
  v4i next_w;
  u32 next_scale = 0;
  Pack<T, 8> next_x[XF];
  const u32 halves = a.w.steps * 2;
  auto fetch = [&](u32 h) {
    next_w = *reinterpret_cast<const v4i*>(codes + (u64)h * 32);
    next_scale = scales[h / 2];
#pragma unroll
    for (int i = 0; i < XF; ++i) next_x[i] = load_batch<T, WIDE>(a, x0 + tid / 8 + 64 * i, h * 64 + tid % 8 * 8);
  };
  auto keep = [&](u32 h, auto ends) {
    char* stage = lds + h % 2 * STAGE;
    const u32 row = tid / 2;
#pragma unroll
    for (u32 e = 0; e < 2; ++e) {  // units of eight bytes, dealt over the banks by the row
      const u32 unit = (tid % 2 * 2 + e + row / 4) % 4;
      *reinterpret_cast<long*>(stage + row * 32 + unit * 8) = e ? (long)(u32)next_w[3] << 32 | (u32)next_w[2] : (long)(u32)next_w[1] << 32 | (u32)next_w[0];
    }
    // (twice for a step and by two threads each, the same value: no branch)
    reinterpret_cast<u32*>(lds + 2 * STAGE)[h / 2 % 2 * MANY_ROWS + tid % MANY_ROWS] = next_scale;
#pragma unroll
    for (int i = 0; i < XF; ++i) {
      if (ends) mask_batch<T, WIDE>(a, next_x[i], h * 64 + tid % 8 * 8);
      v8bf x[PARTS];
      split_pack<T, PARTS>(next_x[i], x);
      const u32 r = tid / 8 + 64 * i;
#pragma unroll
      for (int p = 0; p < PARTS; ++p) *reinterpret_cast<v8bf*>(stage + W_BYTES + p * X_BYTES + r * 128 + (tid % 8 ^ r % 8) * 16) = x[p];
    }
  };
  v4f acc[8][XF] = {};
  fetch(0);
  keep(0, std::true_type());
  fetch(1);
  u32 scale[8];
  auto turn = [&](u32 h, auto ends) __attribute__((always_inline)) {
    __syncthreads();
    const char* stage = lds + h % 2 * STAGE;
    long w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const u32 row = ww + 16 * i + lane % 16;
      w[i] = *reinterpret_cast<const long*>(stage + row * 32 + (lane / 16 + row / 4) % 4 * 8);
      scale[i] = reinterpret_cast<const u32*>(lds + 2 * STAGE)[h / 2 % 2 * MANY_ROWS + row] >> (h % 2 * 16 + lane / 32 * 8) & 255;
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      if (c == 1) {
        // Behind the first products: they run while the next half is put away.  At the end a half too many is, and
        // not read: at a condition the compiler would move the products behind it.
        __builtin_amdgcn_sched_barrier(0);
        keep(h + 1, ends);
        fetch(min(h + 2, halves - 1));
        __builtin_amdgcn_sched_barrier(0);
      }
      v8bf x[XF][PARTS];
#pragma unroll
      for (int j = 0; j < XF; ++j) {
        const u32 r = wx + 16 * j + lane % 16;
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
          x[j][p] = *reinterpret_cast<const v8bf*>(stage + W_BYTES + p * X_BYTES + r * 128 + ((lane / 16 * 2 + c) ^ r % 8) * 16);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const v8bf wv = unpack((u32)(w[i] >> (32 * c)), scale[i]);
#pragma unroll
        for (int j = 0; j < XF; ++j)
#pragma unroll
          for (int p = PARTS - 1; p >= 0; --p) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, x[j][p], acc[i][j], 0, 0, 0);
      }
    }
  };
  // the rows' ends are looked for where they can be
  u32 h = 0;
  for (; h + 1 < a.d / 64; ++h) turn(h, std::false_type());
  for (; h < halves; ++h) turn(h, std::true_type());
  __syncthreads();
  if (w0 + ww < a.w.n) store_results<8, XF>(a, acc, w0 + ww, x0 + wx, lds + wave * store_room<8>());
}

// Few tiles of long rows, which would leave most of the chip idle: 32 4-bit rows x 16 G of the batch a workgroup, whose
// eight waves take an eighth of the steps each, both sides from memory.  Their sums meet in LDS and are added up in
// the order of the steps.
struct Packed {};  // a batch of 4-bit rows
constexpr u32 DEEP_WAVES = 8;
constexpr u32 DEEP_ROWS = 32, DEEP_STRIDE = DEEP_ROWS + 4;

template <typename T, int G>
__global__ __launch_bounds__(64 * DEEP_WAVES, 4) void mx_product_deep_kernel(ProductArgs a, u32 tiles_w) {
  constexpr bool PACKED = __is_same(T, Packed);
  __shared__ __align__(16) float sums[DEEP_WAVES][16 * G][DEEP_STRIDE];
  const u32 tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const u64 w0 = (u64)(blockIdx.x % tiles_w) * DEEP_ROWS, x0 = (u64)(blockIdx.x / tiles_w) * (16 * G);
  const u32 s0 = a.w.steps * wave / DEEP_WAVES, s1 = a.w.steps * (wave + 1) / DEEP_WAVES;
  v4f acc[2][G] = {};
  if constexpr (PACKED) {
    Fragment w[2], x[G];
    auto ask = [&](u32 s) {
#pragma unroll
      for (int i = 0; i < 2; ++i) w[i] = load_fragment(a.w, w0 + 16 * i, s);
#pragma unroll
      for (int j = 0; j < G; ++j) x[j] = load_fragment(a.q, x0 + 16 * j, s);
    };
    ask(min(s0, a.w.steps - 1));
    for (u32 s = s0; s < s1; ++s) {
      Fragment nw[2], nx[G];
#pragma unroll
      for (int i = 0; i < 2; ++i) nw[i] = w[i];
#pragma unroll
      for (int j = 0; j < G; ++j) nx[j] = x[j];
      ask(min(s + 1, s1 - 1));
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < G; ++j) acc[i][j] = mx_mfma(nw[i].codes, nx[j].codes, acc[i][j], nw[i].scale, nx[j].scale);
    }
  } else {
    constexpr int PARTS = parts_of<T>();
    auto turn = [&](u32 s, auto ends) __attribute__((always_inline)) {
      Fragment w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) w[i] = load_fragment(a.w, w0 + 16 * i, s);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const u32 at = s * MX_STEP + lane / 16 * 32 + c * 8;
        Pack<T, 8> in[G];
#pragma unroll
        for (int j = 0; j < G; ++j) in[j] = load_batch<T, true>(a, x0 + 16 * j + lane % 16, at);
        const v8bf wv[2] = {unpack((u32)w[0].codes[c], (u32)w[0].scale), unpack((u32)w[1].codes[c], (u32)w[1].scale)};
#pragma unroll
        for (int j = 0; j < G; ++j) {
          if (ends) mask_batch<T, true>(a, in[j], at);
          v8bf x[PARTS];
          split_pack<T, PARTS>(in[j], x);
#pragma unroll
          for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[i], x[p], acc[i][j], 0, 0, 0);
        }
      }
    };
    u32 s = s0;
    for (; s < min(s1, a.d / MX_STEP); ++s) turn(s, std::false_type());
    for (; s < s1; ++s) turn(s, std::true_type());
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < G; ++j) *reinterpret_cast<v4f*>(&sums[wave][16 * j + lane % 16][16 * i + lane / 16 * 4]) = acc[i][j];
  __syncthreads();
  for (u32 at = tid; at < 16 * G * (DEEP_ROWS / 4); at += 64 * DEEP_WAVES) {
    const u32 r = at / (DEEP_ROWS / 4), c = at % (DEEP_ROWS / 4) * 4;
    v4f sum = *reinterpret_cast<const v4f*>(&sums[0][r][c]);
#pragma unroll
    for (u32 v = 1; v < DEEP_WAVES; ++v) sum += *reinterpret_cast<const v4f*>(&sums[v][r][c]);
    const u64 x = x0 + r, w = w0 + c;
    if (x >= a.nx) continue;
    auto put = [&](auto type) {
      using OUT = decltype(type);
      OUT* to = reinterpret_cast<OUT*>(a.out) + x * a.ldo + w;
      if (a.wide && w + 4 <= a.w.n) {
        Pack<OUT, 4> p;
#pragma unroll
        for (int e = 0; e < 4; ++e) p.v[e] = mx_round<OUT>(sum[e]);
        *reinterpret_cast<Pack<OUT, 4>*>(to) = p;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (w + e < a.w.n) to[e] = mx_round<OUT>(sum[e]);
      }
    };
    if (a.odtype == ANN_F32)
      put(float());
    else if (a.odtype == ANN_F16)
      put(__half());
    else
      put(__bf16());
  }
}

template <typename T, int G>
hipError_t launch_deep(const ProductArgs& a, hipStream_t s) {
  const u32 tiles_w = (u32)(((u64)a.w.n + DEEP_ROWS - 1) / DEEP_ROWS), tiles_x = (a.nx + 16 * G - 1) / (16 * G);
  hipLaunchKernelGGL((mx_product_deep_kernel<T, G>), dim3(tiles_w * tiles_x), dim3(64 * DEEP_WAVES), 0, s, a, tiles_w);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_deep(const ProductArgs& a, hipStream_t s) {
  return a.nx <= 16 ? launch_deep<T, 1>(a, s) : a.nx <= 32 ? launch_deep<T, 2>(a, s) : launch_deep<T, 4>(a, s);
}
// Whether it is the faster one: its time grows with its tiles, that of the kernels with larger tiles with the row's
// length alone as long as these do not fill the chip.  4,096 elements of bf16, by 64 x 4,000 and 64 x 30,000: 21 us
// against 51, and 81 against 55; by 400 x 4,000 and 1,000 x 4,000: 73 against 110, and 159 against 113.  Of fp32, of
// which each product takes three, 32 x 30,000: 132 against 97.
bool deep_pays(const ProductArgs& a, int xdtype) {
  const u32 rows = a.nx <= 16 ? 16 : a.nx <= 32 ? 32 : 64;
  const u64 tiles = (((u64)a.w.n + DEEP_ROWS - 1) / DEEP_ROWS) * (((u64)a.nx + rows - 1) / rows);
  return a.w.steps >= 8 && tiles * rows <= (a.nx > 64 ? 1024 : xdtype == ANN_F32 ? 384 : 512) * 64;
}

template <typename T, int G, int WF, int AHEAD, bool LONG>
hipError_t launch_few(const ProductArgs& a, size_t batch_bytes, u32 runs, hipStream_t s) {
  const u32 tiles = (u32)(((u64)a.w.n + 16 * WF - 1) / (16 * WF));
  // Waves share rows where there is less than one tile for each of 1,024 SIMDs.  One row of 4,096 by 4,000, 16,000 and
  // 20,000: 6.2 us against 14.4 without, 15.0 against 16.4, and 18.3 against 16.9; 32 rows of 1,400 by 16,000 and 40,000:
  // 12.2 against 14.5, and 18.5 against 16.9.
  const u32 share = LONG && tiles < 1024 ? runs : 1;
  constexpr u32 WAVES = FEW_THREADS / 64;
  const size_t lds = batch_bytes + WAVES * few_room<G, WF>(share);
  const auto kernel = mx_product_few_kernel<T, G, WF, AHEAD, LONG>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  const u32 per = WAVES / share, blocks = (tiles + per - 1) / per;
  const u32 room = (u32)(FEW_LDS / lds);  // workgroups that a compute unit holds at once
  const u32 most = 256 * (room > 4 ? 4 : room < 1 ? 1 : room);
  hipLaunchKernelGGL(kernel, dim3(blocks < most ? blocks : most), dim3(FEW_THREADS), lds, s, a, tiles, runs, share);
  return hipGetLastError();
}

template <typename T, int XF>
hipError_t launch_many(const ProductArgs& a, hipStream_t s) {
  constexpr int PARTS = parts_of<T>();
  constexpr int stages = 2 * (MANY_ROWS * 32 + PARTS * 64 * XF * 128) + 2 * MANY_ROWS * 4, room = MANY_THREADS / 64 * store_room<8>();
  constexpr int lds = stages > room ? stages : room;
  auto kernel = mx_product_many_kernel<T, XF, true>;
  if constexpr (XF == 2)  // (up to 64 rows of fewer than eight elements are left to the kernel of few rows)
    if (!a.wide_x) kernel = mx_product_many_kernel<T, XF, false>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  // (launches are counted in threads of 32 bits: long batches go in parts)
  const u32 tiles_w = (u32)(((u64)a.w.n + MANY_ROWS - 1) / MANY_ROWS);
  u64 part = (1u << 22) / tiles_w * (64ull * XF);
  if (part == 0) part = 64 * XF;
  for (u64 at = 0; at < a.nx; at += part) {
    ProductArgs b = a;
    b.nx = (u32)(a.nx - at < part ? a.nx - at : part);
    b.x = a.x + at * a.ldx * sizeof(T);
    b.out = a.out + at * a.ldo * dtype_bytes(a.odtype);
    const u32 tiles = tiles_w * (u32)(((u64)b.nx + 64 * XF - 1) / (64 * XF));
    hipLaunchKernelGGL(kernel, dim3((tiles + 7) / 8 * 8), dim3(MANY_THREADS), lds, s, b, tiles_w, tiles);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

template <typename T, int G>
hipError_t launch_few_rows(const ProductArgs& a, size_t batch, hipStream_t s) {
  // runs of one group of four steps and more
  if constexpr (few_batch(16 * G - 15, LONG_STEPS, parts_of<T>()) <= FEW_BATCH)  // (else no batch of long rows fits)
    if (a.w.steps >= LONG_STEPS)
      return launch_few<T, G, G == 1 ? 1 : 2, G == 1 ? 4 : 2, true>(a, batch, a.w.steps >= 32 ? 8 : a.w.steps >= 16 ? 4 : 2, s);
  return launch_few<T, G, G == 1 ? 2 : 4, 2, false>(a, batch, 1, s);
}

template <typename T>
hipError_t launch_product16(const ProductArgs& a, int xdtype, hipStream_t s) {
  constexpr int PARTS = parts_of<T>();
  const size_t batch = few_batch(a.nx, a.w.steps, PARTS);
  if (a.nx <= 64 && batch <= FEW_BATCH) {
    if (a.nx <= 16) return launch_few_rows<T, 1>(a, batch, s);
    if (a.nx <= 32) return launch_few_rows<T, 2>(a, batch, s);
    if (a.nx <= 48) return launch_few_rows<T, 3>(a, batch, s);
    return launch_few_rows<T, 4>(a, batch, s);
  }
  if (deep_pays(a, xdtype)) return launch_deep<T>(a, s);
  // As wide a tile as the batch fills and registers hold (four columns of fragments of one bf16 number each, two of more).
  // bf16 by rows of 4,096, with 64, 128 and 256 rows of the batch a tile: 64 x 131,072 136 us, 153, 237; 128 x 65,536 109, 74,
  // 116; 192 x 65,536 160, 140, 118; 256 x 65,536 214, 142, 120.  fp32, with 64 and 128: 64 x 65,536 100 and 158, 128 x 65,536 183
  // and 164.  (Few wide tiles can leave compute units idle: 512 x 16,384 114, 74, 110.)
  if (a.nx <= 64) return launch_many<T, 1>(a, s);
  if (a.nx <= 128 || PARTS > 1 || !a.wide_x) return launch_many<T, 2>(a, s);
  if constexpr (PARTS == 1) return launch_many<T, 4>(a, s);
}

hipError_t launch_product(const ProductArgs& a, int xdtype, hipStream_t s) {
  if (xdtype == ANN_F32) return launch_product16<float>(a, xdtype, s);
  if (xdtype == ANN_F16) return launch_product16<__half>(a, xdtype, s);
  if (xdtype == ANN_BF16) return launch_product16<__bf16>(a, xdtype, s);
  if (deep_pays(a, xdtype)) return launch_deep<Packed>(a, s);
  const u64 many_w = ((u64)a.w.n + BOTH_ROWS - 1) / BOTH_ROWS, many_x = ((u64)a.nx + BOTH_ROWS - 1) / BOTH_ROWS;
  const u64 many = many_w * many_x;
  // Short rows of few tiles are left to the smaller tiles: 400 x 10,000, 80 tiles, of 512 elements in 12 us against 14,
  // of 4,096 elements in 79 against 39.
  if (a.w.steps > 2 && many >= (a.w.steps < 8 ? 128 : 24) && many < 1u << 22) {
    constexpr int lds = 2 * (2 * BOTH_ROWS * 128 + 2 * BOTH_ROWS * 8);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(mx_product4_many_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    const u32 tiles = (u32)(many_w * many_x);
    hipLaunchKernelGGL(mx_product4_many_kernel, dim3((tiles + 7) / 8 * 8), dim3(BOTH_THREADS), lds, s, a, (u32)many_w, tiles);
    return hipGetLastError();
  }
  const u32 tiles_w = (u32)(((u64)a.w.n + 127) / 128);
  const u64 tiles = tiles_w * (((u64)a.nx + 127) / 128);
  const dim3 grid((u32)(tiles < (1u << 20) ? tiles : (1u << 20)));
  hipLaunchKernelGGL(mx_product4_kernel, grid, dim3(256), 0, s, a, tiles_w, tiles);
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
  a.odtype = odtype;
  HIP_TRY(launch_product(a, xdtype, static_cast<hipStream_t>(stream)));
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
  a.wide_x = d >= 8;
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
