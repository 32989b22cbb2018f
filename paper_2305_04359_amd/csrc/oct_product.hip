// Products of 8-bit rows with 8-bit rows.
#include <type_traits>

#include "oct.hpp"

namespace annmi {

struct OctProductArgs {
  OctRows w;  // n rows: the columns of `out`
  OctRows x;  // nx rows: its rows
  char* out;
  u64 ldo;
  int odtype;
  u32 wide;  // four results can be written at once
};

// Two ways to multiply rows by rows.  A lane holds its share of a row's elements, the same ones on both sides, in whatever
// order: all 128 of a step share one scale.
//   exact   The codes become bf16 numbers times their scale, which is exact (down to 2^-126), and so are their products in
//           the matrix instruction, whose sums are fp32.
//   coded   The matrix instruction takes the codes, at twice the rate.  It brings eight neighbouring products to the
//           exponent E of the largest of them and drops what lies below 2^(E - 13) before it adds them up (and on
//           from there in fp32): never more than 7 * 2^-13 of the largest products of all eights together.  2,048 x 4,096 of
//           2,048 and of 8,192 normal numbers are off by some 1.6e-5 of the results' rms, with a hundredth of the
//           channels twelve times as large by 7.7e-5.  It serves ANN_BF16, whose own rounding is 1.66e-3: with it
//           1.656e-3 and 1.658e-3.  Of ANN_F16's rounding, 2.07e-4, it would be more than a third: those products are whole.

// a lane's 32 elements of a step, in two halves
struct Codes {
  v4i low, high;
};
// Eight codes as bf16 numbers times their scale.  The conversion reads the exponent bits of its scale alone, so that a
// scale byte needs no care at its ends: 0 is 2^-127 and 255 is NaN.
__device__ __forceinline__ v8bf oct_bf16(u32 low, u32 high, u32 byte) {
  const float scale = __uint_as_float(byte << 23);
  const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, scale, true);
  const v2bf c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, scale, true);
  return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// the c-th quarter of a lane's elements
__device__ __forceinline__ v8bf oct_quarter(const Codes& v, int c, u32 byte) {
  const v4i half = c < 2 ? v.low : v.high;
  return oct_bf16((u32)half[c % 2 * 2], (u32)half[c % 2 * 2 + 1], byte);
}

// The 16 WF x 16 XF results of a wave.  They lie in the matrix instruction's order (a lane holds four neighbours of a
// row of `out`); through LDS of the wave's own they get into runs of a whole row's part, so that stores fill lines
// wherever a row of `out` begins.
template <int WF>
constexpr u32 oct_room() {
  return 16 * (16 * WF + 4) * 4;  // bytes of LDS for a wave: the four floats more keep rows in different banks
}
template <typename OUT, int WF, int XF>
__device__ __forceinline__ void oct_store_as(const OctProductArgs& a, const v4f (&acc)[WF][XF], u64 w0, u64 x0, float* room) {
  constexpr u32 ROW = 16 * WF, STRIDE = ROW + 4;
  const u32 lane = threadIdx.x % 64;
#pragma unroll
  for (int j = 0; j < XF; ++j) {
    if (x0 + 16 * j >= a.x.n) break;
    wave_exchange();
#pragma unroll
    for (int i = 0; i < WF; ++i) *reinterpret_cast<v4f*>(room + lane % 16 * STRIDE + 16 * i + lane / 16 * 4) = acc[i][j];
    wave_exchange();
    OUT* out = reinterpret_cast<OUT*>(a.out) + (x0 + 16 * j) * a.ldo + w0;
    const u32 xs = (u32)min((u64)16, a.x.n - (x0 + 16 * j)), ws = (u32)min((u64)ROW, a.w.n - w0);
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
__device__ __forceinline__ void oct_store(const OctProductArgs& a, const v4f (&acc)[WF][XF], u64 w0, u64 x0, char* room) {
  if (a.odtype == ANN_F32)
    oct_store_as<float, WF, XF>(a, acc, w0, x0, reinterpret_cast<float*>(room));
  else if (a.odtype == ANN_F16)
    oct_store_as<__half, WF, XF>(a, acc, w0, x0, reinterpret_cast<float*>(room));
  else
    oct_store_as<__bf16, WF, XF>(a, acc, w0, x0, reinterpret_cast<float*>(room));
}

// `rows` rows of the batch from `at` on
OctProductArgs rows_from(const OctProductArgs& a, u64 at, u64 rows) {
  OctProductArgs b = a;
  b.x.n = (u32)(a.x.n - at < rows ? a.x.n - at : rows);
  b.x.codes += at * a.x.steps * OCT_STEP;
  b.x.scales += at * oct_words(a.x.steps);
  b.out += at * a.ldo * dtype_bytes(a.odtype);
  return b;
}

// Few rows of x, or few tiles: both sides from memory, 16 WF x 16 XF results a wave, exact.  Lane l holds row l & 15 of a
// fragment; D's column (x) is l & 15 too, its rows (w) 4 (l >> 4) and the three after.  SHARE waves take a part of the steps
// each; their sums meet in LDS and are added up in the order of the steps.  A step's fragments are asked for while the
// one before is multiplied.  One row of 4,096 by 131,072 is bound by memory: 98 us, 5.5 TB/s.
constexpr u32 DIRECT_WAVES = 8;
template <int WF, int XF, int SHARE>
constexpr u32 direct_room() {
  return SHARE > 1 && WF * XF * 1024 > oct_room<WF>() ? WF * XF * 1024 : oct_room<WF>();
}

template <int WF, int XF, int SHARE>
__global__ __launch_bounds__(64 * DIRECT_WAVES) void oct_product_direct_kernel(OctProductArgs a, u32 tiles_w, u64 tiles) {
  constexpr u32 ROOM = direct_room<WF, XF, SHARE>();
  __shared__ __align__(16) char lds[DIRECT_WAVES * ROOM];
  const u32 lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  char* room = lds + wave * ROOM;
  const u64 t = blockIdx.x * (u64)(DIRECT_WAVES / SHARE) + wave / SHARE;
  const bool mine = t < tiles;
  const u64 w0 = mine ? t % tiles_w * (16 * WF) : 0, x0 = mine ? t / tiles_w * (16 * XF) : 0;
  const u32 steps = a.w.steps, words = oct_words(steps);
  const u32 s0 = steps * (wave % SHARE) / SHARE, s1 = steps * (wave % SHARE + 1) / SHARE;
  const uint8_t* wc[WF];
  const uint8_t* xc[XF];
  const u32* wsc[WF];
  const u32* xsc[XF];
  // rows past the last are read as the last one: their results go nowhere
#pragma unroll
  for (int i = 0; i < WF; ++i) {
    const u64 r = min(w0 + 16 * i + lane % 16, (u64)a.w.n - 1);
    wc[i] = a.w.codes + r * steps * OCT_STEP + lane / 16 * 16;
    wsc[i] = a.w.scales + r * words;
  }
#pragma unroll
  for (int j = 0; j < XF; ++j) {
    const u64 r = min(x0 + 16 * j + lane % 16, (u64)a.x.n - 1);
    xc[j] = a.x.codes + r * steps * OCT_STEP + lane / 16 * 16;
    xsc[j] = a.x.scales + r * words;
  }
  v4f acc[WF][XF] = {};
  if (s0 < s1) {
    Codes w[WF], x[XF];
    u32 ws[WF], xs[XF];
    auto ask = [&](u32 s) {
#pragma unroll
      for (int i = 0; i < WF; ++i) {
        w[i].low = *reinterpret_cast<const v4i*>(wc[i] + (u64)s * OCT_STEP);
        w[i].high = *reinterpret_cast<const v4i*>(wc[i] + (u64)s * OCT_STEP + 64);
        ws[i] = wsc[i][s / 4];
      }
#pragma unroll
      for (int j = 0; j < XF; ++j) {
        x[j].low = *reinterpret_cast<const v4i*>(xc[j] + (u64)s * OCT_STEP);
        x[j].high = *reinterpret_cast<const v4i*>(xc[j] + (u64)s * OCT_STEP + 64);
        xs[j] = xsc[j][s / 4];
      }
    };
    ask(s0);
    for (u32 s = s0; s < s1; ++s) {
      Codes nw[WF], nx[XF];
      u32 nws[WF], nxs[XF];
#pragma unroll
      for (int i = 0; i < WF; ++i) nw[i] = w[i], nws[i] = ws[i] >> (s % 4 * 8) & 255;
#pragma unroll
      for (int j = 0; j < XF; ++j) nx[j] = x[j], nxs[j] = xs[j] >> (s % 4 * 8) & 255;
      ask(min(s + 1, s1 - 1));
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        v8bf wv[WF];
#pragma unroll
        for (int i = 0; i < WF; ++i) wv[i] = oct_quarter(nw[i], c, nws[i]);
#pragma unroll
        for (int j = 0; j < XF; ++j) {
          const v8bf xv = oct_quarter(nx[j], c, nxs[j]);
#pragma unroll
          for (int i = 0; i < WF; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[i], xv, acc[i][j], 0, 0, 0);
        }
      }
    }
  }
  if constexpr (SHARE > 1) {
    if (wave % SHARE)
#pragma unroll
      for (int i = 0; i < WF * XF; ++i) *reinterpret_cast<v4f*>(room + lane * 16 + i * 1024) = acc[i / XF][i % XF];
    __syncthreads();
    if (wave % SHARE) return;
    for (u32 o = 1; o < SHARE; ++o)
#pragma unroll
      for (int i = 0; i < WF * XF; ++i) acc[i / XF][i % XF] += *reinterpret_cast<const v4f*>(room + o * ROOM + lane * 16 + i * 1024);
  }
  if (mine && w0 < a.w.n) oct_store<WF, XF>(a, acc, w0, x0, room);
}

template <int WF, int XF, int SHARE>
hipError_t launch_direct(const OctProductArgs& a, hipStream_t s) {
  const u32 tiles_w = (u32)(((u64)a.w.n + 16 * WF - 1) / (16 * WF));
  constexpr u32 PER = DIRECT_WAVES / SHARE;
  // (launches are counted in threads of 32 bits: long batches go in parts)
  u64 part = (1ull << 22) * PER / tiles_w * (16 * XF);
  if (part == 0) part = 16 * XF;
  for (u64 at = 0; at < a.x.n; at += part) {
    const OctProductArgs b = rows_from(a, at, part);
    const u64 tiles = (u64)tiles_w * (((u64)b.x.n + 16 * XF - 1) / (16 * XF));
    hipLaunchKernelGGL((oct_product_direct_kernel<WF, XF, SHARE>), dim3((u32)((tiles + PER - 1) / PER)), dim3(64 * DIRECT_WAVES), 0, s, b, tiles_w, tiles);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Many rows of both sides.  Steps pass through LDS by halves (64 elements), from memory to LDS without registers between;
// a wave takes 32 rows by 32 rows at once.  In LDS the four pieces of 16 bytes of a row's half change places by the row's
// number, so that lanes that read the same piece of neighbouring rows meet all banks: of eight rows as of sixteen.  (By two
// bits of the row's number, which serves eight, half of the time of LDS went into conflicts.)
constexpr u32 HALF = 64;
__device__ __forceinline__ u32 half_place(u32 row, u32 piece) { return piece ^ (row >> 2 & 1) ^ ((row >> 1 ^ row >> 3) & 1) << 1; }
using v16f = float __attribute__((ext_vector_type(16)));

// 32 WF x 32 XF results of a wave: a half's fragments, and what is made of them.  Lane l holds row l & 31 of each side and
// pieces l >> 5 and two on; its results are column (x) l & 31 and rows (w) 4 (l >> 5) and the three after of every eight.
template <int WF, int XF>
struct Wave32 {
  v8i w[WF], x[XF];
  v16f acc[WF][XF];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < WF; ++i)
#pragma unroll
      for (int j = 0; j < XF; ++j) acc[i][j] = v16f{};
  }
  static __device__ __forceinline__ v8i fragment(const char* rows) {
    const u32 lane = threadIdx.x % 64, at = lane % 32 * HALF + half_place(lane, lane / 32) * 16;
    return __builtin_shufflevector(*reinterpret_cast<const v4i*>(rows + at), *reinterpret_cast<const v4i*>(rows + (at ^ 32)), 0, 1, 2, 3, 4, 5, 6, 7);
  }
  __device__ __forceinline__ void read(const char* wrows, const char* xrows) {
#pragma unroll
    for (int j = 0; j < XF; ++j) x[j] = fragment(xrows + 32 * j * HALF);
#pragma unroll
    for (int i = 0; i < WF; ++i) w[i] = fragment(wrows + 32 * i * HALF);
  }
  // BYTE: the step's byte of the scale words
  template <bool CODED, int BYTE>
  __device__ __forceinline__ void multiply(const u32 (&ws)[WF], const u32 (&xs)[XF]) {
    if constexpr (CODED) {
#pragma unroll
      for (int i = 0; i < WF; ++i)
#pragma unroll
        for (int j = 0; j < XF; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[i], x[j], acc[i][j], 0, 0, BYTE, (int)ws[i], BYTE, (int)xs[j]);
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        v8bf xv[XF];
#pragma unroll
        for (int j = 0; j < XF; ++j) xv[j] = oct_bf16((u32)x[j][2 * c], (u32)x[j][2 * c + 1], xs[j] >> (8 * BYTE) & 255);
#pragma unroll
        for (int i = 0; i < WF; ++i) {
          const v8bf wv = oct_bf16((u32)w[i][2 * c], (u32)w[i][2 * c + 1], ws[i] >> (8 * BYTE) & 255);
#pragma unroll
          for (int j = 0; j < XF; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wv, xv[j], acc[i][j], 0, 0, 0);
        }
      }
    }
    // (or the compiler would gather the products of several halves behind the last one's reads)
#pragma unroll
    for (int i = 0; i < WF; ++i)
#pragma unroll
      for (int j = 0; j < XF; ++j) asm volatile("" : "+v"(acc[i][j]));
  }
  // Results to memory, through LDS of the wave's own: 32 rows of `out` by all the wave's columns at once, so that stores
  // fill lines, and neighbouring ones, wherever a row of `out` begins.  (128 bytes of a row at once: 4,096 x 65,536 of 2,048
  // to bf16 639 us, 256 bytes 600.)  They go through the caches: past them that product takes 552 us rather than 585, but with a
  // copy of its results behind it 845 rather than 788.  Pieces of 16 bytes change places by the row's number in LDS.
  template <typename OUT>
  __device__ __forceinline__ void store(const OctProductArgs& a, u64 w0, u64 x0, char* room) const {
    constexpr u32 ROW = 32 * WF * sizeof(OUT), PIECES = ROW / 16, AT_ONCE = 64 / PIECES;  // bytes; rows a store
    constexpr u32 E = 16 / sizeof(OUT);
    const u32 lane = threadIdx.x % 64;
#pragma unroll
    for (int j = 0; j < XF; ++j) {
      wave_exchange();
#pragma unroll
      for (int i = 0; i < WF; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          Pack<OUT, 4> p;
#pragma unroll
          for (int e = 0; e < 4; ++e) p.v[e] = mx_round<OUT>(acc[i][j][4 * q + e]);
          const u32 byte = (32 * i + 8 * q + lane / 32 * 4) * sizeof(OUT);
          *reinterpret_cast<Pack<OUT, 4>*>(room + lane % 32 * ROW + ((byte / 16 ^ lane % 8) * 16 | byte % 16)) = p;
        }
      wave_exchange();
      OUT* out = reinterpret_cast<OUT*>(a.out) + (x0 + 32 * j) * a.ldo + w0;
      const u32 xs = x0 + 32 * j < a.x.n ? (u32)min((u64)32, a.x.n - (x0 + 32 * j)) : 0;
      if (w0 + 32 * WF <= a.w.n) {
#pragma unroll
        for (u32 k = 0; k < 32; k += AT_ONCE) {
          const u32 r = k + lane / PIECES, piece = lane % PIECES;
          const v4i p = *reinterpret_cast<const v4i*>(room + r * ROW + (piece ^ r % 8) * 16);
          if (r < xs) __builtin_memcpy(out + r * a.ldo + piece * E, &p, 16);
        }
      } else {  // the last columns
        const u32 ws = w0 < a.w.n ? (u32)(a.w.n - w0) : 0;
#pragma unroll 1
        for (u32 at = lane; at < 32 * 32 * WF; at += 64) {
          const u32 r = at / (32 * WF), c = at % (32 * WF), byte = c * sizeof(OUT);
          const OUT v = *reinterpret_cast<const OUT*>(room + r * ROW + ((byte / 16 ^ r % 8) * 16 | byte % 16));
          if (r < xs && c < ws) out[r * a.ldo + c] = v;
        }
      }
    }
  }
  static constexpr u32 ROOM = 32 * 32 * WF * 4;  // bytes that this takes at most
  template <bool CODED>
  __device__ __forceinline__ void store_results(const OctProductArgs& a, u64 w0, u64 x0, char* room) const {
    if constexpr (CODED)
      store<__bf16>(a, w0, x0, room);
    else if (a.odtype == ANN_F32)
      store<float>(a, w0, x0, room);
    else
      store<__half>(a, w0, x0, room);
  }
};

// One side's rows of a tile as the WAVES waves of a workgroup bring them to LDS, 16 rows at a time a wave, 16 bytes a
// lane.  Rows past the last are read as the last one: their results go nowhere.
template <int ROWS, int WAVES>
struct Side {
  static constexpr int LOADS = ROWS / (16 * WAVES);
  const uint8_t* codes;
  const u32* scales;
  u32 last;  // row
  u32 offset[LOADS];
  __device__ __forceinline__ void set(const OctRows& m, u64 row0) {
    const u32 lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    codes = m.codes + row0 * m.steps * OCT_STEP;
    scales = m.scales + row0 * oct_words(m.steps);
    last = (u32)min((u64)ROWS, m.n - row0) - 1;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      offset[i] = min((wave + WAVES * i) * 16 + lane / 4, last) * m.steps * OCT_STEP + half_place(lane / 4, lane % 4) * 16;
  }
  __device__ __forceinline__ void fetch(u32 half, char* to) const {
    typedef __attribute__((address_space(1))) const void* From;
    typedef __attribute__((address_space(3))) void* To;
    const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      __builtin_amdgcn_global_load_lds((From)(codes + (u64)half * HALF + offset[i]), (To)(to + (wave + WAVES * i) * 1024), 16, 0, 0);
  }
  // scale words of the rows of N fragments from `row` of the tile on
  template <int N>
  __device__ __forceinline__ void fetch_scales(u32 (&to)[N], u32 row, u32 word, u32 words) const {
#pragma unroll
    for (int i = 0; i < N; ++i) to[i] = scales[min(row + 32 * i + threadIdx.x % 32, last) * words + word];
  }
};

// The tile of a workgroup.  Chiplets take workgroups in turn: each gets a run of tiles.  A run goes through eight tiles' rows
// of x for one tile's rows of w before it takes the next rows of w, so that both stay in the chiplet's cache.
struct TileAt {
  u64 w, x;
};
__device__ __forceinline__ TileAt tile_at(u32 t, u32 tiles_w, u32 tiles_x) {
  const u32 size = 8 * tiles_w, group = t / size, first = group * 8, across = min(8u, tiles_x - first), in = t % size;
  return {in / across, first + in % across};
}

// BW x BX results a workgroup of four waves, 64 x 64 a wave: 128 x 128, or 256 x 64 for batches of few rows.  Two
// workgroups and more a compute unit, one of which stores or waits while another multiplies.  33 x 500,001 of 200 to fp32
// take 38 us, 4.4 TB/s (by tiles of 128 x 128 45); 64 x 131,072 of 4,096 136 us to fp32 and 128 to bf16 (4.2 TB/s).
constexpr u32 SMALL = 128, NARROW_W = 256, NARROW_X = 64, SMALL_BUFFERS = 3;
template <bool CODED, int BW, int BX>
__global__ __launch_bounds__(256, 2) void oct_product_small_kernel(OctProductArgs a, u32 tiles_w, u32 tiles) {
  static_assert(BW * BX == 4 * 64 * 64);
  constexpr u32 BUFFER = (BW + BX) * HALF;
  __shared__ __align__(1024) char lds[SMALL_BUFFERS * BUFFER];
  const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const u32 per = (tiles + 7) / 8, t = blockIdx.x % 8 * per + blockIdx.x / 8;
  if (t >= tiles) return;
  const TileAt at = tile_at(t, tiles_w, tiles / tiles_w);
  const u32 ww = wave % (BW / 64) * 64, wx = wave / (BW / 64) * 64;  // the wave's part of the tile
  const u32 steps = a.w.steps, words = oct_words(steps), halves = 2 * steps;
  Side<BW, 4> w;
  Side<BX, 4> x;
  w.set(a.w, at.w * BW);
  x.set(a.x, at.x * BX);
  constexpr int LOADS = w.LOADS + x.LOADS;
  auto fetch = [&](u32 h) {  // (past the last half: the last one again, which nobody reads)
    char* to = lds + h % SMALL_BUFFERS * BUFFER;
    w.fetch(min(h, halves - 1), to);
    x.fetch(min(h, halves - 1), to + BW * HALF);
  };
  Wave32<2, 2> v;
  v.clear();
  u32 ws[2], xs[2], next_w[2], next_x[2];
  w.fetch_scales(ws, ww, 0, words);
  x.fetch_scales(xs, wx, 0, words);
  fetch(0);
  fetch(1);
  auto half = [&](u32 h, auto byte) {
    // this wave's loads of the half are in LDS, and its reads of the half before are done; then so are all waves'
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
    fetch(h + 2);
    const char* rows = lds + h % SMALL_BUFFERS * BUFFER;
    v.read(rows + ww * HALF, rows + (BW + wx) * HALF);
    v.template multiply<CODED, byte>(ws, xs);
  };
  u32 h = 0;
  for (; h + 8 <= halves; h += 8) {
    w.fetch_scales(next_w, ww, min(h / 8 + 1, words - 1), words);
    x.fetch_scales(next_x, wx, min(h / 8 + 1, words - 1), words);
    half(h, std::integral_constant<int, 0>());
    half(h + 1, std::integral_constant<int, 0>());
    half(h + 2, std::integral_constant<int, 1>());
    half(h + 3, std::integral_constant<int, 1>());
    half(h + 4, std::integral_constant<int, 2>());
    half(h + 5, std::integral_constant<int, 2>());
    half(h + 6, std::integral_constant<int, 3>());
    half(h + 7, std::integral_constant<int, 3>());
#pragma unroll
    for (int i = 0; i < 2; ++i) ws[i] = next_w[i], xs[i] = next_x[i];
  }
  for (; h < halves; h += 2) {
    half(h, std::integral_constant<int, 0>());
    half(h + 1, std::integral_constant<int, 0>());
#pragma unroll
    for (int i = 0; i < 2; ++i) ws[i] >>= 8, xs[i] >>= 8;
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  v.template store_results<CODED>(a, at.w * BW + ww, at.x * BX + wx, lds + wave * v.ROOM);
}

// 256 x 256 results a workgroup of eight waves, 128 x 64 a wave, two waves a SIMD, in two teams: while one team's
// waves multiply a half the other's read theirs from LDS and ask for the half three on.  8,192 x 8,192 of 8,192 to bf16
// take 470 us, 2.34 PFLOP/s; 4,096 x 65,536 of 2,048 592 us, 1.86 PFLOP/s, of which the results' way to memory is some 120;
// 4,096 x 4,096 of 8,192 to fp32 (exact) 212 us, 1.30 PFLOP/s.  Of random codes no more than 3.3 PFLOP/s come out when
// nothing is loaded and nothing read from LDS, 2.95 when nothing is loaded: the clock falls under the load.  Workgroups that
// stay for several tiles, with the next one's halves on their way before the results leave, were 2 % faster where
// results took most (639 us and 626 with another way to store them) and no faster elsewhere.
constexpr u32 LARGE = 256, LARGE_BUFFERS = 4;
constexpr u32 LARGE_LDS = LARGE_BUFFERS * 2 * LARGE * HALF;
template <bool CODED>
__global__ __launch_bounds__(512) void oct_product_large_kernel(OctProductArgs a, u32 tiles_w, u32 tiles) {
  constexpr u32 BUFFER = 2 * LARGE * HALF;
  extern __shared__ __align__(1024) char lds[];
  const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const u32 per = (tiles + 7) / 8, t = blockIdx.x % 8 * per + blockIdx.x / 8;
  if (t >= tiles) return;
  const TileAt at = tile_at(t, tiles_w, tiles / tiles_w);
  const u32 ww = wave % 2 * 128, wx = wave / 2 * 64;  // the wave's part of the tile
  const bool late = wave >= 4;                        // the second team
  const u32 steps = a.w.steps, words = oct_words(steps), halves = 2 * steps;
  Side<LARGE, 8> w, x;
  w.set(a.w, at.w * LARGE);
  x.set(a.x, at.x * LARGE);
  constexpr int LOADS = 2 * Side<LARGE, 8>::LOADS;
  auto fetch = [&](u32 h) {  // (past the last half: the last one again, which nobody reads)
    char* to = lds + h % LARGE_BUFFERS * BUFFER;
    w.fetch(min(h, halves - 1), to);
    x.fetch(min(h, halves - 1), to + LARGE * HALF);
  };
  Wave32<4, 2> v;
  v.clear();
  u32 ws[4], xs[2], next_w[4], next_x[2];
  w.fetch_scales(ws, ww, 0, words);
  x.fetch_scales(xs, wx, 0, words);
  fetch(0);
  fetch(1);
  fetch(2);
  // This wave's loads but those of the last two halves are in LDS, and its reads are done; then so are the others'.  The
  // half that is read behind it was asked for three halves ago.
  auto turn = [&]() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * LOADS) : "memory"); };
  auto half = [&](u32 h, auto byte) {
    const char* rows = lds + h % LARGE_BUFFERS * BUFFER;
    v.read(rows + ww * HALF, rows + (LARGE + wx) * HALF);
    fetch(h + 3);  // (where the half before was: both teams have read it)
    turn();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
    v.template multiply<CODED, byte>(ws, xs);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    turn();
  };
  turn();
  if (late) asm volatile("s_barrier" ::: "memory");  // half a turn behind, from here to the end
  u32 h = 0;
  for (; h + 8 <= halves; h += 8) {
    w.fetch_scales(next_w, ww, min(h / 8 + 1, words - 1), words);
    x.fetch_scales(next_x, wx, min(h / 8 + 1, words - 1), words);
    half(h, std::integral_constant<int, 0>());
    half(h + 1, std::integral_constant<int, 0>());
    half(h + 2, std::integral_constant<int, 1>());
    half(h + 3, std::integral_constant<int, 1>());
    half(h + 4, std::integral_constant<int, 2>());
    half(h + 5, std::integral_constant<int, 2>());
    half(h + 6, std::integral_constant<int, 3>());
    half(h + 7, std::integral_constant<int, 3>());
#pragma unroll
    for (int i = 0; i < 4; ++i) ws[i] = next_w[i];
#pragma unroll
    for (int j = 0; j < 2; ++j) xs[j] = next_x[j];
  }
  for (; h < halves; h += 2) {
    half(h, std::integral_constant<int, 0>());
    half(h + 1, std::integral_constant<int, 0>());
#pragma unroll
    for (int i = 0; i < 4; ++i) ws[i] >>= 8;
#pragma unroll
    for (int j = 0; j < 2; ++j) xs[j] >>= 8;
  }
  if (!late) asm volatile("s_barrier" ::: "memory");
  asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");  // (no load is on its way to where results pass)
  v.template store_results<CODED>(a, at.w * LARGE + ww, at.x * LARGE + wx, lds + wave * v.ROOM);
}

template <bool CODED>
hipError_t launch_large(const OctProductArgs& a, hipStream_t s) {
  const auto kernel = oct_product_large_kernel<CODED>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)LARGE_LDS);
  if (e != hipSuccess) return e;
  const u32 tiles_w = (u32)(((u64)a.w.n + LARGE - 1) / LARGE), tiles = tiles_w * (u32)(((u64)a.x.n + LARGE - 1) / LARGE);
  hipLaunchKernelGGL(kernel, dim3((tiles + 7) / 8 * 8), dim3(512), LARGE_LDS, s, a, tiles_w, tiles);
  return hipGetLastError();
}
template <bool CODED, int BW, int BX>
hipError_t launch_small(const OctProductArgs& a, hipStream_t s) {
  const u32 tiles_w = (u32)(((u64)a.w.n + BW - 1) / BW);
  // (launches are counted in threads of 32 bits: long batches go in parts)
  u64 part = (1ull << 23) / tiles_w * BX;
  if (part == 0) part = BX;
  for (u64 at = 0; at < a.x.n; at += part) {
    const OctProductArgs b = rows_from(a, at, part);
    const u32 tiles = tiles_w * (u32)(((u64)b.x.n + BX - 1) / BX);
    hipLaunchKernelGGL((oct_product_small_kernel<CODED, BW, BX>), dim3((tiles + 7) / 8 * 8), dim3(256), 0, s, b, tiles_w, tiles);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <bool CODED>
hipError_t launch_tiles(const OctProductArgs& a, hipStream_t s) {
  if (a.x.n <= NARROW_X) return launch_small<CODED, NARROW_W, NARROW_X>(a, s);
  // By what a turn of workgroups over the chip takes: 256 large tiles, 256 small ones or twice as many.  What a tile
  // takes besides its steps is more for large ones.  To bf16 by large tiles and by small ones: 2,048 x 8,192 of 4,096 elements
  // 67 us and 91, 1,024 x 4,096 of 4,096 46 and 27, 2,048 x 4,096 of 8,192 97 and 93, 4,096 x 32,768 of 1,024 170 and
  // 196, 256 x 131,072 of 1,024 47 and 53, 1,000 x 100,000 of 256 63 and 56; 1,000 x 10,000 of 1,000 to fp32 36 and 31.
  const u64 large = (((u64)a.w.n + LARGE - 1) / LARGE) * (((u64)a.x.n + LARGE - 1) / LARGE);
  const u64 small = (((u64)a.w.n + SMALL - 1) / SMALL) * (((u64)a.x.n + SMALL - 1) / SMALL);
  const u64 cost_large = (large + 255) / 256 * (a.w.steps < 16 ? 77 : 64);
  const u64 cost_small = small / 512 * 45 + (small % 512 == 0 ? 0 : small % 512 <= 256 ? 25 : 45);
  if (a.w.steps >= 4 && large < 1u << 22 && cost_large <= cost_small) return launch_large<CODED>(a, s);
  return launch_small<CODED, SMALL, SMALL>(a, s);
}

hipError_t launch_oct_product(const OctProductArgs& a, hipStream_t s) {
  const u64 tiles = (((u64)a.w.n + 31) / 32) * (((u64)a.x.n + 31) / 32);
  if (a.x.n <= 16) {
    // Waves that share a tile's steps read longer pieces of fewer rows at a time, and the last turn of workgroups costs less;
    // tiles of 64 rows read the batch half as often.  Each its own tile of 32, eight sharing one of 32, four and eight one of 64:
    // 1 row of 4,096 by 131,072 118 us, 100, 100 and 98, 16 rows 140, 145, 120 and 120; 1 by 65,600 107, 57, 70 and 60.
    // 1 row of 1,024 by 100,000 25, 20, 24 and 24, 16 rows 28, 25, 27 and 27, by 131,072 32, 34, 31 and 35; 1 row of 200 by 65,536
    // 5.6, 7.4, 6.2 and 8.6; 1 of 768 by 20,000 9.6, 6.4, 8.0 and 7.2, by 40,000 9.9, 9.6, 11 and 12.
    if (tiles < (a.w.steps >= 6 ? 2048 : 1024)) return launch_direct<2, 1, 8>(a, s);
    if (a.w.steps < 4 || a.w.n >= 1u << 27) return launch_direct<2, 1, 1>(a, s);  // (of the others' tiles there may be too many to launch)
    if (a.w.steps >= 24) return launch_direct<4, 1, 8>(a, s);
    return a.x.n <= 4 && a.w.steps >= 8 ? launch_direct<2, 1, 8>(a, s) : launch_direct<4, 1, 4>(a, s);
  }
  if (tiles <= 640) return launch_direct<2, 2, 8>(a, s);
  // (bf16 rounds twenty times as coarsely as the codes' products are cut; fp16 does not)
  return a.odtype == ANN_BF16 ? launch_tiles<true>(a, s) : launch_tiles<false>(a, s);
}

}  // namespace annmi

using namespace annmi;

extern "C" {

int ann_oct_product(const uint8_t* xcodes_dev, const uint8_t* xscales_dev, uint64_t nx, const uint8_t* codes_dev,
                   const uint8_t* scales_dev, uint64_t n, uint32_t d, void* out_dev, ann_dtype out_dtype, uint64_t ldo,
                   void* stream) try {
  int rc = check_oct_rows("ann_oct_product", codes_dev, scales_dev, n, d);
  if (rc) return rc;
  rc = check_oct_rows("ann_oct_product", xcodes_dev, xscales_dev, nx, d);
  if (rc) return rc;
  const u64 osz = dtype_bytes(out_dtype);
  if (osz < 2) return fail(ANN_EINVAL, "out must be ANN_F32, ANN_F16 or ANN_BF16");
  if (ldo < n) return fail(ANN_EINVAL, "ldo must be at least n");
  if (nx == 0 || n == 0) return ANN_OK;
  if (!out_dev) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(out_dev, osz)) return fail(ANN_EINVAL, "out not aligned to its elements");
  const u32 steps = oct_steps(d);
  OctProductArgs a{{codes_dev, reinterpret_cast<const u32*>(scales_dev), (u32)n, steps},
                  {xcodes_dev, reinterpret_cast<const u32*>(xscales_dev), (u32)nx, steps},
                  static_cast<char*>(out_dev), ldo, out_dtype, aligned_to(out_dev, 4 * osz) && ldo % 4 == 0};
  HIP_TRY(launch_oct_product(a, static_cast<hipStream_t>(stream)));
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

}  // extern "C"
