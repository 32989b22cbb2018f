// The k nearest of all microscaled 4-bit rows: scores on the matrix cores, of which only the largest of each
// group of rows leaves the chip.
//
// The points of a row of scores are ordered by (score downwards, id).  Let the groups of GROUP consecutive rows be
// ordered by (largest score downwards, group).  The k best points lie in the first k groups: a point p outside of
// them has k groups before its own; each holds a point whose score is above p's, or equal with a smaller id.  So
// the first kernel writes one number for each group, and the second one scores the rows of k groups again.
#include "mx.hpp"

namespace annmi {

constexpr u32 SEARCH_GROUP = 64;
constexpr u32 SEARCH_MOST_K = 128;
constexpr u64 SEARCH_SCRATCH_FLOATS = 1ull << 28;  // of group maxima held at a time, where 64 queries fit in them
constexpr u64 SEARCH_MOST_AT_ONCE = 1ull << 22;   // queries of a launch: its threads are counted in 32 bits

struct MxSearchArgs {
  MxRows w, q;
  const float* norms;   // null: inner products
  const float* qnorms;
  u32 q0, nq;           // the queries of this launch
  u32 groups, pitch, k; // pitch: floats from one query's maxima to the next's
  float* most;          // (nq, pitch)
  float* coarse;        // (nq, coarse_pitch): the largest of every `per_coarse` of them, or null
  u32 coarse_pitch, per_coarse;
  u32* ids;
  float* dists;
};

__device__ __forceinline__ v4i load_codes(const MxRows& m, u64 row, u32 step) {
  return *reinterpret_cast<const v4i*>(m.codes + (row * m.steps + step) * MX_STEP_BYTES + threadIdx.x % 64 / 16 * 16);
}
__device__ __forceinline__ int load_scale(const MxRows& m, u64 row, u32 step) {
  return m.scales[(row * m.steps + step) * MX_STEP_SCALES + threadIdx.x % 64 / 16];
}

// What the sum of a row starts from: 0, or - |x|^2 / 2, and -inf past the last row, which no maximum takes.  Without
// norms something else of at least that size is read and not used, so that no branch waits for the load.
__device__ __forceinline__ float load_norm(const MxSearchArgs& a, u64 row) {
  const float* from = a.norms ? a.norms : reinterpret_cast<const float*>(a.w.scales);
  return from[min(row, (u64)a.w.n - 1)];
}
__device__ __forceinline__ float first_sum(const MxSearchArgs& a, u64 row, float norm) {
  return row >= a.w.n ? -__builtin_inff() : a.norms ? -0.5f * norm : 0.0f;
}
// of four rows from row0 + 4 (lane / 16) on, from the lanes that hold the norms of row0 + lane % 16
__device__ __forceinline__ v4f first_sums(const MxSearchArgs& a, u64 row0, float norm) {
  const u32 lane = threadIdx.x % 64;
  const float mine = first_sum(a, row0 + lane % 16, norm);
  const int from = (int)(lane / 16 * 4);
  return v4f{__shfl(mine, from), __shfl(mine, from + 1), __shfl(mine, from + 2), __shfl(mine, from + 3)};
}

__device__ __forceinline__ float most_of(float m, v4f v) {
  return __builtin_fmaxf(__builtin_fmaxf(__builtin_fmaxf(__builtin_fmaxf(m, v[0]), v[1]), v[2]), v[3]);
}

// The maxima of four columns groups over the four lanes that share a column: lane l gets the one of group
// ((l / 32) | (l / 16 % 2 * 2)), column l % 16.
__device__ __forceinline__ float join_four(float m0, float m1, float m2, float m3) {
  using v2u = u32 __attribute__((ext_vector_type(2)));
  auto both = [](auto p) {
    const v2u v = __builtin_bit_cast(v2u, p);
    return __builtin_fmaxf(__uint_as_float(v.x), __uint_as_float(v.y));
  };
  const float a = both(__builtin_amdgcn_permlane32_swap(__float_as_uint(m0), __float_as_uint(m1), false, false));
  const float b = both(__builtin_amdgcn_permlane32_swap(__float_as_uint(m2), __float_as_uint(m3), false, false));
  return both(__builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false));
}
__device__ __forceinline__ u32 joined_group(u32 lane) { return lane / 32 | lane / 16 % 2 * 2; }

// The queries' fragments, held by a wave for good; the scales of a query's steps share a register.
template <int STEPS, int QF>
struct Queries {
  v4i codes[QF][STEPS];
  int scales[QF];
  __device__ __forceinline__ void load(const MxSearchArgs& a, u64 first) {
#pragma unroll
    for (int j = 0; j < QF; ++j) {
      const u64 row = a.q0 + min(first + 16 * j + threadIdx.x % 16, (u64)a.nq - 1);
      u32 b = 0;
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        codes[j][s] = load_codes(a.q, row, s);
        b |= (u32)load_scale(a.q, row, s) << (8 * s);
      }
      scales[j] = (int)b;
    }
  }
};

template <int BYTE>
__device__ __forceinline__ v4f mx_mfma_byte(v4i a, v4i b, v4f c, int scale_a, int scale_b) {
  const v8i x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, BYTE, scale_a, BYTE, scale_b);
}
template <int STEPS, int QF, int S = 0>
__device__ __forceinline__ void score_tile(const v4i (&w)[STEPS], int scales, const Queries<STEPS, QF>& q, v4f first, v4f (&acc)[QF]) {
#pragma unroll
  for (int j = 0; j < QF; ++j) acc[j] = mx_mfma_byte<S>(w[S], q.codes[j][S], S == 0 ? first : acc[j], scales, q.scales[j]);
  if constexpr (S + 1 < STEPS) score_tile<STEPS, QF, S + 1>(w, scales, q, first, acc);
}

// Up to 16 QF queries: every wave scores groups of its own, whose rows it asks for one group ahead.  Bound by the
// memory that the rows come from: a million rows of 128 take 14.6 us, 4.9 TB/s.
template <int STEPS, int QF>
__global__ __launch_bounds__(256) void mx_group_few_kernel(MxSearchArgs a) {
  const u32 lane = threadIdx.x % 64;
  const u32 waves = gridDim.x * 4;
  u32 g = blockIdx.x * 4 + threadIdx.x / 64;
  Queries<STEPS, QF> q;
  q.load(a, 0);
  struct Ahead {
    v4i w[4][STEPS];
    u32 b[4][STEPS];
    float norm[4];
  } next;
  auto ask = [&](u32 group) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u64 row0 = (u64)group * SEARCH_GROUP + 16 * i;
      const u64 row = min(row0 + lane % 16, (u64)a.w.n - 1);
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        next.w[i][s] = load_codes(a.w, row, s);
        next.b[i][s] = reinterpret_cast<const u32*>(a.w.scales)[row * a.w.steps + s];
      }
      next.norm[i] = load_norm(a, row);
    }
  };
  if (g < a.groups) ask(g);
  for (; g < a.groups; g += waves) {
    const Ahead now = next;
    ask(min(g + waves, a.groups - 1));
    float m[4] = {-__builtin_inff(), -__builtin_inff(), -__builtin_inff(), -__builtin_inff()};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32 scales = 0;
#pragma unroll
      for (int s = 0; s < STEPS; ++s) scales |= (now.b[i][s] >> (lane / 16 * 8) & 255) << (8 * s);
      v4f acc[QF];
      score_tile<STEPS, QF>(now.w[i], (int)scales, q, first_sums(a, (u64)g * SEARCH_GROUP + 16 * i, now.norm[i]), acc);
#pragma unroll
      for (int j = 0; j < QF; ++j) m[j] = most_of(m[j], acc[j]);
    }
    const float joined = join_four(m[0], m[1], m[2], m[3]);
    const u32 x = joined_group(lane) * 16 + lane % 16;
    if (x < a.nq) a.most[(u64)x * a.pitch + g] = joined;
  }
}

// Many queries: eight waves, WR of which share the 16 QF queries they hold and take groups in turn; all rows pass
// through LDS, in stages of four groups (two where rows are long), laid out as the fragments are read.  Bound by the
// matrix cores: beside a product of 16 x 16 scores and 128 elements stand two instructions that take its maximum.
// 10,000 queries on a million rows of two steps take 1,057 us, 4.8 PFLOP/s, the matrix cores at work 66 % of the time.
constexpr u32 SEARCH_THREADS = 512;
template <int STEPS>
constexpr u32 stage_groups() {
  return STEPS <= 2 ? 4 : 2;
}

template <int STEPS, int QF, int WR>
__global__ __launch_bounds__(SEARCH_THREADS) void mx_group_many_kernel(MxSearchArgs a, u32 blocks_q, u32 ranges) {
  constexpr u32 GS = stage_groups<STEPS>(), ROWS = GS * SEARCH_GROUP, TILES = ROWS / 16;
  constexpr u32 LOADS = ROWS * STEPS * MX_STEP_BYTES / 16 / SEARCH_THREADS;
  constexpr u32 SCALES = (ROWS * STEPS + SEARCH_THREADS - 1) / SEARCH_THREADS;
  struct Stage {
    v4i codes[TILES * STEPS][64];
    u32 scales[TILES][64];
    float first[ROWS];
  };
  extern __shared__ __align__(16) char lds[];
  Stage* stages = reinterpret_cast<Stage*>(lds);
  const u32 tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  // Chiplets take workgroups in turn: each gets a run of them that read the same rows.
  const u32 all = blocks_q * ranges, per = (all + 7) / 8, t = blockIdx.x % 8 * per + blockIdx.x / 8;
  if (t >= all) return;
  const u32 range = t / blocks_q;
  const u32 total = (a.groups + GS - 1) / GS;  // stages
  const u32 s0 = (u32)((u64)total * range / ranges), s1 = (u32)((u64)total * (range + 1) / ranges);
  const u64 x0 = (u64)(t % blocks_q) * (8 / WR * 16 * QF) + wave / WR * (16 * QF);
  Queries<STEPS, QF> q;
  q.load(a, x0);

  v4i next_w[LOADS];
  u32 next_scale[SCALES];
  float next_norm = 0.0f;
  u64 next_row = 0;
  auto fetch = [&](u32 stage) {
    const u64 row0 = (u64)stage * ROWS;
#pragma unroll
    for (u32 i = 0; i < LOADS; ++i) {
      const u32 at = i * SEARCH_THREADS + tid, frag = at / 64, r = frag / STEPS * 16 + at % 16;
      next_w[i] = *reinterpret_cast<const v4i*>(a.w.codes + (min(row0 + r, (u64)a.w.n - 1) * STEPS + frag % STEPS) * MX_STEP_BYTES + at / 16 % 4 * 16);
    }
#pragma unroll
    for (u32 i = 0; i < SCALES; ++i) {
      const u32 at = min(i * SEARCH_THREADS + tid, ROWS * STEPS - 1);
      next_scale[i] = reinterpret_cast<const u32*>(a.w.scales)[min(row0 * STEPS + at, (u64)a.w.n * STEPS - 1)];
    }
    next_row = row0 + tid % ROWS;
    next_norm = load_norm(a, next_row);
  };
  auto keep = [&](Stage& to) {
#pragma unroll
    for (u32 i = 0; i < LOADS; ++i) (&to.codes[0][0])[i * SEARCH_THREADS + tid] = next_w[i];
#pragma unroll
    for (u32 i = 0; i < SCALES; ++i) {
      const u32 at = i * SEARCH_THREADS + tid, r = at / STEPS, s = at % STEPS;
      if (at < ROWS * STEPS)
#pragma unroll
        for (u32 g = 0; g < 4; ++g) reinterpret_cast<uint8_t*>(&to.scales[r / 16][g * 16 + r % 16])[s] = (uint8_t)(next_scale[i] >> (8 * g));
    }
    if (tid < ROWS) to.first[tid] = first_sum(a, next_row, next_norm);
  };
  fetch(s0);
  keep(stages[s0 % 2]);
  fetch(min(s0 + 1, s1 - 1));
  for (u32 st = s0; st < s1; ++st) {
    __syncthreads();
    const Stage& here = stages[st % 2];
    float joined[GS / WR][QF / 4];
#pragma unroll
    for (u32 n = 0; n < GS / WR; ++n) {
      if (n == 1 || GS == WR) {
        // Behind the first products.  At the end a stage too many is put away, and not read: at a condition the
        // compiler would move the products behind it.
        keep(stages[(st + 1) % 2]);
        fetch(min(st + 2, s1 - 1));
      }
      const u32 g = n * WR + wave % WR;
      float m[QF];
#pragma unroll
      for (int j = 0; j < QF; ++j) m[j] = -__builtin_inff();
#pragma unroll
      for (u32 i = 0; i < 4; ++i) {
        v4i w[STEPS];
#pragma unroll
        for (u32 s = 0; s < STEPS; ++s) w[s] = here.codes[(g * 4 + i) * STEPS + s][lane];
        v4f acc[QF];
        score_tile<STEPS, QF>(w, (int)here.scales[g * 4 + i][lane], q, *reinterpret_cast<const v4f*>(&here.first[(g * 4 + i) * 16 + lane / 16 * 4]), acc);
#pragma unroll
        for (int j = 0; j < QF; ++j) m[j] = most_of(m[j], acc[j]);
      }
#pragma unroll
      for (int j = 0; j < QF; j += 4) joined[n][j / 4] = join_four(m[j], m[j + 1], m[j + 2], m[j + 3]);
    }
#pragma unroll
    for (int j = 0; j < QF / 4; ++j) {
      const u64 x = x0 + 64 * j + joined_group(lane) * 16 + lane % 16;
      if (x >= a.nq) continue;
      float* to = a.most + x * a.pitch + (u64)st * GS;  // (the pitch has room for a whole last stage)
      if constexpr (WR == 1) {
        float m = joined[0][j];
#pragma unroll
        for (u32 n = 1; n < GS; ++n) m = __builtin_fmaxf(m, joined[n][j]);
        a.coarse[x * a.coarse_pitch + st] = m;
      }
      if constexpr (WR == 1 && GS == 4)
        *reinterpret_cast<v4f*>(to) = v4f{joined[0][j], joined[1][j], joined[2][j], joined[3][j]};
      else
#pragma unroll
        for (u32 n = 0; n < GS / WR; ++n) to[n * WR + wave % WR] = joined[n][j];
    }
  }
}

// Rows of more steps: a wave scores 64 rows (a group) and 64 queries, step by step from memory, with no step on its way ahead
// and no LDS.  One query of a million rows of 768 and 1,024 takes 146 and 211 us with its picking (their bytes 84 and 111 at a
// copy's rate; 66 for 512 elements, by the kernel of few queries), ten thousand 20 and 36 ms (4.1 for 512).
__global__ __launch_bounds__(256) void mx_group_long_kernel(MxSearchArgs a, u64 tiles) {
  const u32 lane = threadIdx.x % 64;
  const u64 t = (u64)blockIdx.x * 4 + threadIdx.x / 64;
  if (t >= tiles) return;
  const u64 g = t % a.groups, w0 = g * SEARCH_GROUP;
  const u64 x0 = t / a.groups * 64;
  v4f acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const v4f c = first_sums(a, w0 + 16 * i, load_norm(a, w0 + 16 * i + lane % 16));
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = c;
  }
  for (u32 s = 0; s < a.w.steps; ++s) {
    v4i w[4], x[4];
    int ws[4], xs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u64 wr = min(w0 + 16 * i + lane % 16, (u64)a.w.n - 1), xr = a.q0 + min(x0 + 16 * i + lane % 16, (u64)a.nq - 1);
      w[i] = load_codes(a.w, wr, s);
      ws[i] = load_scale(a.w, wr, s);
      x[i] = load_codes(a.q, xr, s);
      xs[i] = load_scale(a.q, xr, s);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = mx_mfma(w[i], x[j], acc[i][j], ws[i], xs[j]);
  }
  float m[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m[j] = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 4; ++i) m[j] = most_of(m[j], acc[i][j]);
  }
  const float joined = join_four(m[0], m[1], m[2], m[3]);
  const u64 x = x0 + joined_group(lane) * 16 + lane % 16;
  if (x < a.nq) a.most[x * a.pitch + g] = joined;
}

// A workgroup per query.  The k-th largest of its threads' maxima over the groups is a bound that k groups at least
// reach; the few that do are ranked, the first k scored again, and the k best points ranked.  For one query of a million
// rows 10 us, a chain of trips to memory and barriers; for 10,000 queries 282 us, vector instructions.
constexpr u32 PICK_BOUNDS = 256;  // maxima, of one or four threads each, of which the k-th largest is the bound
constexpr u32 PICK_FEW = 512;  // candidates that are ranked by counting the ones before each

struct PickLds {
  u32 hist[PICK_BOUNDS];
  u32 chosen[SEARCH_MOST_K];
  u32 prefix, left, count, bound, scan[16];
};

// The first k of `count` maxima by (size downwards, place), by a radix selection of the k-th largest key: where too
// many reach the bound below (equal maxima).
template <u32 THREADS>
__device__ void choose_equal(const float* most, u32 count, u32 k, u32 least, PickLds& s) {
  const u32 tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  if (tid == 0) s.prefix = 0, s.left = min(k, count), s.count = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) s.hist[tid] = 0;
    __syncthreads();
    const u32 prefix = s.prefix;
    for (u32 i = tid; i < count; i += THREADS) {
      const u32 key = float_key(most[i]);
      if (shift == 24 || key >> (shift + 8) == prefix) atomicAdd(&s.hist[key >> shift & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      u32 left = s.left, b = 255;
      while (b > 0 && s.hist[b] < left) left -= s.hist[b--];
      s.left = left;
      s.prefix = prefix << 8 | b;
    }
    __syncthreads();
  }
  const u32 cut = s.prefix, ties = s.left;  // maxima above the cut, and the first `ties` of those at it
  __syncthreads();
  if (tid == 0) s.left = 0, s.bound = cut;
  __syncthreads();
  // in the order of places, so that the ties taken are the first ones
  for (u32 i0 = 0; i0 < count; i0 += THREADS) {
    const u32 i = i0 + tid;
    const u32 key = i < count ? float_key(most[i]) : 0u;
    const bool tie = key == cut && key > least;
    const u64 votes = __ballot(tie);
    if (lane == 0) s.scan[wave] = (u32)__popcll(votes);
    __syncthreads();
    u32 before = s.left + (u32)__popcll(votes & ((1ull << lane) - 1));
    for (u32 w = 0; w < wave; ++w) before += s.scan[w];
    if (i < count && ((key > cut && key > least) || (tie && before < ties))) s.chosen[atomicAdd(&s.count, 1u)] = i;
    __syncthreads();
    if (tid == 0)
      for (u32 w = 0; w < THREADS / 64; ++w) s.left += s.scan[w];
    __syncthreads();
  }
}

// found[0 .. count): keys and places; the first k of them into s.chosen, the k-th key into s.bound
template <u32 THREADS>
__device__ __forceinline__ void choose_ranked(const u64* found, u32 count, u32 k, PickLds& s) {
  for (u32 c = threadIdx.x; c < count; c += THREADS) {
    const u64 key = found[c];
    u32 rank = 0;
    for (u32 i = 0; i < count; ++i) rank += found[i] < key;
    if (rank < k) s.chosen[rank] = (u32)key;
    if (rank == k - 1) s.bound = ~(u32)(key >> 32);
  }
  if (threadIdx.x == 0) s.count = min(count, k);
  __syncthreads();
}

// The first k of `count` maxima (16-byte aligned) by (size downwards, place): s.count of them in s.chosen; where that
// is k, s.bound is the last one's key.
template <u32 THREADS>
__device__ void choose(const float* most, u32 count, u32 k, u32 least, u64* found, PickLds& s) {
  constexpr u32 AHEAD = THREADS == 256 ? 8 : 4, SHARE = THREADS / PICK_BOUNDS;
  const u32 tid = threadIdx.x, fours = (count + 3) / 4;
  const v4f* all = reinterpret_cast<const v4f*>(most);
  v4f x[AHEAD];
  auto ask = [&](u32 at) {
#pragma unroll
    for (u32 u = 0; u < AHEAD; ++u) x[u] = all[min(at + u * THREADS + tid, fours - 1)];
  };
  // (the places past the last are none; a maximum read twice does no harm)
  auto value = [&](u32 at, u32 u, u32 e) { return (at + u * THREADS + tid) * 4 + e < count ? x[u][e] : -__builtin_inff(); };
  float m = -__builtin_inff();
  for (u32 at = 0; at < fours; at += AHEAD * THREADS) {
    ask(at);
#pragma unroll
    for (u32 u = 0; u < AHEAD; ++u)
#pragma unroll
      for (u32 e = 0; e < 4; ++e) m = __builtin_fmaxf(m, value(at, u, e));
  }
#pragma unroll
  for (u32 v = 1; v < SHARE; v *= 2) m = __builtin_fmaxf(m, __shfl_xor(m, (int)v));
  const u32 mine = float_key(m), place = tid / SHARE;
  if (tid % SHARE == 0) s.hist[place] = mine;
  if (tid == 0) s.count = 0;
  __syncthreads();
  // (the threads that share a maximum rank it against a part of the others each)
  u32 before = 0;
#pragma unroll 4
  for (u32 i = tid % SHARE * 4; i < PICK_BOUNDS; i += SHARE * 4) {
    using v4u = u32 __attribute__((ext_vector_type(4)));
    const v4u h = *reinterpret_cast<const v4u*>(&s.hist[i]);
#pragma unroll
    for (u32 e = 0; e < 4; ++e) before += h[e] > mine || (h[e] == mine && i + e < place);
  }
#pragma unroll
  for (u32 v = 1; v < SHARE; v *= 2) before += (u32)__shfl_xor((int)before, (int)v);
  if (before == k - 1) s.bound = max(mine, least + 1);
  __syncthreads();
  const u32 bound = s.bound;
  const float at_least = key_float(bound);
  for (u32 at = 0; at < fours; at += AHEAD * THREADS) {
    if (fours > AHEAD * THREADS) ask(at);  // (else they are all here)
#pragma unroll
    for (u32 u = 0; u < AHEAD; ++u)
#pragma unroll
      for (u32 e = 0; e < 4; ++e)
        if (value(at, u, e) >= at_least) {
          const u32 to = atomicAdd(&s.count, 1u);
          if (to < PICK_FEW) found[to] = (u64)~float_key(x[u][e]) << 32 | ((at + u * THREADS + tid) * 4 + e);
        }
  }
  __syncthreads();
  const u32 reached = s.count;
  __syncthreads();
  if (reached <= PICK_FEW)
    choose_ranked<THREADS>(found, reached, k, s);
  else
    choose_equal<THREADS>(most, count, k, least, s);
}

template <u32 THREADS>
__global__ __launch_bounds__(THREADS, 4) void mx_pick_kernel(MxSearchArgs a) {
  extern __shared__ u64 found[];  // as many as the rows of k groups, up to a power of two for the sort
  __shared__ __align__(16) PickLds s;
  const u32 tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const u32 q = blockIdx.x;
  const float* most = a.most + (u64)q * a.pitch;
  const u32 least = float_key(-__builtin_inff());  // keys up to this one are of groups without a score

  if (a.coarse) {  // the first k groups are in the first k groups of groups
    choose<THREADS>(a.coarse + (u64)q * a.coarse_pitch, (a.groups + a.per_coarse - 1) / a.per_coarse, a.k, least, found, s);
    const u32 parts = s.count * a.per_coarse;
    __syncthreads();
    if (tid == 0) s.count = 0;
    __syncthreads();
    for (u32 i = tid; i < parts; i += THREADS) {
      const u32 g = s.chosen[i / a.per_coarse] * a.per_coarse + i % a.per_coarse;
      const u32 key = g < a.groups ? float_key(most[g]) : 0u;
      if (key > least) found[atomicAdd(&s.count, 1u)] = (u64)~key << 32 | g;
    }
    __syncthreads();
    const u32 reached = s.count;
    __syncthreads();
    choose_ranked<THREADS>(found, reached, a.k, s);
  } else {
    choose<THREADS>(most, a.groups, a.k, least, found, s);
  }
  const u32 nchosen = s.count;
  // k groups: k points reach the smallest of their maxima, and no other point matters
  const u32 low = nchosen == a.k ? max(s.bound, least + 1) : least + 1;
  __syncthreads();
  if (tid == 0) s.count = 0;
  __syncthreads();
  const u64 qrow = (u64)a.q0 + q;
  for (u32 c = wave; c < nchosen; c += THREADS / 64) {
    const u64 w0 = (u64)s.chosen[c] * SEARCH_GROUP;
    v4f acc[4];
    u64 row[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      row[i] = min(w0 + 16 * i + lane % 16, (u64)a.w.n - 1);
      acc[i] = first_sums(a, w0 + 16 * i, load_norm(a, w0 + 16 * i + lane % 16));
    }
    for (u32 st = 0; st < a.w.steps; st += 2) {  // two steps' loads on their way at once
      v4i x[2], w[4][2];
      int xs[2], ws[4][2];
#pragma unroll
      for (u32 e = 0; e < 2; ++e) {
        const u32 step = min(st + e, a.w.steps - 1);
        x[e] = load_codes(a.q, qrow, step);
        xs[e] = load_scale(a.q, qrow, step);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i][e] = load_codes(a.w, row[i], step), ws[i][e] = load_scale(a.w, row[i], step);
      }
#pragma unroll
      for (u32 e = 0; e < 2; ++e) {
        if (st + e >= a.w.steps) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = mx_mfma(w[i][e], x[e], acc[i], ws[i][e], xs[e]);
      }
    }
    // (all columns are this query's: one of them is used)
    if (lane % 16 == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const u64 id = w0 + 16 * i + lane / 16 * 4 + r;
          const u32 key = float_key(acc[i][r]);
          if (id < a.w.n && key >= low) found[atomicAdd(&s.count, 1u)] = (u64)~key << 32 | id;
        }
  }
  __syncthreads();
  const u32 count = s.count;
  auto put = [&](u32 at, u64 key) {
    const u64 to = qrow * a.k + at;
    const float score = key_float(~(u32)(key >> 32));
    const float dist = a.norms ? __builtin_fmaf(-2.0f, score, a.qnorms[qrow]) : 0.0f - score;
    // (|q|^2, or the distance, beyond fp32: distances grow with the place, so that none behind it is finite either)
    const bool fine = dist < __builtin_inff();
    a.ids[to] = fine ? (u32)key : ANN_NONE;
    a.dists[to] = !fine ? __builtin_inff() : a.norms ? __builtin_fmaxf(0.0f, dist) : dist;
  };
  if (count <= PICK_FEW) {
    for (u32 c = tid; c < count; c += THREADS) {
      const u64 key = found[c];
      u32 rank = 0;
      for (u32 i = 0; i < count; ++i) rank += found[i] < key;
      if (rank < a.k) put(rank, key);
    }
  } else {
    u32 size = 2;
    while (size < count) size *= 2;
    for (u32 i = count + tid; i < size; i += THREADS) found[i] = ~0ull;
    __syncthreads();
    for (u32 run = 2; run <= size; run *= 2)
      for (u32 gap = run / 2; gap > 0; gap /= 2) {
        for (u32 i = tid; i < size / 2; i += THREADS) {
          const u32 lo = i / gap * 2 * gap + i % gap, hi = lo + gap;
          const u64 x = found[lo], y = found[hi];
          if ((x > y) == ((lo & run) == 0)) found[lo] = y, found[hi] = x;
        }
        __syncthreads();
      }
    for (u32 i = tid; i < a.k; i += THREADS) put(i, found[i]);
  }
  for (u32 i = count + tid; i < a.k; i += THREADS) {
    a.ids[qrow * a.k + i] = ANN_NONE;
    a.dists[qrow * a.k + i] = __builtin_inff();
  }
}

template <int STEPS>
hipError_t launch_groups(MxSearchArgs& a, hipStream_t s) {
  if (a.nq <= 64) {
    a.coarse = nullptr;
    const u32 blocks = (a.groups + 3) / 4;
    const dim3 grid(blocks < 1024 ? blocks : 1024);
    if (a.nq <= 16)
      hipLaunchKernelGGL((mx_group_few_kernel<STEPS, 1>), grid, dim3(256), 0, s, a);
    else if (a.nq <= 32)
      hipLaunchKernelGGL((mx_group_few_kernel<STEPS, 2>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((mx_group_few_kernel<STEPS, 4>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
  }
  constexpr int QF = STEPS <= 2 ? 8 : 4;
  constexpr u32 GS = stage_groups<STEPS>(), ROWS = GS * SEARCH_GROUP;
  constexpr u32 lds = 2 * (ROWS * STEPS * MX_STEP_BYTES + ROWS * 4 * 4 + ROWS * 4);
  // waves that hold the same queries, where there are too few for all eight
  const bool shared = a.nq <= 16 * QF * 8 / GS;
  const u32 per = 16 * QF * 8 / (shared ? GS : 1), blocks_q = (a.nq + per - 1) / per;
  const u32 total = (a.groups + GS - 1) / GS;
  // A compute unit holds one workgroup: as many ranges as make whole turns of 256 workgroups, or nearly.  (260 of them
  // take twice as long as 250.)
  u32 ranges = blocks_q < 256 ? 256 / blocks_q : 1;
  for (u32 r = ranges, best = 0; r <= total && r <= 8 * ranges && best < 95; ++r) {
    const u64 groups_of = (u64)blocks_q * r, full = 100 * groups_of / ((groups_of + 255) / 256 * 256);
    if (full > best) best = (u32)full, ranges = r;
  }
  if (ranges > total) ranges = total;
  const auto kernel = shared ? mx_group_many_kernel<STEPS, QF, GS> : mx_group_many_kernel<STEPS, QF, 1>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  if (shared) a.coarse = nullptr;
  a.per_coarse = GS;
  hipLaunchKernelGGL(kernel, dim3((blocks_q * ranges + 7) / 8 * 8), dim3(SEARCH_THREADS), lds, s, a, blocks_q, ranges);
  return hipGetLastError();
}

constexpr u64 search_pitch(u64 n) { return (n + 4 * SEARCH_GROUP - 1) / (4 * SEARCH_GROUP) * 4; }  // whole stages of groups

// the largest of the maxima of a stage, kept apart by launches of many queries (a stage has two groups at least)
constexpr u64 search_coarse_pitch(u64 n) { return (search_pitch(n) / 2 + 3) / 4 * 4; }

u64 search_queries_at_once(u64 pitch, u64 nq) {
  u64 most = SEARCH_SCRATCH_FLOATS / pitch / 64 * 64;
  if (most < 64) most = 64;
  if (most > SEARCH_MOST_AT_ONCE) most = SEARCH_MOST_AT_ONCE;
  return nq < most ? nq : most;
}

int check_search(u64 n, u32 d, u64 nq, u32 k) {
  if (n > MX_MOST_ROWS || nq > MX_MOST_ROWS) return fail(ANN_EINVAL, "ann_mx_search: rows must stay below 2^31");
  if (d < 1 || d > MX_MOST_D) return fail(ANN_EINVAL, "ann_mx_search: d must be 1 to %u", MX_MOST_D);
  if (k < 1 || k > SEARCH_MOST_K) return fail(ANN_EINVAL, "ann_mx_search: k must be 1 to %u", SEARCH_MOST_K);
  return ANN_OK;
}

u64 search_scratch(u64 n, u64 nq) {
  const u64 pitch = search_pitch(n);
  return pitch == 0 ? 0 : search_queries_at_once(pitch, nq) * (pitch + search_coarse_pitch(n)) * 4;
}

__global__ void mx_none_kernel(u32* ids, float* dists, u64 count) {
  for (u64 i = (u64)blockIdx.x * 256 + threadIdx.x; i < count; i += (u64)gridDim.x * 256) {
    ids[i] = ANN_NONE;
    dists[i] = __builtin_inff();
  }
}

}  // namespace annmi

using namespace annmi;

extern "C" {

int ann_mx_search_scratch(uint64_t n, uint32_t d, uint64_t nq, uint32_t k, uint64_t* bytes) try {
  if (!bytes) return fail(ANN_EINVAL, "null argument");
  int rc = check_search(n, d, nq, k);
  if (rc) return rc;
  *bytes = search_scratch(n, nq);
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

int ann_mx_search(const uint8_t* codes_dev, const uint8_t* scales_dev, const float* norms_dev, uint64_t n, uint32_t d,
                  ann_metric metric, const uint8_t* qcodes_dev, const uint8_t* qscales_dev, const float* qnorms_dev,
                  uint64_t nq, uint32_t k, uint32_t* ids_dev, float* dists_dev, void* scratch_dev, uint64_t scratch_bytes,
                  void* stream) try {
  if (metric != ANN_L2SQ && metric != ANN_MIPS) return fail(ANN_EINVAL, "unknown metric");
  int rc = check_search(n, d, nq, k);
  if (rc) return rc;
  rc = check_mx_rows("ann_mx_search", codes_dev, scales_dev, n, d);
  if (rc) return rc;
  rc = check_mx_rows("ann_mx_search", qcodes_dev, qscales_dev, nq, d);
  if (rc) return rc;
  if (nq == 0) return ANN_OK;
  if (!ids_dev || !dists_dev) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(ids_dev, 4) || !aligned_to(dists_dev, 4)) return fail(ANN_EINVAL, "outputs not aligned to their elements");
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (n == 0) {
    hipLaunchKernelGGL(mx_none_kernel, dim3(1024), dim3(256), 0, st, ids_dev, dists_dev, nq * k);
    HIP_TRY(hipGetLastError());
    return ANN_OK;
  }
  if (metric == ANN_L2SQ && (!norms_dev || !qnorms_dev))
    return fail(ANN_EINVAL, "squared distances need the norms of rows and queries (norms_dev of ann_mx_quantize)");
  if (metric == ANN_L2SQ && (!aligned_to(norms_dev, 4) || !aligned_to(qnorms_dev, 4)))
    return fail(ANN_EINVAL, "norms not aligned to their elements");
  if (!scratch_dev || !aligned_to(scratch_dev, 16) || scratch_bytes < search_scratch(n, nq))
    return fail(ANN_EINVAL, "scratch: %llu bytes are needed, 16-byte aligned (ann_mx_search_scratch)",
                (unsigned long long)search_scratch(n, nq));
  MxSearchArgs a{};
  a.w = {codes_dev, scales_dev, (u32)n, mx_steps(d)};
  a.q = {qcodes_dev, qscales_dev, (u32)nq, mx_steps(d)};
  a.norms = metric == ANN_L2SQ ? norms_dev : nullptr;
  a.qnorms = qnorms_dev;
  a.groups = (u32)((n + SEARCH_GROUP - 1) / SEARCH_GROUP);
  a.k = k;
  a.most = static_cast<float*>(scratch_dev);
  a.ids = ids_dev;
  a.dists = dists_dev;
  a.pitch = (u32)search_pitch(n);
  const u64 part = search_queries_at_once(a.pitch, nq);
  size_t room = PICK_FEW;  // (four groups of each of the first k groups of groups as well)
  while (room < (size_t)(k < a.groups ? k : a.groups) * SEARCH_GROUP) room *= 2;
  room *= 8;
  // A thousand threads for a query where there are not enough queries for all compute units: with the scoring, of a million
  // rows of 128, 1, 64 and 256 queries take 25 us against 39 with 256 threads, 29 against 43, 49 against 61; 1,000 queries
  // 164 against 153, and of 20,000 rows 55 against 35.
  const auto pick = part <= 256 ? mx_pick_kernel<1024> : mx_pick_kernel<256>;
  const u32 pick_threads = part <= 256 ? 1024 : 256;
  HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(pick), hipFuncAttributeMaxDynamicSharedMemorySize, (int)room));
  for (u64 q0 = 0; q0 < nq; q0 += part) {
    a.q0 = (u32)q0;
    a.nq = (u32)(nq - q0 < part ? nq - q0 : part);
    a.coarse = a.most + part * a.pitch;
    a.coarse_pitch = (u32)search_coarse_pitch(n);
    if (a.w.steps == 1) {
      HIP_TRY(launch_groups<1>(a, st));
    } else if (a.w.steps == 2) {
      HIP_TRY(launch_groups<2>(a, st));
    } else if (a.w.steps == 3) {
      HIP_TRY(launch_groups<3>(a, st));
    } else if (a.w.steps == 4) {
      HIP_TRY(launch_groups<4>(a, st));
    } else {
      const u64 tiles = a.groups * (((u64)a.nq + 63) / 64);
      a.coarse = nullptr;
      hipLaunchKernelGGL(mx_group_long_kernel, dim3((u32)((tiles + 3) / 4)), dim3(256), 0, st, a, tiles);
      HIP_TRY(hipGetLastError());
    }
    hipLaunchKernelGGL(pick, dim3(a.nq), dim3(pick_threads), room, st, a);
    HIP_TRY(hipGetLastError());
  }
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

}  // extern "C"
