// Beam search: the best continuations of each group of beams, and the states of a decoder in the order of the beams that go on.
//
// The continuation of beam b by entry j is worth total_b + log q, q = softmax of the beam's scores at j.  Within a beam
// that order is the scores' own, so that a part of a row need hand on no more than its k best scores, beside its largest
// score and the sum of exp relative to it: one pass over the scores.  Beams are compared by their log sums, in 64 bits: the
// order is that of the real numbers but where two differ by less than some 1e-12.
#include <algorithm>

#include "mx.hpp"

namespace annmi {

constexpr u32 BEAM_MOST_BEAMS = 64;
constexpr u32 BEAM_MOST_K = 128;
constexpr u32 BEAM_MOST_N = (1u << 24) - 1;  // an id, a score and a beam fit in one key of 64 bits
constexpr u32 BEAM_THREADS = 256;
constexpr u32 BEAM_EACH = 16;  // entries of a thread
constexpr u32 BEAM_CHUNK = BEAM_THREADS * BEAM_EACH;
constexpr u32 BEAM_LIST = 1024;  // entries of a chunk that are brought into order

struct BeamArgs {
  const char* scores;
  u64 groups;
  u32 beams, n, k;
  u64 ld;
  const float* totals;
  const uint8_t* finished;
  u32 pad;
  u32 chunks;  // of a row
  u64* best;   // for each chunk its k best: score key << 32 | ~id, downwards, 0 where there are fewer
  double* sums;
  float* most;
  u32* parents;
  u32* ids;
  float* out;
};

// exp x for x <= 0, within 1.1e-12 of itself; 1e-304 for all that is below -700, and for NaN.  2^n times 2^f, |f| <= 1/2,
// by the polynomial that has its values at the nine Chebyshev points of that range.  Adding 1.5 * 2^52 leaves n in the low
// bits of the sum.
__device__ __forceinline__ double beam_exp(double x) {
  constexpr double MAGIC = 6755399441055744.0, LOG2E = 1.4426950408889634074;
  const double d = __builtin_fmax(x, -700.0) * LOG2E, t = d + MAGIC, f = d - (t - MAGIC);
  double p = 0x1.63d136366db24p-20;
  p = __builtin_fma(p, f, 0x1.00dc4a532fb8ep-16);
  p = __builtin_fma(p, f, 0x1.4308ac85aa947p-13);
  p = __builtin_fma(p, f, 0x1.5d8745a728441p-10);
  p = __builtin_fma(p, f, 0x1.3b2ab7181b755p-7);
  p = __builtin_fma(p, f, 0x1.c6b08dd6fd234p-5);
  p = __builtin_fma(p, f, 0x1.ebfbdff823cedp-3);
  p = __builtin_fma(p, f, 0x1.62e42fef84cf0p-1);
  p = __builtin_fma(p, f, 1.0);
  return __hiloint2double(__double2hiint(p) + ((int)__double_as_longlong(t) << 20), __double2loint(p));
}
// z - most, 0 among infinities
__device__ __forceinline__ double beam_below(float z, float most) { return z == most ? 0.0 : (double)z - most; }

// whether a beam goes on by its scores
__device__ __forceinline__ bool beam_lives(const BeamArgs& a, u64 row) {
  const float total = a.totals[row];
  return total > -INFINITY && !(a.finished && a.finished[row]);
}

// Sorts the first `count` keys downwards, in room for the next power of two; the whole workgroup.
template <u32 THREADS, typename Swap>
__device__ __forceinline__ void sort_down(u32 size, Swap swap) {
  for (u32 run = 2; run <= size; run *= 2)
    for (u32 gap = run / 2; gap > 0; gap /= 2) {
      for (u32 i = threadIdx.x; i < size / 2; i += THREADS) {
        const u32 low = i / gap * (2 * gap) + i % gap, high = low + gap;
        swap(low, high, (low & run) == 0);  // (the larger first where true)
      }
      __syncthreads();
    }
}
__device__ __forceinline__ u32 power_of_two(u32 v) { return v <= 1 ? 1 : 1u << (32 - __clz(v - 1)); }

// The largest of a wave, the same in every lane.
template <int CTRL>
__device__ __forceinline__ u32 beam_row_max(u32 v) {
  return max(v, (u32)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ u32 wave_largest(u32 v) {
  v = beam_row_max<0xB1>(v);   // the neighbour
  v = beam_row_max<0x4E>(v);   // two away
  v = beam_row_max<0x124>(v);  // four and eight around in 16 lanes
  v = beam_row_max<0x128>(v);
  return max(max((u32)__builtin_amdgcn_readlane((int)v, 0), (u32)__builtin_amdgcn_readlane((int)v, 16)),
             max((u32)__builtin_amdgcn_readlane((int)v, 32), (u32)__builtin_amdgcn_readlane((int)v, 48)));
}
// The m-th largest of a wave's values, and the largest.
__device__ __forceinline__ u32 wave_mth(u32 v, u32 m, u32* first) {
  u32 best = *first = wave_largest(v);
  for (u32 i = 1; i < m && best; ++i) {
    const u64 holds = __ballot(v == best);
    if (threadIdx.x % 64 == (u32)__builtin_ctzll(holds)) v = 0;  // one of those that hold it
    best = wave_largest(v);
  }
  return best;
}

// how far a thread's i-th entry lies from its first one: pieces of E entries, the workgroup's next to each other
template <u32 E>
__device__ __forceinline__ constexpr u32 beam_step(u32 i) {
  return i / E * (BEAM_THREADS * E) + i % E;
}

// Lists exactly the k best of a chunk that has more: the k-th best's key, of the score and the place in the chunk, is found
// bit by bit by counting.  For chunks of many equal scores.
template <u32 E>
__device__ __forceinline__ u32 beam_exactly(const float (&v)[BEAM_EACH], u32 place, u32 from, u32 k, u64* list, u32 (*counts)[BEAM_THREADS / 64], u32* count) {
  constexpr u32 BITS = 12;  // of the place
  static_assert(BEAM_CHUNK == 1u << BITS);
  u64 least = 0;
  for (int bit = 31 + BITS; bit >= 0; --bit) {
    const u64 tried = least | 1ull << bit;
    u32 mine = 0;
#pragma unroll
    for (u32 i = 0; i < BEAM_EACH; ++i) mine += v[i] > -INFINITY && ((u64)float_key(v[i]) << BITS | (BEAM_CHUNK - 1 - (place + beam_step<E>(i)))) >= tried;
#pragma unroll
    for (int w = 1; w < 64; w *= 2) mine += __shfl_xor(mine, w);
    if (threadIdx.x % 64 == 0) counts[bit % 2][threadIdx.x / 64] = mine;
    __syncthreads();  // (the counts before these are read by then)
    u32 all = 0;
#pragma unroll
    for (u32 w = 0; w < BEAM_THREADS / 64; ++w) all += counts[bit % 2][w];
    if (all >= k) least = tried;
  }
  if (threadIdx.x == 0) *count = 0;
  __syncthreads();
#pragma unroll
  for (u32 i = 0; i < BEAM_EACH; ++i)
    if (v[i] > -INFINITY && ((u64)float_key(v[i]) << BITS | (BEAM_CHUNK - 1 - (place + beam_step<E>(i)))) >= least)
      list[atomicAdd(count, 1u)] = (u64)float_key(v[i]) << 32 | (u32)~(from + place + beam_step<E>(i));
  __syncthreads();
  return *count;
}

// One chunk of a row a workgroup, 16 entries a thread, which stay in registers.  Every wave finds the ceil(k / 4)-th best
// of its threads' best ones; the least of these is a bound that k entries reach at least, and few more in most orders;
// they are listed and brought into order.  (Masks of the lowest number are scores: where so few others are left that
// the masks are the bound beam_exactly makes the list, with 1 % left of the 50,001 in 93 us, with 0.1 % in 192.)  64 groups of 5
// beams of 50,001 fp32 take 24 us, 2.7 TB/s: a wave waits for half of its life, for memory and at the barriers between bound,
// list and order.
template <typename T>
__global__ __launch_bounds__(BEAM_THREADS) void beam_chunk_kernel(BeamArgs a) {
  constexpr u32 E = 16 / sizeof(T), WAVES = BEAM_THREADS / 64;
  __shared__ u64 list[BEAM_LIST];
  __shared__ double sums[BEAM_THREADS];
  __shared__ u32 bounds[WAVES], tops[WAVES], counts[2][WAVES], count;
  const u32 wave = threadIdx.x / 64;
  const u64 tiles = a.groups * a.beams * a.chunks;
  for (u64 b = blockIdx.x; b < tiles; b += gridDim.x) {
    const u64 row = b / a.chunks;
    if (!beam_lives(a, row)) continue;  // (nothing of it is read)
    const u32 from = (u32)(b % a.chunks) * BEAM_CHUNK, there = min(BEAM_CHUNK, a.n - from);
    const T* z = reinterpret_cast<const T*>(a.scores) + row * a.ld + from;
    float v[BEAM_EACH];
    // (where a chunk is not full, all waves have some of it: a wave without entries gives no bound)
    const u32 place = (there < BEAM_CHUNK ? threadIdx.x % 64 * WAVES + wave : threadIdx.x) * E;
#pragma unroll
    for (u32 u = 0; u < BEAM_EACH / E; ++u) {
      const u32 at = place + u * (BEAM_THREADS * E);
      if (at + E <= there) {
        const AnyPack<T, E> in = *reinterpret_cast<const AnyPack<T, E>*>(z + at);
#pragma unroll
        for (u32 e = 0; e < E; ++e) v[u * E + e] = mx_float(static_cast<T>(in.v[e]));
      } else {
#pragma unroll
        for (u32 e = 0; e < E; ++e) v[u * E + e] = at + e < there ? mx_float(z[min(at + e, there - 1)]) : -INFINITY;
      }
    }
    float head = -INFINITY;  // (NaN is no number to fmax)
#pragma unroll
    for (u32 i = 0; i < BEAM_EACH; ++i) head = __builtin_fmaxf(head, v[i]);
    u32 first;
    const u32 mth = wave_mth(head > -INFINITY ? float_key(head) : 0u, (a.k + WAVES - 1) / WAVES, &first);
    __syncthreads();  // (the last turn's readers)
    if (threadIdx.x % 64 == 0) bounds[wave] = mth, tops[wave] = first;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    u32 bound = bounds[0], top = tops[0];
#pragma unroll
    for (u32 w = 1; w < WAVES; ++w) bound = min(bound, bounds[w]), top = max(top, tops[w]);
    const float most = key_float(top);
    if (top == 0) {  // nothing that is not masked
      if (threadIdx.x == 0) a.sums[b] = 0.0, a.most[b] = -INFINITY;
      for (u32 i = threadIdx.x; i < a.k; i += BEAM_THREADS) a.best[b * a.k + i] = 0;
      continue;
    }
    const float least = bound ? key_float(bound) : -__FLT_MAX__;  // (no entry is -inf or NaN)
    u32 mask = 0;
#pragma unroll
    for (u32 i = 0; i < BEAM_EACH; ++i) mask |= (u32)(v[i] >= least) << i;
    if (mask) {
      u32 slot = atomicAdd(&count, (u32)__popc(mask));  // (in any order: the keys differ)
      for (; mask; mask &= mask - 1, ++slot) {
        const u32 at = place + beam_step<E>(__builtin_ctz(mask));
        if (slot < BEAM_LIST) list[slot] = (u64)float_key(mx_float(z[at])) << 32 | (u32)~(from + at);
      }
    }
    double sum = 0.0;
    if (most < INFINITY) {
#pragma unroll
      for (u32 i = 0; i < BEAM_EACH; ++i) sum += beam_exp((double)v[i] - most);  // (as good as 0 for -inf and NaN)
    } else {
#pragma unroll
      for (u32 i = 0; i < BEAM_EACH; ++i) sum += v[i] == most;
    }
    sums[threadIdx.x] = sum;
    __syncthreads();
    u32 listed = count;
    if (wave == WAVES - 1) {  // (the first waves have the list)
      const u32 lane = threadIdx.x % 64;
      double all = 0.0;
#pragma unroll
      for (u32 i = 0; i < BEAM_THREADS / 64; ++i) all += sums[lane + 64 * i];
#pragma unroll
      for (int w = 1; w < 64; w *= 2) all += __shfl_xor(all, w);
      if (lane == 0) a.sums[b] = all, a.most[b] = most;
    }
    if (listed > BEAM_LIST) listed = beam_exactly<E>(v, place, from, a.k, list, counts, &count);
    // an entry's place is how many are larger
    for (u32 mine = threadIdx.x; mine < listed; mine += BEAM_THREADS) {
      const u64 entry = list[mine];
      u32 place = 0;
#pragma unroll 8
      for (u32 i = 0; i < listed; ++i) place += list[i] > entry;
      if (place < a.k) a.best[b * a.k + place] = entry;
    }
    for (u32 i = listed + threadIdx.x; i < a.k; i += BEAM_THREADS) a.best[b * a.k + i] = 0;
  }
}

// A group a workgroup: the beams' log sums, then the chunks' lists, first all their best ones, then all second ones, and so on,
// a thousand at a time.  What is below a bound that k of the first thousand reach, or not better than the k-th so far, is
// left out; when all lists' next ones are, the rest is too.  A chain of barriers and short trips to
// memory: 7 us for one group, 8 for 64.
constexpr u32 PICK_THREADS = 1024, PICK_ROOM = 2048;
__global__ __launch_bounds__(PICK_THREADS) void beam_pick_kernel(BeamArgs a) {
  constexpr u32 WAVES = PICK_THREADS / 64;
  // worth, as a key that is larger for more; and behind it beam, score and id
  __shared__ u64 worth[PICK_ROOM], tie[PICK_ROOM];
  __shared__ double logs[BEAM_MOST_BEAMS];
  __shared__ float mosts[BEAM_MOST_BEAMS], totals[BEAM_MOST_BEAMS];
  __shared__ u32 state[BEAM_MOST_BEAMS];  // 0: no continuation, 1: finished, 2: by its scores
  __shared__ u32 bounds[WAVES], count;
  const u32 lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  auto worth_key = [](double v) {
    const u64 bits = (u64)__double_as_longlong(v + 0.0);
    return bits >> 63 ? ~bits : bits | 1ull << 63;
  };
  // Brings the list into order downwards, as far as the first k; what lies behind its end up to there becomes empty.
  auto order = [&](u32 listed) {
    const u32 mine = threadIdx.x;
    if (listed <= PICK_THREADS) {  // an entry's place is how many are larger
      u64 entry = 0, entry_tie = 0;
      u32 place = mine;
      if (mine < listed) {
        entry = worth[mine];
        entry_tie = tie[mine];
        place = 0;
#pragma unroll 8
        for (u32 i = 0; i < listed; ++i) {
          const u64 w = worth[i], t = tie[i];
          place += (u32)(w > entry) | ((u32)(w == entry) & (u32)(t > entry_tie));
        }
      }
      __syncthreads();
      if (place < a.k) worth[place] = entry, tie[place] = entry_tie;
      __syncthreads();
      return;
    }
    const u32 size = power_of_two(listed);
    for (u32 i = listed + mine; i < size; i += PICK_THREADS) worth[i] = 0, tie[i] = 0;
    __syncthreads();
    sort_down<PICK_THREADS>(size, [&](u32 low, u32 high, bool down) {
      const u64 x = worth[low], y = worth[high], xt = tie[low], yt = tie[high];
      if ((x < y || (x == y && xt < yt)) == down) worth[low] = y, worth[high] = x, tie[low] = yt, tie[high] = xt;
    });
  };
  for (u64 g = blockIdx.x; g < a.groups; g += gridDim.x) {
    __syncthreads();  // (the last group's readers)
    for (u32 b = wave; b < a.beams; b += WAVES) {
      const u64 row = g * a.beams + b;
      const bool lives = beam_lives(a, row);
      float most = -INFINITY;
      double sum = 0.0;
      if (lives) {
        for (u32 c = lane; c < a.chunks; c += 64) most = __builtin_fmaxf(most, a.most[row * a.chunks + c]);
#pragma unroll
        for (int w = 1; w < 64; w *= 2) most = __builtin_fmaxf(most, __shfl_xor(most, w));
        for (u32 c = lane; c < a.chunks; c += 64) {
          const double s = a.sums[row * a.chunks + c];
          if (s > 0.0) sum += s * beam_exp(beam_below(a.most[row * a.chunks + c], most));
        }
#pragma unroll
        for (int w = 1; w < 64; w *= 2) sum += __shfl_xor(sum, w);
      }
      if (lane == 0) {
        const float total = a.totals[row];
        totals[b] = total;
        mosts[b] = most;
        logs[b] = log(sum);
        state[b] = lives ? (most > -INFINITY ? 2 : 0) : total > -INFINITY ? 1 : 0;
      }
    }
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    // finished beams go on as they are
    if (threadIdx.x < a.beams && state[threadIdx.x] == 1) {
      const u32 at = atomicAdd(&count, 1u);
      worth[at] = worth_key(totals[threadIdx.x]);
      tie[at] = (u64)(63 - threadIdx.x) << 56 | (u64)(0xFFFFFFu - a.pad);
    }
    const u32 lists = a.beams * a.chunks;
    const u64 all = (u64)lists * a.k;
    u64 least = 0, least_tie = 0;  // the k-th so far: others have to be better
    u32 since = 0;                 // entries in a row that were not
    for (u64 first = 0; first < all && since < lists; first += PICK_THREADS) {
      const u64 at = first + lane * WAVES + wave;  // (so that every wave has some of the lists' best ones)
      u64 key = 0, key_tie = 0;
      if (at < all) {
        const u32 l = (u32)(at % lists), b = l / a.chunks;
        if (state[b] == 2) {
          const u64 e = a.best[((g * a.beams + b) * a.chunks + l % a.chunks) * a.k + at / lists];
          if (e) {
            const u32 score = (u32)(e >> 32), id = ~(u32)e;
            const double v = totals[b] + (beam_below(key_float(score), mosts[b]) - logs[b]);
            if (v > -INFINITY) {
              key = worth_key(v);
              key_tie = (u64)(63 - b) << 56 | (u64)score << 24 | (0xFFFFFFu - id);
            }
          }
        }
      }
      bool better = key > least || (key == least && key_tie > least_tie);
      if (first == 0) {
        // the upper halves of the keys: the least of the waves' ceil(k / 16)-th largest ones
        u32 top;
        const u32 mth = wave_mth((u32)(key >> 32), (a.k + WAVES - 1) / WAVES, &top);
        if (lane == 0) bounds[wave] = mth;
        __syncthreads();
        u32 bound = bounds[0];
#pragma unroll
        for (u32 w = 1; w < WAVES; ++w) bound = min(bound, bounds[w]);
        better = better && (u32)(key >> 32) >= bound;
      }
      __syncthreads();  // (the finished ones, or the last turn's list)
      const u32 before = count;
      __syncthreads();
      if (better) {
        const u32 slot = atomicAdd(&count, 1u);
        worth[slot] = key;
        tie[slot] = key_tie;
      }
      __syncthreads();
      const u32 listed = count;
      since = listed == before ? since + PICK_THREADS : 0;
      const bool last = first + PICK_THREADS >= all || since >= lists;
      if (first == 0 || last || listed + PICK_THREADS > PICK_ROOM) {
        order(listed);
        least = worth[a.k - 1];
        least_tie = tie[a.k - 1];
        if (threadIdx.x == 0) count = min(listed, a.k);
        __syncthreads();
      }
    }
    for (u32 i = threadIdx.x; i < a.k; i += PICK_THREADS) {
      const bool some = i < count;
      const u64 key = worth[i], t = tie[i];
      const u64 bits = key >> 63 ? key & ~(1ull << 63) : ~key;
      a.parents[g * a.k + i] = some ? 63 - (u32)(t >> 56) : ANN_NONE;
      a.ids[g * a.k + i] = some ? 0xFFFFFFu - (u32)(t & 0xFFFFFFu) : ANN_NONE;
      a.out[g * a.k + i] = some ? (float)__longlong_as_double((long long)bits) : -INFINITY;
    }
  }
}

// A thread takes a piece of VEC bytes of the rows of all k beams that go on, so that nobody else reads or writes that piece,
// and rows can change places where they are: it reads MOST of them before it writes any, all of them in that case.  There
// rows that stay where they are are not touched.  Bound by memory: 16 layers of 64 rows of 2.3 MB in groups of 8 take 668 us
// beside them and 575 in place, on other cards up to 704 and 697 (with stores that the caches keep 3 to 5 % more).  Chiplets take
// workgroups in turn: each gets runs of pieces, whose rows' parts are longer (without runs 744 and 611, of 32 669 and 574, of 256
// 689 and 587).  Offsets that are multiples of four bytes only cost more than twice the time, others seven times: 2.1 GB in rows
// of 2,046 bytes 4.8 ms, of 2,044 1.55, of 2,048 0.67.
constexpr u64 REORDER_RUN = 64;
struct ReorderArgs {
  const char* in;
  char* out;
  const u32* parents;
  u64 outer, outer_in, outer_out;  // count; strides in bytes
  u64 groups, row_in, row_out;
  u32 beams, k;
  u32 mid, pieces;  // runs of a row, pieces of VEC bytes of a run
  u64 mid_in, mid_out;
  u64 parts;  // workgroups for a row
  u32 in_place;
};
template <int VEC>
struct PieceOf;
template <>
struct PieceOf<16> {
  using type = v4i;
};
template <>
struct PieceOf<4> {
  using type = int;
};
template <>
struct PieceOf<1> {
  using type = char;
};

template <int VEC, int MOST>
__global__ __launch_bounds__(256) void beam_reorder_kernel(ReorderArgs a) {
  using P = typename PieceOf<VEC>::type;
  const u64 tiles = a.outer * a.groups * a.parts;
  for (u64 t = blockIdx.x; t < tiles; t += gridDim.x) {
    const u64 turn = t / (8 * REORDER_RUN) * (8 * REORDER_RUN);
    const u64 tt = turn + 8 * REORDER_RUN <= tiles ? turn + t % 8 * REORDER_RUN + t / 8 % REORDER_RUN : t;
    const u64 og = tt / a.parts, g = og % a.groups, o = og / a.groups;
    const u64 at = tt % a.parts * 256 + threadIdx.x;
    if (at >= (u64)a.mid * a.pieces) continue;
    const u64 m = at / a.pieces, piece = at % a.pieces * VEC;
    const char* in = a.in + o * a.outer_in + g * a.beams * a.row_in + m * a.mid_in + piece;
    char* out = a.out + o * a.outer_out + g * a.k * a.row_out + m * a.mid_out + piece;
    const u32* parents = a.parents + g * a.k;
    for (u32 first = 0; first < a.k; first += MOST) {
      P v[MOST];
#pragma unroll
      for (u32 i = 0; i < MOST; ++i) {
        if (first + i >= a.k) break;
        const u32 p = parents[first + i];
        if (p < a.beams && !(a.in_place && p == first + i)) v[i] = *reinterpret_cast<const P*>(in + p * a.row_in);
      }
#pragma unroll
      for (u32 i = 0; i < MOST; ++i) {
        if (first + i >= a.k) break;
        const u32 p = parents[first + i];
        if (p < a.beams && !(a.in_place && p == first + i)) __builtin_nontemporal_store(v[i], reinterpret_cast<P*>(out + (first + i) * a.row_out));
      }
    }
  }
}

template <int VEC>
hipError_t launch_reorder(ReorderArgs a, u64 run_bytes, hipStream_t s) {
  a.pieces = (u32)(run_bytes / VEC);
  a.parts = ((u64)a.mid * a.pieces + 255) / 256;
  const u64 tiles = a.outer * a.groups * a.parts;
  auto kernel = beam_reorder_kernel<VEC, 8>;
  if (a.in_place && a.k > 8) kernel = a.k <= 16 ? beam_reorder_kernel<VEC, 16> : a.k <= 32 ? beam_reorder_kernel<VEC, 32> : beam_reorder_kernel<VEC, 64>;
  hipLaunchKernelGGL(kernel, dim3((u32)std::min<u64>(tiles, 1u << 22)), dim3(256), 0, s, a);
  return hipGetLastError();
}

u32 beam_chunks(u64 n) { return (u32)((n + BEAM_CHUNK - 1) / BEAM_CHUNK); }

template <typename T>
hipError_t launch_beam(const BeamArgs& a, hipStream_t s) {
  const u64 tiles = a.groups * a.beams * a.chunks;
  hipLaunchKernelGGL(beam_chunk_kernel<T>, dim3((u32)std::min<u64>(tiles, 1u << 22)), dim3(BEAM_THREADS), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(beam_pick_kernel, dim3((u32)std::min<u64>(a.groups, 1u << 21)), dim3(PICK_THREADS), 0, s, a);
  return hipGetLastError();
}

int check_beams(u64 groups, u32 beams, u64 n, u32 k) {
  if (beams < 1 || beams > BEAM_MOST_BEAMS) return fail(ANN_EINVAL, "beams must be 1 to %u", BEAM_MOST_BEAMS);
  if (groups >= (1ull << 31) / beams) return fail(ANN_EINVAL, "groups * beams must stay below 2^31");
  if (n < 1 || n > BEAM_MOST_N) return fail(ANN_EINVAL, "n must be 1 to %u", BEAM_MOST_N);
  if (k < 1 || k > BEAM_MOST_K) return fail(ANN_EINVAL, "k must be 1 to %u", BEAM_MOST_K);
  return ANN_OK;
}

}  // namespace annmi

using namespace annmi;

extern "C" {

int ann_beam_select_scratch(uint64_t groups, uint32_t beams, uint64_t n, uint32_t k, uint64_t* bytes) try {
  if (!bytes) return fail(ANN_EINVAL, "null argument");
  const int rc = check_beams(groups, beams, n, k);
  if (rc) return rc;
  *bytes = groups * beams * beam_chunks(n) * (8ull * k + 8 + 4);
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

int ann_beam_select(const void* scores_dev, uint64_t groups, uint32_t beams, uint64_t n, ann_dtype dtype, uint64_t ld,
                    const float* totals_dev, const uint8_t* finished_dev, uint32_t pad_id, uint32_t k, uint32_t* parents_dev,
                    uint32_t* ids_dev, float* totals_out_dev, void* scratch_dev, uint64_t scratch_bytes, void* stream) try {
  const u64 esz = dtype_bytes(dtype);
  if (esz < 2) return fail(ANN_EINVAL, "scores must be ANN_F32, ANN_F16 or ANN_BF16");
  uint64_t need = 0;
  const int rc = ann_beam_select_scratch(groups, beams, n, k, &need);
  if (rc) return rc;
  if (ld < n) return fail(ANN_EINVAL, "ld must be at least n");
  if (finished_dev && pad_id >= n) return fail(ANN_EINVAL, "pad_id must be below n");
  if (groups == 0) return ANN_OK;
  if (!scores_dev || !totals_dev || !parents_dev || !ids_dev || !totals_out_dev || !scratch_dev) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(scores_dev, esz) || !aligned_to(totals_dev, 4) || !aligned_to(parents_dev, 4) || !aligned_to(ids_dev, 4) || !aligned_to(totals_out_dev, 4))
    return fail(ANN_EINVAL, "an array is not aligned to its elements");
  if (scratch_bytes < need) return fail(ANN_EINVAL, "scratch must hold %llu bytes", (unsigned long long)need);
  if (!aligned_to(scratch_dev, 16)) return fail(ANN_EINVAL, "scratch must be 16-byte aligned");
  // (one group's results may be there before another has read its beams' totals)
  const uintptr_t from = reinterpret_cast<uintptr_t>(totals_dev), to = reinterpret_cast<uintptr_t>(totals_out_dev);
  if (!(from == to && k == beams) && from < to + groups * k * 4 && to < from + groups * beams * 4)
    return fail(ANN_EINVAL, "the totals must lie apart, or in one place with k = beams");
  BeamArgs a{};
  a.scores = static_cast<const char*>(scores_dev);
  a.groups = groups;
  a.beams = beams;
  a.n = (u32)n;
  a.k = k;
  a.ld = ld;
  a.totals = totals_dev;
  a.finished = finished_dev;
  a.pad = pad_id;
  a.chunks = beam_chunks(n);
  const u64 lists = groups * beams * a.chunks;
  a.best = static_cast<u64*>(scratch_dev);
  a.sums = reinterpret_cast<double*>(a.best + lists * k);
  a.most = reinterpret_cast<float*>(a.sums + lists);
  a.parents = parents_dev;
  a.ids = ids_dev;
  a.out = totals_out_dev;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == ANN_F32)
    HIP_TRY(launch_beam<float>(a, st));
  else if (dtype == ANN_F16)
    HIP_TRY(launch_beam<__half>(a, st));
  else
    HIP_TRY(launch_beam<__bf16>(a, st));
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

int ann_beam_reorder(const void* in_dev, void* out_dev, const uint32_t* parents_dev, uint64_t groups, uint32_t beams, uint32_t k,
                     uint64_t outer, uint64_t outer_in, uint64_t outer_out, uint64_t row_in, uint64_t row_out, uint64_t mid,
                     uint64_t mid_in, uint64_t mid_out, uint64_t run_bytes, void* stream) try {
  if (beams < 1 || beams > BEAM_MOST_BEAMS || k < 1 || k > BEAM_MOST_BEAMS) return fail(ANN_EINVAL, "beams and k must be 1 to %u", BEAM_MOST_BEAMS);
  if (groups >= (1ull << 31) / BEAM_MOST_BEAMS || outer >= 1ull << 31 || mid >= 1ull << 31 || run_bytes >= 1ull << 31)
    return fail(ANN_EINVAL, "groups must stay below 2^25, outer, mid and run_bytes below 2^31");
  if (groups == 0 || outer == 0 || mid == 0 || run_bytes == 0) return ANN_OK;
  if (!in_dev || !out_dev || !parents_dev) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(parents_dev, 4)) return fail(ANN_EINVAL, "parents not aligned to their elements");
  // Where rows, their runs and the outer ones lie must be told apart by their strides, and all of it must fit in memory.
  u64 span[2];
  const u64 strides[2][3] = {{outer_in, row_in, mid_in}, {outer_out, row_out, mid_out}};
  for (int side = 0; side < 2; ++side) {
    u64 counts[3] = {outer, groups * (side ? k : beams), mid};
    u64 step[3] = {strides[side][0], strides[side][1], strides[side][2]};
    for (int i = 0; i < 3; ++i)  // by their strides, upwards
      for (int j = i + 1; j < 3; ++j)
        if (step[j] < step[i]) std::swap(step[i], step[j]), std::swap(counts[i], counts[j]);
    unsigned __int128 end = run_bytes;
    for (int i = 0; i < 3; ++i) {
      if (counts[i] == 1) continue;
      if (step[i] < end) return fail(ANN_EINVAL, "rows, their runs or outer parts overlap");
      end += (unsigned __int128)step[i] * (counts[i] - 1);
      if (end >= 1ull << 62) return fail(ANN_EINVAL, "strides too large");
    }
    span[side] = (u64)end;
  }
  const uintptr_t from = reinterpret_cast<uintptr_t>(in_dev), to = reinterpret_cast<uintptr_t>(out_dev);
  ReorderArgs a{};
  a.in_place = from == to;
  if (a.in_place) {
    if (k != beams || (outer > 1 && outer_in != outer_out) || (groups * k > 1 && row_in != row_out) || (mid > 1 && mid_in != mid_out))
      return fail(ANN_EINVAL, "rows that change places where they are need k = beams and the same strides");
  } else if (from < to + span[1] && to < from + span[0]) {
    return fail(ANN_EINVAL, "the arrays must be one and the same or lie apart");
  }
  a.in = static_cast<const char*>(in_dev);
  a.out = static_cast<char*>(out_dev);
  a.parents = parents_dev;
  a.outer = outer;
  a.outer_in = outer_in;
  a.outer_out = outer_out;
  a.groups = groups;
  a.row_in = row_in;
  a.row_out = row_out;
  a.beams = beams;
  a.k = k;
  a.mid = (u32)mid;
  a.mid_in = mid_in;
  a.mid_out = mid_out;
  // the widest piece that all of it is a multiple of
  u64 bits = from | to | run_bytes;
  if (outer > 1) bits |= outer_in | outer_out;
  if (groups * beams > 1) bits |= row_in;
  if (groups * k > 1) bits |= row_out;
  if (mid > 1) bits |= mid_in | mid_out;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (bits % 16 == 0)
    HIP_TRY(launch_reorder<16>(a, run_bytes, st));
  else if (bits % 4 == 0)
    HIP_TRY(launch_reorder<4>(a, run_bytes, st));
  else
    HIP_TRY(launch_reorder<1>(a, run_bytes, st));
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

}  // extern "C"
