// One id drawn for each row of scores, by temperature, top-k, top-p and min-p.
//
// All three rules keep a prefix of the candidates sorted by (score downwards, id), so the kept ones are told by a
// cut: every key above it, and the first `ties` of those at it.  The cuts of top-k (by counts) and top-p (by
// masses) are found by histograms over ever shorter ranges of keys, a small top-k's by a bound from the best scores of the
// row's parts.  Masses are sums of weights rounded to multiples
// of a power of two: whole numbers, whose sums depend on no order.  The draw sums the kept weights in fp64 in a
// fixed order.
#include <type_traits>

#include "mx.hpp"

namespace annmi {

constexpr u32 SAMPLE_THREADS = 1024;
constexpr u32 SAMPLE_WAVES = SAMPLE_THREADS / 64;
constexpr u32 SAMPLE_BINS = 1024;  // one for each thread
constexpr u32 SAMPLE_FEW = 1024;   // so many kept by top-k are sorted in LDS, and the row is not read again
constexpr u32 SAMPLE_TOPS = 1024;  // most of the best scores of a row's parts

// What the launches of a divided call know of a row.
enum SampleKind : u32 {
  ROW_DONE,  // drawn
  ROW_CUT,   // kept: above `lowest`, or at it with an id below tie_end
  ROW_WHOLE  // left to the kernel that takes whole rows
};
struct SampleState {
  u64 tie_end;
  u64 before, want, total;  // counts or masses: above the bin of the cut, up to the cut, of all candidates
  float lowest;
  u32 kind, bin, few;       // few: all candidates up to the bin are listed, not just the bin's
};

struct SampleArgs {
  const char* scores;
  u64 ld, n;
  u32 rows;
  u32 unit;  // weights count in units of 2^-unit in the masses of top-p
  ann_sample_opts o;
  const float* uniform;
  u32* ids;
  float* logprobs;
  // Divided rows (chunks > 0): `groups` workgroups for a row, `per` chunks of `chunk` entries each.  Sums are kept for
  // each chunk, so that they do not depend on how many rows there are.
  u32 chunks, chunk, groups, per;
  u32 rules;           // top-k or top-p may be on
  u32 no_hist;         // a bound serves all rows
  u32 no_mass;         // rows that are not drawn from their lists are left whole
  u32 top_lanes;       // so many lanes share one of `tops`
  u32 tops_of_row;     // 256 / top_lanes for each chunk
  float* most;         // (rows, chunks): best scores
  float* tops;         // (rows, tops_of_row): of parts of the chunks
  double* others;      // masses other than the best candidates'
  u32* ones;           // numbers of best candidates
  u64* hist;           // (rows, SAMPLE_BINS)
  u64* list;           // (rows, capacity): candidates around the cut
  u32 capacity;
  u32* listed;
  float* bound;        // (rows): of those whose k best are told by one
  double* table;       // of the weights: TABLE entries
  SampleState* state;
};

constexpr u32 SAMPLE_LEAST = 0x007FFFFFu;  // float_key(-inf): candidates have larger keys

// low bits of a key that are the same in all values of one sign of a type
template <typename T>
constexpr u32 key_grain() {
  return sizeof(T) == 4 ? 0 : __is_same(T, __half) ? 13 : 16;
}

constexpr u32 TABLE_BITS = 9;
constexpr u32 TABLE = 1u << TABLE_BITS;
__device__ __forceinline__ double table_entry(u32 i) { return exp2(i / (double)TABLE); }
// (a copy: to work it out anew takes a divided call's workgroups longer than all else that they do but once)
template <u32 THREADS>
__device__ __forceinline__ void take_table(const double* from, double* to) {
  for (u32 i = threadIdx.x; i < TABLE; i += THREADS) to[i] = from[i];
}

// exp((score - best) / temperature), within 1e-14 + 5e-16 |x| of itself, where x is the exponent: a power of two, times
// 2^(j / 512) from a table, times the rest, whose logarithm is below ln 2 / 1024, by three terms of its series.  (The next term
// makes 9e-15, the roundings of the difference, the factor and their product 2^-51 |x|.)  Below 1e-300 a weight counts as 0.  Adding 1.5 * 2^52 leaves the
// whole number of 512ths of an octave in the low bits of the sum.
struct Weights {
  float most;          // the best score
  double best, scale;  // as the sums take it; 512 / (temperature ln 2)
  const double* table;
  __device__ __forceinline__ double raw(float score) const {  // (not of +inf); 2^-1000 for all that is smaller
    constexpr double MAGIC = 6755399441055744.0, C = 0.0013538030870311431;  // C: ln 2 / 512
    const double d = __builtin_fmax((static_cast<double>(score) - best) * scale, -512000.0);
    const double t = d + MAGIC;
    const double r = d - (t - MAGIC);
    const int n = static_cast<int>(__double_as_longlong(t));
    const double p = __builtin_fma(__builtin_fma(__builtin_fma(r, C * C * C / 6, C * C / 2), r, C), r, 1.0);
    const double v = table[n & (TABLE - 1)] * p;
    return __hiloint2double(__double2hiint(v) + ((n >> TABLE_BITS) << 20), __double2loint(v));
  }
  __device__ __forceinline__ double of(float score) const {
    const double v = raw(score);
    return score == most ? 1.0 : v > 1e-300 ? v : 0.0;
  }
  // in units of 2^-unit, to the nearest; unit <= 50: adding 2^52 leaves the whole number in the low bits
  __device__ __forceinline__ u64 units(float score, double unit) const { return in_units(of(score), unit); }
  __device__ __forceinline__ u64 in_units(double weight, double unit) const {
    const double v = __builtin_fma(weight, unit, 4503599627370496.0);
    return (u64)((u32)__double2hiint(v) & 0xFFFFFu) << 32 | (u32)__double2loint(v);
  }
};

using True = std::integral_constant<bool, true>;
using False = std::integral_constant<bool, false>;

// Keeps the compiler from taking a value only where it is used: the values of a piece are to be taken side by side.
__device__ __forceinline__ void taken(double& v) { asm volatile("" : "+v"(v)); }

// A row's entries from..to, dealt to `ranks` threads in pieces of 16 bytes, AHEAD of them on their way at once: the
// first ones from where the reader is made, so that what stands between that and `run` hides their way.  run(f) calls
// f(id, scores) for each; what the first and last piece lack of a whole one is -inf, as are no candidates.
template <int AHEAD, typename T>
struct Reader {
  static constexpr u32 V = 16 / sizeof(T);
  using Piece = Pack<T, V>;
  const T* row;
  u64 from, to, head, tail;
  u32 rank, ranks, pieces;
  Piece x[AHEAD];
  __device__ __forceinline__ void ask(u32 p) {
    const Piece* at = reinterpret_cast<const Piece*>(row + head);
#pragma unroll
    for (u32 u = 0; u < AHEAD; ++u) x[u] = at[min(p + u * ranks, pieces - 1)];
  }
  __device__ __forceinline__ Reader(const T* row_, u64 from_, u64 to_, u32 rank_, u32 ranks_) : row(row_), from(from_), to(to_), rank(rank_), ranks(ranks_) {
    const u64 skew = reinterpret_cast<uintptr_t>(row + from) % 16 / sizeof(T);
    head = min(to, from + (V - skew) % V);
    pieces = (u32)((to - head) / V);
    tail = head + (u64)pieces * V;
    if (pieces) ask(rank);
  }
  template <typename F>
  __device__ __forceinline__ void run(F f) {
    for (u32 p = rank; p < pieces; p += AHEAD * ranks) {
      if (p != rank) ask(p);
#pragma unroll
      for (u32 u = 0; u < AHEAD; ++u) {
        __builtin_amdgcn_sched_barrier(0);  // (or several pieces would be worked on at once, in too many registers)
        if (p + u * ranks >= pieces) break;
        float v[V];
#pragma unroll
        for (u32 e = 0; e < V; ++e) v[e] = mx_float(x[u].v[e]);
        f(head + (u64)(p + u * ranks) * V, v);
      }
    }
    if (rank < 2) {
      const u64 lo = rank ? tail : from, hi = rank ? to : head;
      float v[V];
#pragma unroll
      for (u32 e = 0; e < V; ++e) v[e] = lo + e < hi ? mx_float(row[lo + e]) : -__builtin_inff();
      if (lo < hi) f(lo, v);
    }
  }
};
template <int AHEAD, typename T, typename F>
__device__ __forceinline__ void each(const T* row, u64 from, u64 to, u32 rank, u32 ranks, F f) {
  Reader<AHEAD, T>(row, from, to, rank, ranks).run(f);
}

struct SampleLds {
  alignas(16) u64 hist[SAMPLE_BINS];    // counts or masses; sorted candidates
  u64 weight[SAMPLE_BINS];  // of the candidates that are sorted (bits of doubles)
  double table[TABLE];
  u64 wave[SAMPLE_WAVES];
  u64 word;
  u32 count, bin;
};

// sums over the workgroup in a fixed order, the same in every thread: of all, and of this thread's and those before
template <typename V, u32 WAVES = SAMPLE_WAVES>
__device__ V block_scan(V v, u64* words, V* upto) {
  const u32 lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
  for (int w = 1; w < 64; w *= 2) {
    const V x = __shfl_up(v, w);
    if (lane >= (u32)w) v += x;
  }
  __syncthreads();
  if (lane == 63) words[wave] = __builtin_bit_cast(u64, v);
  __syncthreads();
  V sums = __builtin_bit_cast(V, words[lane % WAVES]);
#pragma unroll
  for (u32 w = 1; w < WAVES; w *= 2) {
    const V x = __shfl_up(sums, w, WAVES);
    if (lane % WAVES >= w) sums += x;
  }
  const V before = __shfl(sums, (int)(wave + 63) % 64);
  *upto = wave ? before + v : v;
  return __shfl(sums, WAVES - 1);
}

// s.hist[0 .. count) upwards, all of them different, at most one for each thread.  Few are placed by counting the ones
// before each; more by a bitonic network (256: 0.6 us against 2.6).
__device__ void block_sort(SampleLds& s, u32 count) {
  const u32 i = threadIdx.x;
  __syncthreads();
  if (count <= 256) {
    const u64 mine = i < count ? s.hist[i] : 0;
    u32 rank = 0;
    if (i < count) {
      using v2l = u64 __attribute__((ext_vector_type(2)));
      const v2l* all = reinterpret_cast<const v2l*>(s.hist);
#pragma unroll 4
      for (u32 j = 0; j < count / 2; ++j) {
        const v2l x = all[j];
        rank += (x[0] < mine) + (x[1] < mine);
      }
      if (count % 2) rank += s.hist[count - 1] < mine;
    }
    __syncthreads();
    if (i < count) s.hist[rank] = mine;
    __syncthreads();
    return;
  }
  const u32 size = count <= 512 ? 512 : 1024;
  if (i >= count && i < size) s.hist[i] = ~0ull;
  for (u32 run = 2; run <= size; run *= 2)
    for (u32 gap = run / 2; gap > 0; gap /= 2) {
      __syncthreads();
      if (i < size / 2) {
        const u32 lo = i / gap * 2 * gap + i % gap, hi = lo + gap;
        const u64 x = s.hist[lo], y = s.hist[hi];
        if ((x > y) == ((lo & run) == 0)) s.hist[lo] = y, s.hist[hi] = x;
      }
    }
  __syncthreads();
}

struct Cut {
  u32 key;
  u64 ties;  // how many of the candidates at `key` are kept, the first ones by id
  u64 at;    // how many there are, where `ties` is a number
};

// A row's settings, and what follows from its best score.
struct RowRules {
  float temperature, top_p, min_p, per_score;
  u32 top_k, best;
  double u, floor_w;
  Weights w;
  bool k_on, p_on;
  __device__ __forceinline__ RowRules(const SampleArgs& a, u64 r, const double* table) {
    temperature = a.o.temperature_dev ? a.o.temperature_dev[r] : a.o.temperature;
    top_k = a.o.top_k_dev ? a.o.top_k_dev[r] : a.o.top_k;
    top_p = a.o.top_p_dev ? a.o.top_p_dev[r] : a.o.top_p;
    min_p = a.o.min_p_dev ? a.o.min_p_dev[r] : a.o.min_p;
    k_on = top_k > 0 && top_k < a.n;
    p_on = top_p > 0.0f && top_p < 1.0f;
    floor_w = min_p < 1.0f ? static_cast<double>(min_p) : 1.0;
    u = static_cast<double>(a.uniform[r]);
    // (1 and above: no running mass exceeds it, so that the last kept one is taken; below 0 and NaN count as 0)
    u = !(u >= 0.0) ? 0.0 : u < 1.0 ? u : __builtin_inf();
    // The first histogram is linear in the score, 32 bins for each unit of max(temperature, 1) below the best, the
    // last one open; equal scores share a bin, and the bins fall with the score.
    per_score = 32.0f / (temperature > 1.0f ? temperature : 1.0f);
    w.table = table;
  }
  // false: the row has no candidates
  __device__ __forceinline__ bool set_best(float most) {
    best = float_key(most);
    w.most = key_float(best);  // (+0 for -0)
    // (an infinite temperature has scale 0; next to an infinite best score any other has weight 0 all the same)
    const bool finite = w.most < __builtin_inff();
    w.best = finite ? static_cast<double>(w.most) : 1e300;
    w.scale = finite ? 738.6598609351493 / static_cast<double>(temperature) : 1.0;
    return best > SAMPLE_LEAST;
  }
  // the share of top-p of a mass in whole units
  __device__ __forceinline__ u64 wanted_mass(u64 total) const {
    const u64 want = (u64)ceil(static_cast<double>(top_p) * static_cast<double>(total));
    return want < 1 ? 1 : want > total ? total : want;
  }
  __device__ __forceinline__ bool greedy() const { return !(temperature > 0.0f); }
  __device__ __forceinline__ u32 linear_bin(float v) const {
    // (the smaller of 1023 and a NaN is 1023: inf * 0, or +inf next to a best of +inf, which is put right)
    const float z = __builtin_fminf((w.most - v) * per_score, (float)(SAMPLE_BINS - 1));
    return v == w.most ? 0u : (u32)z;
  }
  // The largest key of a candidate whose bin is b or above, or SAMPLE_LEAST: the bins fall with the key.  64 keys are
  // tried at once, by whole waves.
  __device__ __forceinline__ u32 last_of(u32 b) const {
    const u32 lane = threadIdx.x % 64;
    u64 lo = SAMPLE_LEAST, hi = (u64)best + 1;  // at or below lo: b or above; from hi on: below b
    while (hi - lo > 1) {
      const u64 step = (hi - lo + 63) / 64, x = lo + step * (lane + 1);
      const u64 reach = __ballot(x < hi && linear_bin(key_float((u32)x)) >= b);
      lo += step * (u32)__popcll(reach);
      hi = min(hi, lo + step);
    }
    return (u32)lo;
  }
  // The smallest key not below `from` whose weight reaches the floor of min-p.  Weights fall with the key; 64 keys
  // around the one that the logarithm gives are tried at once, by whole waves.
  __device__ __forceinline__ u32 min_p_key(u32 from) const {
    const u32 lane = threadIdx.x % 64;
    if (w.most < __builtin_inff() && temperature < __builtin_inff()) {
      const u32 near = float_key(static_cast<float>(w.best + static_cast<double>(temperature) * log(floor_w)));
      const u32 first = max(from, min(near - 32, best - 63));  // (keys of candidates are far above 63)
      const u64 reach = __ballot(first + lane <= best && w.of(key_float(first + lane)) >= floor_w);
      if (reach && (first == from || !(reach & 1))) return first + (u32)__builtin_ctzll(reach);
    }
    u32 lo = from, hi = best;  // hi reaches it
    while (lo < hi) {
      const u32 mid = lo + (hi - lo) / 2;
      if (w.of(key_float(mid)) >= floor_w)
        hi = mid;
      else
        lo = mid + 1;
    }
    return hi;
  }
};

// Few candidates, s.hist[0 .. count): those of rank below `limit` by (key downwards, id) are cut by top-p and min-p,
// sorted by id and drawn from, a thread for each.
__device__ void draw_few(const SampleArgs& a, u64 r, const RowRules& rules, u64 limit, u32 count, double unit, SampleLds& s) {
  const u32 tid = threadIdx.x;
  block_sort(s, count);
  const bool mine = tid < limit && tid < count;
  const u64 entry = mine ? s.hist[tid] : 0;
  const float score = key_float(~(u32)(entry >> 32));
  const double weight = mine ? rules.w.of(score) : 0.0;
  u64 upto;
  const u64 units = mine ? rules.w.units(score, unit) : 0;
  const u64 total = block_scan<u64>(units, s.wave, &upto);
  bool keep = mine;
  if (rules.p_on) keep = keep && upto - units < rules.wanted_mass(total);
  if (rules.min_p > 0.0f) keep = keep && weight >= rules.floor_w;
  const u32 kept = (u32)__syncthreads_count(keep);  // (the first ones)
  if (keep) s.hist[tid] = (entry & 0xFFFFFFFFull) << 32 | tid;
  s.weight[tid] = __builtin_bit_cast(u64, weight);
  block_sort(s, kept);
  const bool there = tid < kept;
  const u32 from = there ? (u32)s.hist[tid] : 0;
  const double x = there ? __builtin_bit_cast(double, s.weight[from]) : 0.0;
  double run, others;
  const double sum = block_scan<double>(x, s.wave, &run);
  // the mass without this one, not as a difference from the whole where it is the best: it may be all the mass
  const double rest = block_scan<double>(from == 0 ? 0.0 : x, s.wave, &others);
  const double aim = rules.u * sum;
  if (tid == 0) s.word = ~0ull, s.count = 0;
  __syncthreads();
  if (x > 0.0) {
    if (run > aim) atomicMin(reinterpret_cast<unsigned long long*>(&s.word), (unsigned long long)tid);
    atomicMax(&s.count, tid);
  }
  __syncthreads();
  const u32 at = s.word != ~0ull ? (u32)s.word : s.count;
  if (tid == at) {
    a.ids[r] = (u32)(s.hist[tid] >> 32);
    if (a.logprobs) a.logprobs[r] = static_cast<float>(-log1p((from == 0 ? rest : 1.0 + rest - x) / x));
  }
}

// The same for at most 64 candidates, `entry` of each lane, by one wave without the others: same sums in the same
// order.  `room`: 64 places of LDS of the wave's own.
__device__ void draw_by_wave(const SampleArgs& a, u64 r, const RowRules& rules, u64 limit, u32 count, u64 entry, double unit, u64* room) {
  const u32 lane = threadIdx.x % 64;
  // the lane's entry becomes the one whose rank it is, among those of the first `among` lanes
  auto sort = [&](u64 mine, u32 among) {
    using v2l = u64 __attribute__((ext_vector_type(2)));
    wave_exchange();
    room[lane] = lane < among ? mine : ~0ull;
    wave_exchange();
    u32 rank = 0;
#pragma unroll 4
    for (u32 j = 0; j < among; j += 2) {
      const v2l x = *reinterpret_cast<const v2l*>(room + j);
      rank += (x[0] < mine) + (x[1] < mine);
    }
    wave_exchange();
    if (lane < among) room[rank] = mine;
    wave_exchange();
    return room[lane];
  };
  auto scan = [&](auto v) {
#pragma unroll
    for (int w = 1; w < 64; w *= 2) {
      const auto x = __shfl_up(v, w);
      if (lane >= (u32)w) v += x;
    }
    return v;
  };
  entry = sort(entry, count);
  const bool mine = lane < limit && lane < count;
  const float score = key_float(~(u32)(entry >> 32));
  const double weight = mine ? rules.w.of(score) : 0.0;
  bool keep = mine;
  if (rules.p_on) {
    const u64 units = mine ? rules.w.units(score, unit) : 0, upto = scan(units);
    const u64 want = rules.wanted_mass(__shfl(upto, 63));  // (by all lanes)
    keep = keep && upto - units < want;
  }
  if (rules.min_p > 0.0f) keep = keep && weight >= rules.floor_w;
  const u32 kept = (u32)__popcll(__ballot(keep));  // (the first ones)
  const u64 by_id = sort((entry & 0xFFFFFFFFull) << 32 | lane, kept);
  const bool there = lane < kept;
  const u32 from = there ? (u32)by_id & 63 : 0;
  const double there_weight = __shfl(weight, (int)from);
  const double x = there ? there_weight : 0.0;
  const double run = scan(x), sum = __shfl(run, 63);
  // the mass without this one, not as a difference from the whole where it is the best: it may be all the mass
  const double rest = __shfl(scan(from == 0 ? 0.0 : x), 63);
  const u64 above = __ballot(x > 0.0 && run > rules.u * sum), some = __ballot(x > 0.0);
  const u32 at = above ? (u32)__builtin_ctzll(above) : 63u - (u32)__builtin_clzll(some);
  if (lane == at) {
    a.ids[r] = (u32)(by_id >> 32);
    if (a.logprobs) a.logprobs[r] = static_cast<float>(-log1p((from == 0 ? rest : 1.0 + rest - x) / x));
  }
}

// A workgroup per row.  The row is read once for its best score, once to three times for each cut, once for the draw
// (and a sixteenth of it, and so on, to find the draw's place); all but the first time from the caches.
template <typename T>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(SampleArgs a) {
  __shared__ SampleLds s;
  const u32 tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  constexpr u32 GRAIN = key_grain<T>();
  for (u64 r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* row = reinterpret_cast<const T*>(a.scores) + r * a.ld;
    if (a.state[r].kind != ROW_WHOLE) continue;
    __syncthreads();
    take_table<SAMPLE_THREADS>(a.table, s.table);
    RowRules rules(a, r, s.table);
    auto all = [&](auto f) { each<4>(row, 0, a.n, tid, SAMPLE_THREADS, f); };
    constexpr u32 V = 16 / sizeof(T);

    float most = -__builtin_inff();
    each<4>(row, 0, a.n, tid, SAMPLE_THREADS, [&](u64, const float (&v)[V]) {
#pragma unroll
      for (u32 e = 0; e < V; ++e) most = __builtin_fmaxf(most, v[e]);  // (passes over NaN)
    });
#pragma unroll
    for (int w = 1; w < 64; w *= 2) most = __builtin_fmaxf(most, __shfl_xor(most, w));
    __syncthreads();
    if (lane == 0) s.wave[wave] = __float_as_uint(most);
    __syncthreads();
    for (u32 w = 0; w < SAMPLE_WAVES; ++w) most = __builtin_fmaxf(most, __uint_as_float((u32)s.wave[w]));
    if (!rules.set_best(most)) {  // (the same in all threads)
      if (tid == 0) {
        a.ids[r] = ANN_NONE;
        if (a.logprobs) a.logprobs[r] = -__builtin_inff();
      }
      continue;
    }
    const u32 best = rules.best;
    most = rules.w.most;
    if (rules.greedy()) {
      if (tid == 0) s.word = ~0ull;
      __syncthreads();
      u64 first = ~0ull;
      all([&](u64 i, const float (&v)[V]) {
#pragma unroll
        for (u32 e = 0; e < V; ++e)
          if (v[e] == most) first = min(first, i + e);
      });
      if (first != ~0ull) atomicMin(reinterpret_cast<unsigned long long*>(&s.word), (unsigned long long)first);
      __syncthreads();
      if (tid == 0) {
        a.ids[r] = (u32)s.word;
        if (a.logprobs) a.logprobs[r] = 0.0f;
      }
      continue;
    }
    const Weights& w = rules.w;
    const double unit = ldexp(1.0, (int)a.unit);
    Cut cut = {SAMPLE_LEAST + 1, ~0ull, ~0ull};

    // Finds the key at which the running count (or mass), from the best key down, reaches `aim(total)`; candidates
    // below floor.key do not count, and of those at it floor.ties do.  False: the total is 0 or below the aim.
    auto select = [&](const Cut& floor, bool mass, auto aim, Cut* found, u64* rest) -> bool {
      u32 hi = best, lo = floor.key, shift = 0;
      u64 want = 0;
      const bool some_ties = mass && floor.ties != ~0ull;  // counted by number: equal keys have equal weights
      for (int level = 0;; ++level) {
        __syncthreads();
        s.hist[tid] = 0;
        __syncthreads();
        const float lowest = key_float(lo), highest = key_float(hi);
        const float none = some_ties ? key_float(floor.key) : -__builtin_inff();
        auto count = [&](auto first, auto masses) {
          all([&](u64, const float (&v)[V]) {
            bool in[V], any = false;
#pragma unroll
            for (u32 e = 0; e < V; ++e) any |= in[e] = v[e] >= lowest && v[e] <= highest && v[e] != none;
            if (!any) return;
            double raw[V];
            if (masses)
#pragma unroll
              for (u32 e = 0; e < V; ++e) raw[e] = w.raw(v[e]), taken(raw[e]);
#pragma unroll
            for (u32 e = 0; e < V; ++e)
              if (in[e])
                atomicAdd(reinterpret_cast<unsigned long long*>(&s.hist[first ? rules.linear_bin(v[e]) : (hi - float_key(v[e])) >> shift]),
                          (unsigned long long)(masses ? w.in_units(v[e] == most ? 1.0 : raw[e], unit) : 1ull));
          });
        };
        if (level == 0)
          mass ? count(True(), True()) : count(True(), False());
        else
          mass ? count(False(), True()) : count(False(), False());
        __syncthreads();
        if (tid == 0 && some_ties && floor.key >= lo)
          s.hist[level ? (hi - floor.key) >> shift : rules.linear_bin(key_float(floor.key))] += floor.ties * w.units(key_float(floor.key), unit);
        __syncthreads();
        const u64 mine = s.hist[tid];
        u64 upto;
        const u64 total = block_scan<u64>(mine, s.wave, &upto);
        if (level == 0) {
          want = aim(total);
          if (want == 0 || want > total) return false;
        }
        if (upto >= want && upto - mine < want) s.bin = tid, s.word = want - (upto - mine);
        __syncthreads();
        const u32 b = s.bin;
        want = s.word;
        found->at = s.hist[b];
        if (level == 0) {
          // the keys of the bin, by bisection: the bins fall with the key
          u32 x = lo, y = hi;
          while (x < y) {  // the largest key whose bin is b or above
            const u32 mid = x + (y - x + 1) / 2;
            if (rules.linear_bin(key_float(mid)) >= b)
              x = mid;
            else
              y = mid - 1;
          }
          const u32 top = x;
          x = lo, y = top;
          while (x < y) {  // the smallest key whose bin is b
            const u32 mid = x + (y - x) / 2;
            if (rules.linear_bin(key_float(mid)) <= b)
              y = mid;
            else
              x = mid + 1;
          }
          hi = top, lo = x;
        } else {
          hi -= b << shift;
          lo = max(lo, hi - ((1u << shift) - 1));
        }
        // The type's values are the keys whose low bits are 0 (not negative) or 1 (negative): up to the end of the
        // block of the largest value that is not above hi.
        constexpr u32 LOW = (1u << GRAIN) - 1;
        hi = (hi >> 31) || (hi & LOW) == LOW ? hi | LOW : (hi & ~LOW) - 1;
        if (hi >> GRAIN == lo >> GRAIN) {  // one value
          found->key = hi >> 31 ? hi & ~LOW : hi;
          *rest = want;
          return true;
        }
        const u32 bits = 32 - __builtin_clz(hi - lo);
        shift = bits > 10 + GRAIN ? bits - 10 : GRAIN;
      }
    };

    u64 tie_end = a.n;
    float lowest = key_float(cut.key);
    u64 lo = 0, hi = a.n;
    double others = 0.0, bests = 0.0, aim = 0.0;
    if (rules.k_on) {
      Cut found;
      u64 ties;
      if (select(cut, false, [&](u64 total) { return (u64)rules.top_k < total ? (u64)rules.top_k : 0; }, &found, &ties)) {
        cut = found;
        cut.ties = ties;
      }
    }
    if (cut.ties != ~0ull && rules.top_k - cut.ties + cut.at <= SAMPLE_FEW) {
      __syncthreads();
      if (tid == 0) s.count = 0;
      __syncthreads();
      lowest = key_float(cut.key);
      all([&](u64 i, const float (&v)[V]) {
#pragma unroll
        for (u32 e = 0; e < V; ++e)
          if (v[e] >= lowest) s.hist[atomicAdd(&s.count, 1u)] = (u64)~float_key(v[e]) << 32 | (i + e);
      });
      __syncthreads();
      draw_few(a, r, rules, rules.top_k, s.count, unit, s);
      continue;
    }
    if (rules.p_on) {
      Cut found;
      u64 left;
      if (select(cut, true, [&](u64 total) { return rules.wanted_mass(total); }, &found, &left)) {
        const u64 each_one = w.units(key_float(found.key), unit);
        const u64 need = each_one ? (left + each_one - 1) / each_one : ~0ull, at = each_one ? found.at / each_one : ~0ull;
        if (found.key != cut.key || cut.ties == ~0ull)
          cut = {found.key, need, at};
        else if (need < cut.ties)  // (`at` of top-k counts the ones that it dropped as well)
          cut.ties = need;
      }
    }
    if (rules.min_p > 0.0f) {
      const u32 key = rules.min_p_key(cut.key);
      if (key > cut.key) cut.key = key, cut.ties = ~0ull;
    }
    lowest = key_float(cut.key);
    // Where only some of those at the cut are kept, they are the first ones by id: those below `tie_end`.
    if (cut.ties < cut.at) {
      // narrowed down like the draw below: runs of the span, counted by a wave each
      u64 lo = 0, hi = a.n, before = 0;
      while (hi - lo > SAMPLE_THREADS) {
        const u64 run = ((hi - lo + SAMPLE_WAVES - 1) / SAMPLE_WAVES + 63) / 64 * 64;
        const u64 from = min(hi, lo + wave * run), to = min(hi, from + run);
        u32 mine = 0;
        each<4>(row, from, to, lane, 64, [&](u64, const float (&v)[V]) {
#pragma unroll
          for (u32 e = 0; e < V; ++e) mine += v[e] == lowest;
        });
#pragma unroll
        for (int v = 1; v < 64; v *= 2) mine += (u32)__shfl_xor((int)mine, v);
        __syncthreads();
        if (lane == 0) s.wave[wave] = mine;
        __syncthreads();
        u32 at = 0;
        while (at + 1 < SAMPLE_WAVES && before + s.wave[at] <= cut.ties) before += s.wave[at++];
        lo += at * run;
        hi = min(hi, lo + run);
      }
      const u64 i = lo + tid;
      const u64 tie = i < hi && mx_float(row[i]) == lowest;
      u64 upto;
      block_scan<u64>(tie, s.wave, &upto);
      if (tie && before + upto - 1 == cut.ties) s.word = i;
      __syncthreads();
      tie_end = s.word;
    }
    // The draw: the span that holds it is dealt to the waves in runs, whose masses tell which run it is.  The best
    // candidates' weights, 1 each, are kept apart, so that a mass that is nearly all the drawn one's loses nothing.
    bool whole = true;
    while (whole || hi - lo > 4 * SAMPLE_THREADS) {
      u64 run = (hi - lo + SAMPLE_WAVES - 1) / SAMPLE_WAVES;
      run = (run + 63) / 64 * 64;
      const u64 from = min(hi, lo + wave * run), to = min(hi, from + run);
      double mine = 0.0;
      u32 ones = 0;
      each<2>(row, from, to, lane, 64, [&](u64 i, const float (&v)[V]) {
        bool keep[V], any = false;
#pragma unroll
        for (u32 e = 0; e < V; ++e) {
          keep[e] = v[e] >= lowest;
          if (v[e] == lowest) keep[e] = i + e < tie_end;
          any |= keep[e];
        }
        if (!any) return;
        double raw[V];
#pragma unroll
        for (u32 e = 0; e < V; ++e) raw[e] = w.raw(keep[e] && v[e] != most ? v[e] : -__builtin_inff()), taken(raw[e]);
#pragma unroll
        for (u32 e = 0; e < V; ++e) {
          ones += keep[e] && v[e] == most;
          mine += raw[e] > 1e-300 ? raw[e] : 0.0;
        }
      });
#pragma unroll
      for (int v = 1; v < 64; v *= 2) mine += __shfl_xor(mine, v), ones += (u32)__shfl_xor((int)ones, v);
      __syncthreads();
      if (lane == 0) s.wave[wave] = __builtin_bit_cast(u64, mine), s.hist[wave] = ones;
      __syncthreads();
      // (every wave alike, a lane for each run)
      const double rest = __builtin_bit_cast(double, s.wave[lane % SAMPLE_WAVES]), one = static_cast<double>(s.hist[lane % SAMPLE_WAVES]);
      if (whole) {
        others = rest, bests = one;
#pragma unroll
        for (int v = 1; v < (int)SAMPLE_WAVES; v *= 2) others += __shfl_xor(others, v, SAMPLE_WAVES), bests += __shfl_xor(bests, v, SAMPLE_WAVES);
        aim = rules.u * (bests + others);
        whole = false;
      }
      const double mass = rest + one;
      double upto = mass;
#pragma unroll
      for (int v = 1; v < (int)SAMPLE_WAVES; v *= 2) {
        const double x = __shfl_up(upto, v, SAMPLE_WAVES);
        if (lane % SAMPLE_WAVES >= (u32)v) upto += x;
      }
      const u64 above = __ballot(lane < SAMPLE_WAVES && mass > 0.0 && upto > aim), some = __ballot(lane < SAMPLE_WAVES && mass > 0.0);
      // (none above, by rounding: the last run that holds anything)
      const u32 at = above ? (u32)__builtin_ctzll(above) : 63u - (u32)__builtin_clzll(some);
      const double before = __shfl(upto, (int)(at + 63) % 64);
      aim -= at ? before : 0.0;
      lo += at * run;
      hi = min(hi, lo + run);
    }
    // the last span, a thread for four entries
    float v[4];
    double weight[4], mine = 0.0, run;
    u32 some = 0;  // of the four, which hold anything
#pragma unroll
    for (u32 e = 0; e < 4; ++e) {
      const u64 i = lo + tid * 4 + e;
      v[e] = i < hi ? mx_float(row[i]) : -__builtin_inff();
      weight[e] = v[e] > lowest || (v[e] == lowest && i < tie_end) ? w.of(v[e]) : 0.0;
      mine += weight[e];
      some |= (weight[e] > 0.0) << e;
    }
    block_scan<double>(mine, s.wave, &run);
    if (tid == 0) s.word = ~0ull, s.count = 0;
    __syncthreads();
    if (some) {
      if (run > aim) atomicMin(reinterpret_cast<unsigned long long*>(&s.word), (unsigned long long)tid);
      atomicMax(&s.count, tid);
    }
    __syncthreads();
    if (tid == (s.word != ~0ull ? (u32)s.word : s.count)) {
      double upto = run - mine;
      u32 at = 31 - __builtin_clz(some);  // (none above the aim, by rounding: the last that holds anything)
#pragma unroll
      for (int e = 3; e >= 0; --e) {
        double before = upto;
        for (int f = 0; f < e; ++f) before += weight[f];
        if (weight[e] > 0.0 && before + weight[e] > aim) at = e;
      }
      a.ids[r] = (u32)(lo + tid * 4 + at);
      if (a.logprobs) {
        float score = v[0];
        double x = weight[0];
#pragma unroll
        for (u32 e = 1; e < 4; ++e)
          if (at == e) score = v[e], x = weight[e];
        a.logprobs[r] = static_cast<float>(-log1p((score == most ? bests - 1.0 + others : bests + others - x) / x));
      }
    }
  }
}


// Divided rows: several workgroups share each.  One launch takes the best scores of the chunks and of their parts.  Where
// these tell the k best, the next finds the bound, else one takes the chunks' histograms (added up per row: whole
// numbers).  One lists the candidates around the cut, one finds the cut from these or, where top-k keeps few, draws, one
// takes the chunks' masses, and one draws.  Rows whose cut needs more than the list holds are left to the kernel above, as are
// rows with top-p whose top-k drops nothing or keeps more than some 1,000 (64 x 50,001 with top-p 0.9: top-k 1,100 114 us, 900
// 64 us; of 600 candidates, top-k 1,000 76 us, 400 41 us) and, in calls with one top-k of up to 512 for all rows, those that
// take the best candidate alone (one such row of 64 x 50,001: 41 us against 34).
// Times of a launch for one row of 128,000 bf16 with top-p, and for 500 such of fp16 with settings of their own (128 MB, 26 us
// at a copy's rate): best scores 3.6 and 24 us, bound - and 10, histograms 6 and 35, lists 5.5 and 30, cuts 5 and 35,
// masses 8.5 and 44, draw 9 and 16, what is left whole 3.5 and 6.  One row: the chain of launches and, inside of each, of
// two or three trips to memory.  500 rows: vector instructions, most of them in fp64 for the weights, which histograms
// and masses need of every entry.
constexpr u32 SPLIT_THREADS = 256;
constexpr u32 SPLIT_CHUNKS = 256;  // most of a row
constexpr u32 SPLIT_LIST = 16384, SPLIT_LEAST_LIST = 6144;  // most candidates of a list
constexpr u32 SPLIT_CHUNK = 4096;  // entries of one, where a row has no more than 256 of that size

struct SplitLds {
  u64 hist[SAMPLE_BINS];
  double table[TABLE];
  u64 wave[SPLIT_THREADS / 64];
  u64 word[3];
  u32 count, place;
};

struct Part {  // of a row: what a workgroup takes
  u64 r, from, to;
  u32 group, c0, c1;
  __device__ __forceinline__ explicit Part(const SampleArgs& a) {
    r = blockIdx.x / a.groups;
    group = blockIdx.x % a.groups;
    c0 = min(group * a.per, a.chunks), c1 = min(c0 + a.per, a.chunks);
    from = (u64)c0 * a.chunk, to = min(a.n, (u64)c1 * a.chunk);
  }
};

__device__ __forceinline__ float split_max(float v, u64* words) {
#pragma unroll
  for (int w = 1; w < 64; w *= 2) v = __builtin_fmaxf(v, __shfl_xor(v, w));
  __syncthreads();
  if (threadIdx.x % 64 == 0) words[threadIdx.x / 64] = __float_as_uint(v);
  __syncthreads();
#pragma unroll
  for (u32 w = 0; w < SPLIT_THREADS / 64; ++w) v = __builtin_fmaxf(v, __uint_as_float((u32)words[w]));
  return v;
}
__device__ __forceinline__ float row_best(const SampleArgs& a, u64 r, u64* words) {
  return split_max(threadIdx.x < a.chunks ? a.most[r * a.chunks + threadIdx.x] : -__builtin_inff(), words);
}

// Whether the k best are told by a bound.  Where k parts of a row have a score of at least some value, so have k
// candidates; that value is the k-th largest of the parts' best scores.  With k up to half of the parts, some 1.4 k
// candidates reach it where good scores lie in no order, and no histogram is needed.
constexpr u32 BOUND_MOST_K = SAMPLE_FEW / 4;
__host__ __device__ __forceinline__ bool bound_serves(u32 top_k, u32 tops_of_row) { return top_k > 0 && top_k <= BOUND_MOST_K && top_k <= tops_of_row / 2; }
// A value that k of the tops reach and none that is much larger does: the upper 20 bits of the k-th largest key, found
// bit by bit, by one wave for a row.  (By one of each workgroup that lists: 66 us against 36 for 500 rows.)
__device__ __forceinline__ float kth_top(const float* tops, u32 count, u32 k) {
  constexpr u32 EACH = SAMPLE_TOPS / 64;
  const u32 lane = threadIdx.x % 64;
  u32 key[EACH], found = 0;
#pragma unroll
  for (u32 i = 0; i < EACH; ++i) key[i] = __float_as_uint(tops[min(i * 64 + lane, count - 1)]);  // (all on their way at once)
#pragma unroll
  for (u32 i = 0; i < EACH; ++i) key[i] = i * 64 + lane < count ? float_key(__uint_as_float(key[i])) : 0u;
  for (u32 bit = 1u << 31; bit >= 1u << 12; bit >>= 1) {
    u32 reach = 0;
#pragma unroll
    for (u32 i = 0; i < EACH; ++i) {
      if (i * 64 >= count) break;
      reach += (u32)__popcll(__ballot(key[i] >= (found | bit)));
    }
    if (reach >= k) found |= bit;
  }
  return key_float(max(found, SAMPLE_LEAST));
}

template <typename T>
__global__ __launch_bounds__(SPLIT_THREADS) void sample_best_kernel(SampleArgs a) {
  __shared__ u64 words[SPLIT_THREADS / 64];
  constexpr u32 V = 16 / sizeof(T);
  const Part p(a);
  const T* row = reinterpret_cast<const T*>(a.scores) + p.r * a.ld;
  for (u32 c = p.c0; c < p.c1; ++c) {
    float most = -__builtin_inff();
    each<4>(row, (u64)c * a.chunk, min(a.n, (u64)(c + 1) * a.chunk), threadIdx.x, SPLIT_THREADS, [&](u64, const float (&v)[V]) {
#pragma unroll
      for (u32 e = 0; e < V; ++e) most = __builtin_fmaxf(most, v[e]);  // (passes over NaN)
    });
    if (a.rules) {
      float top = most;
      for (u32 w = 1; w < a.top_lanes; w *= 2) top = __builtin_fmaxf(top, __shfl_xor(top, (int)w));
      if (threadIdx.x % a.top_lanes == 0) a.tops[p.r * a.tops_of_row + (c * SPLIT_THREADS + threadIdx.x) / a.top_lanes] = top;
    }
    most = split_max(most, words);
    if (threadIdx.x == 0) a.most[p.r * a.chunks + c] = most;
  }
  if (blockIdx.x == 0)
    for (u32 i = threadIdx.x; i < TABLE; i += SPLIT_THREADS) a.table[i] = table_entry(i);
  if (a.rules) {  // clears the row's histogram, a share each
    for (u32 b = p.group * SPLIT_THREADS + threadIdx.x; b < SAMPLE_BINS; b += a.groups * SPLIT_THREADS) a.hist[p.r * SAMPLE_BINS + b] = 0;
    if (p.group == 0 && threadIdx.x == 0) a.listed[p.r] = 0;
  }
}

__global__ __launch_bounds__(64) void sample_bound_kernel(SampleArgs a) {
  const u64 r = blockIdx.x;
  const u32 top_k = a.o.top_k_dev ? a.o.top_k_dev[r] : a.o.top_k;
  if (!bound_serves(top_k, a.tops_of_row)) return;
  const float bound = kth_top(a.tops + r * a.tops_of_row, a.tops_of_row, top_k);
  if (threadIdx.x == 0) a.bound[r] = bound;
}

template <typename T>
__global__ __launch_bounds__(SPLIT_THREADS) void sample_hist_kernel(SampleArgs a) {
  __shared__ SplitLds s;
  constexpr u32 V = 16 / sizeof(T);
  const u32 tid = threadIdx.x;
  const Part p(a);
  const T* row = reinterpret_cast<const T*>(a.scores) + p.r * a.ld;
  RowRules rules(a, p.r, s.table);
  if (rules.greedy() || !(rules.k_on || rules.p_on)) return;
  if (rules.k_on && bound_serves(rules.top_k, a.tops_of_row)) return;
  Reader<4, T> entries(row, p.from, p.to, tid, SPLIT_THREADS);
  if (!rules.set_best(row_best(a, p.r, s.wave))) return;
  const bool masses = !rules.k_on;
  if (masses)
    take_table<SPLIT_THREADS>(a.table, s.table);
  for (u32 b = tid; b < SAMPLE_BINS; b += SPLIT_THREADS) s.hist[b] = 0;
  __syncthreads();
  const double unit = ldexp(1.0, (int)a.unit);
  const float most = rules.w.most;
  auto count = [&](auto of_masses) {
    entries.run([&](u64, const float (&v)[V]) {
      double raw[V];
      if (of_masses)
#pragma unroll
        for (u32 e = 0; e < V; ++e) raw[e] = rules.w.raw(v[e]), taken(raw[e]);
#pragma unroll
      for (u32 e = 0; e < V; ++e)
        if (v[e] > -__builtin_inff())
          atomicAdd(reinterpret_cast<unsigned long long*>(&s.hist[rules.linear_bin(v[e])]),
                    (unsigned long long)(of_masses ? rules.w.in_units(v[e] == most ? 1.0 : raw[e], unit) : 1ull));
    });
  };
  masses ? count(True()) : count(False());
  __syncthreads();
  for (u32 b = tid; b < SAMPLE_BINS; b += SPLIT_THREADS)
    if (s.hist[b]) atomicAdd(reinterpret_cast<unsigned long long*>(&a.hist[p.r * SAMPLE_BINS + b]), (unsigned long long)s.hist[b]);
}

template <typename T>
__global__ __launch_bounds__(SPLIT_THREADS) void sample_list_kernel(SampleArgs a) {
  __shared__ SplitLds s;
  constexpr u32 V = 16 / sizeof(T), BINS = SAMPLE_BINS / SPLIT_THREADS;
  const u32 tid = threadIdx.x;
  const Part p(a);
  const T* row = reinterpret_cast<const T*>(a.scores) + p.r * a.ld;
  RowRules rules(a, p.r, nullptr);
  SampleState state{};
  state.kind = ROW_CUT;
  state.bin = ~0u;
  // Into LDS first, and to the row's list at once; what LDS has no room for goes there by itself (or, with `spill` off,
  // nowhere: s.count tells).
  auto put = [&](u32 at, u64 entry) {  // (too many for the list: its count alone says so)
    if (at < a.capacity) a.list[p.r * a.capacity + at] = entry;
  };
  auto gather = [&](auto& entries, auto listed, bool spill) {
    if (tid == 0) s.count = 0;
    __syncthreads();
    entries.run([&](u64 i, const float (&v)[V]) {
      bool any = false;
#pragma unroll
      for (u32 e = 0; e < V; ++e) any |= listed(v[e]);
      if (!any) return;
#pragma unroll
      for (u32 e = 0; e < V; ++e)
        if (listed(v[e])) {
          const u64 entry = (u64)~float_key(v[e]) << 32 | (i + e);
          const u32 at = atomicAdd(&s.count, 1u);
          if (at < SAMPLE_BINS)
            s.hist[at] = entry;
          else if (spill)
            put(atomicAdd(&a.listed[p.r], 1u), entry);
        }
    });
    __syncthreads();
  };
  auto hand_over = [&]() {
    const u32 count = min(s.count, SAMPLE_BINS);
    if (tid == 0 && count) s.place = atomicAdd(&a.listed[p.r], count);
    __syncthreads();
    for (u32 i = tid; i < count; i += SPLIT_THREADS) put(s.place + i, s.hist[i]);
  };
  if (rules.greedy() || !(rules.k_on || rules.p_on)) {
  } else if (rules.k_on && bound_serves(rules.top_k, a.tops_of_row)) {
    Reader<4, T> entries(row, p.from, p.to, tid, SPLIT_THREADS);
    const float bound = a.bound[p.r];
    state.bin = 0, state.want = rules.top_k, state.few = 1;
    auto above = [&](float v) { return v >= bound && v > -__builtin_inff(); };
    gather(entries, above, false);
    if (s.count > 2 * BOUND_MOST_K) {
      // Good scores side by side: of a workgroup's own entries only the first `top_k` matter, and those that share a bin of
      // the histogram with the last of them.  (64 sorted rows of 50,001, k = 50: 51 us
      // against 143 that the kernel of whole rows takes.)
      rules.set_best(row_best(a, p.r, s.wave));
      __syncthreads();
      for (u32 b = tid; b < SAMPLE_BINS; b += SPLIT_THREADS) s.hist[b] = 0;
      __syncthreads();
      each<4>(row, p.from, p.to, tid, SPLIT_THREADS, [&](u64, const float (&v)[V]) {
#pragma unroll
        for (u32 e = 0; e < V; ++e)
          if (above(v[e])) atomicAdd(reinterpret_cast<unsigned long long*>(&s.hist[rules.linear_bin(v[e])]), 1ull);
      });
      __syncthreads();
      u64 bin[BINS], mine = 0, upto;
#pragma unroll
      for (u32 i = 0; i < BINS; ++i) mine += bin[i] = s.hist[tid * BINS + i];
      block_scan<u64, SPLIT_THREADS / 64>(mine, s.wave, &upto);
      u64 before = upto - mine;
#pragma unroll
      for (u32 i = 0; i < BINS; ++i) {
        if (before < rules.top_k && before + bin[i] >= rules.top_k) s.word[0] = tid * BINS + i;
        before += bin[i];
      }
      __syncthreads();
      if (tid < 64) s.word[1] = rules.last_of((u32)s.word[0] + 1) + 1;
      __syncthreads();
      const float low = key_float((u32)s.word[1]);
      Reader<4, T> again(row, p.from, p.to, tid, SPLIT_THREADS);
      gather(again, [&](float v) { return above(v) && v >= low; }, true);
    }
    hand_over();
  } else if (rules.set_best(row_best(a, p.r, s.wave))) {
    Reader<4, T> entries(row, p.from, p.to, tid, SPLIT_THREADS);
    u64 bin[BINS], mine = 0, upto;
#pragma unroll
    for (u32 i = 0; i < BINS; ++i) mine += bin[i] = a.hist[p.r * SAMPLE_BINS + tid * BINS + i];
    const u64 total = block_scan<u64, SPLIT_THREADS / 64>(mine, s.wave, &upto);
    const u64 want = !rules.k_on ? rules.wanted_mass(total) : rules.top_k < total ? rules.top_k : 0;
    if (want == 0) {
      // top-k drops nothing; what top-p keeps then needs masses that were not counted
      if (rules.p_on) state.kind = ROW_WHOLE;
    } else {
      u64 before = upto - mine;
#pragma unroll
      for (u32 i = 0; i < BINS; ++i) {
        if (before < want && before + bin[i] >= want) s.word[0] = tid * BINS + i, s.word[1] = before, s.word[2] = bin[i];
        before += bin[i];
      }
      __syncthreads();
      state.bin = (u32)s.word[0], state.before = s.word[1], state.want = want, state.total = total;
      const u64 in_bin = s.word[2];
      if (rules.k_on) {
        state.few = state.before + in_bin <= SAMPLE_FEW;
        if (!state.few && (in_bin > a.capacity || rules.p_on)) state.kind = ROW_WHOLE;
      }
      if (state.kind == ROW_CUT) {
        __syncthreads();
        // the keys of the bin, an end by a wave each
        if (tid < 128) s.word[tid / 64] = tid < 64 ? rules.last_of(state.bin + 1) + 1 : state.few ? rules.best : rules.last_of(state.bin);
        __syncthreads();
        const float low = key_float((u32)s.word[0]), top = key_float((u32)s.word[1]);
        gather(entries, [&](float v) { return v >= low && v <= top; }, true);
        hand_over();
      }
    }
  }
  // (without the launches that follow, rows whose list does not end in a draw: greedy and empty ones among them)
  if (a.no_mass && state.kind == ROW_CUT && !state.few) state.kind = ROW_WHOLE;
  if (p.group == 0 && tid == 0) a.state[p.r] = state;
}

template <typename T>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_cut_kernel(SampleArgs a) {
  __shared__ SampleLds s;
  const u32 tid = threadIdx.x;
  const u64 r = blockIdx.x;
  SampleState state = a.state[r];
  if (state.kind != ROW_CUT) return;
  take_table<SAMPLE_THREADS>(a.table, s.table);
  RowRules rules(a, r, s.table);
  float most = tid < a.chunks ? a.most[r * a.chunks + tid] : -__builtin_inff();
#pragma unroll
  for (int w = 1; w < 64; w *= 2) most = __builtin_fmaxf(most, __shfl_xor(most, w));
  if (tid % 64 == 0) s.wave[tid / 64] = __float_as_uint(most);
  __syncthreads();
  for (u32 w = 0; w < SAMPLE_WAVES; ++w) most = __builtin_fmaxf(most, __uint_as_float((u32)s.wave[w]));
  __syncthreads();
  if (!rules.set_best(most)) {
    if (tid == 0 && state.few) {  // (others are left to the draw, which may not follow)
      a.ids[r] = ANN_NONE;
      if (a.logprobs) a.logprobs[r] = -__builtin_inff();
      a.state[r].kind = ROW_DONE;
    }
    return;
  }
  if (rules.greedy()) return;  // (the draw needs no cut)
  u32 lowest = SAMPLE_LEAST + 1;
  state.tie_end = a.n;
  if (state.bin != ~0u) {
    const u64* list = a.list + r * a.capacity;
    u32 count = a.listed[r];
    bool left = count > a.capacity;
    const double unit = ldexp(1.0, (int)a.unit);
    if (!left && count > SAMPLE_FEW) {
      // A long list: entries sort as (key downwards, id) and are all different; the histogram of their range, and of
      // the part of the cut again, until few are left.
      u64 lo = ~0ull, hi = 0;
      for (u32 i = tid; i < count; i += SAMPLE_THREADS) lo = min(lo, list[i]), hi = max(hi, list[i]);
#pragma unroll
      for (int w = 1; w < 64; w *= 2) lo = min(lo, __shfl_xor(lo, w)), hi = max(hi, __shfl_xor(hi, w));
      if (tid % 64 == 0) s.wave[tid / 64] = lo, s.hist[tid / 64] = hi;
      __syncthreads();
      for (u32 w = 0; w < SAMPLE_WAVES; ++w) lo = min(lo, s.wave[w]), hi = max(hi, s.hist[w]);
      u32 some;
      do {
        const u32 bits = 64 - __builtin_clzll(hi - lo), shift = bits > 10 ? bits - 10 : 0;
        __syncthreads();
        s.hist[tid] = 0;
        __syncthreads();
        for (u32 i = tid; i < count; i += SAMPLE_THREADS) {
          const u64 entry = list[i];
          if (entry < lo || entry > hi) continue;
          atomicAdd(reinterpret_cast<unsigned long long*>(&s.hist[(entry - lo) >> shift]),
                    (unsigned long long)(rules.k_on ? 1 : rules.w.units(key_float(~(u32)(entry >> 32)), unit)));
        }
        __syncthreads();
        const u64 mine = s.hist[tid];
        u64 upto;
        block_scan<u64>(mine, s.wave, &upto);
        if (state.before + upto >= state.want && state.before + upto - mine < state.want) s.bin = tid, s.word = upto - mine;
        if (tid == 0) s.count = 0;
        __syncthreads();
        lo += (u64)s.bin << shift;
        hi = min(hi, lo + (((u64)1 << shift) - 1));  // (of one type: mixed ones are compared as doubles)
        state.before += s.word;
        for (u32 i = tid; i < count; i += SAMPLE_THREADS) {
          const u64 entry = list[i];
          if (entry < lo || entry > hi) continue;
          const u32 at = atomicAdd(&s.count, 1u);
          if (at < SAMPLE_FEW) s.hist[at] = entry;
        }
        __syncthreads();
        some = s.count;
      } while (some > SAMPLE_FEW);
      count = some;
      if (state.few) {
        // (a bound's: the first `want` are drawn from, up to the one that the count reaches)
        __syncthreads();
        block_sort(s, count);
        const u64 last = s.hist[state.want - state.before - 1];
        __syncthreads();
        if (tid == 0) s.count = 0;
        __syncthreads();
        for (u32 i = tid; i < a.listed[r]; i += SAMPLE_THREADS)
          if (list[i] <= last) s.hist[atomicAdd(&s.count, 1u)] = list[i];
        __syncthreads();
        count = s.count;
      }
      __syncthreads();
    } else if (!left && state.few && count <= 64) {
      __syncthreads();
      if (tid < 64) draw_by_wave(a, r, rules, rules.top_k, count, tid < count ? list[tid] : 0, unit, s.hist);
      if (tid == 0) a.state[r].kind = ROW_DONE;
      return;
    } else if (!left && tid < count) {
      s.hist[tid] = list[tid];
    }
    if (left) {
      if (tid == 0) a.state[r].kind = ROW_WHOLE;
      return;
    }
    __syncthreads();
    if (rules.k_on && state.few) {
      draw_few(a, r, rules, rules.top_k, count, unit, s);
      if (tid == 0) a.state[r].kind = ROW_DONE;
      return;
    }
    block_sort(s, count);
    const u64 entry = tid < count ? s.hist[tid] : 0;
    const u64 amount = tid >= count ? 0 : rules.k_on ? 1 : rules.w.units(key_float(~(u32)(entry >> 32)), unit);
    u64 upto;
    block_scan<u64>(amount, s.wave, &upto);
    // the last one kept: the first at which the count (or mass) is reached
    if (tid < count && state.before + upto - amount < state.want && state.before + upto >= state.want) s.word = entry;
    __syncthreads();
    lowest = ~(u32)(s.word >> 32);
    state.tie_end = (s.word & 0xFFFFFFFFull) + 1;
  }
  if (rules.min_p > 0.0f) {
    const u32 key = rules.min_p_key(lowest);
    if (key > lowest) lowest = key, state.tie_end = a.n;
  }
  if (tid == 0) {
    state.lowest = key_float(lowest);
    a.state[r] = state;
  }
}

template <typename T>
__global__ __launch_bounds__(SPLIT_THREADS) void sample_mass_kernel(SampleArgs a) {
  __shared__ SplitLds s;
  constexpr u32 V = 16 / sizeof(T);
  const u32 tid = threadIdx.x;
  const Part p(a);
  if (a.rules && a.state[p.r].kind != ROW_CUT) return;
  const T* row = reinterpret_cast<const T*>(a.scores) + p.r * a.ld;
  RowRules rules(a, p.r, s.table);
  if (rules.greedy()) return;
  auto chunk = [&](u32 c) { return Reader<4, T>(row, (u64)c * a.chunk, min(a.n, (u64)(c + 1) * a.chunk), tid, SPLIT_THREADS); };
  Reader<4, T> entries = chunk(p.c0);
  take_table<SPLIT_THREADS>(a.table, s.table);
  if (!rules.set_best(row_best(a, p.r, s.wave))) return;
  float lowest = key_float(SAMPLE_LEAST + 1);
  u64 tie_end = a.n;
  if (a.rules)
    lowest = a.state[p.r].lowest, tie_end = a.state[p.r].tie_end;
  else if (rules.min_p > 0.0f)
    lowest = key_float(rules.min_p_key(SAMPLE_LEAST + 1));
  const Weights& w = rules.w;
  const float most = w.most;
  for (u32 c = p.c0; c < p.c1; ++c) {
    double mine = 0.0;
    u32 ones = 0;
    if (c != p.c0) entries = chunk(c);
    entries.run([&](u64 i, const float (&v)[V]) {
      bool keep[V], any = false;
#pragma unroll
      for (u32 e = 0; e < V; ++e) {
        keep[e] = v[e] >= lowest;
        if (v[e] == lowest) keep[e] = i + e < tie_end;
        any |= keep[e];
      }
      if (!any) return;
      double raw[V];
#pragma unroll
      for (u32 e = 0; e < V; ++e) raw[e] = w.raw(keep[e] && v[e] != most ? v[e] : -__builtin_inff()), taken(raw[e]);
#pragma unroll
      for (u32 e = 0; e < V; ++e) {
        ones += keep[e] && v[e] == most;
        mine += raw[e] > 1e-300 ? raw[e] : 0.0;
      }
    });
    u64 one_upto;
    double upto;
    const double sum = block_scan<double, SPLIT_THREADS / 64>(mine, s.wave, &upto);
    const u64 one = block_scan<u64, SPLIT_THREADS / 64>(ones, s.wave, &one_upto);
    if (tid == 0) a.others[p.r * a.chunks + c] = sum, a.ones[p.r * a.chunks + c] = (u32)one;
  }
}

// A workgroup per row: the chunk that holds the draw, by the chunks' masses, then the entry.
template <typename T>
__global__ __launch_bounds__(SPLIT_THREADS) void sample_draw_kernel(SampleArgs a) {
  __shared__ SplitLds s;
  constexpr u32 EACH = SPLIT_CHUNK / SPLIT_THREADS, WAVES = SPLIT_THREADS / 64, V = 16 / sizeof(T);
  const u32 tid = threadIdx.x;
  const u64 r = blockIdx.x;
  const bool chunk = tid < a.chunks;
  const u64 place = r * a.chunks + (chunk ? tid : 0);
  const float most_here = a.most[place];
  const double other = a.others[place];
  const u32 one = a.ones[place];
  SampleState state{};
  state.kind = ROW_CUT;
  if (a.rules) state = a.state[r];
  if (state.kind != ROW_CUT) return;
  take_table<SPLIT_THREADS>(a.table, s.table);
  RowRules rules(a, r, s.table);
  const T* row = reinterpret_cast<const T*>(a.scores) + r * a.ld;
  if (tid == 0) s.word[0] = ~0ull, s.word[1] = ~0ull;
  if (!rules.set_best(split_max(chunk ? most_here : -__builtin_inff(), s.wave))) {  // (the same in all threads)
    if (tid == 0) {
      a.ids[r] = ANN_NONE;
      if (a.logprobs) a.logprobs[r] = -__builtin_inff();
    }
    return;
  }
  const Weights& w = rules.w;
  const float most = w.most;
  auto* words = reinterpret_cast<unsigned long long*>(s.word);
  if (rules.greedy()) {
    if (chunk && most_here == most) atomicMin(&words[0], (unsigned long long)tid);
    __syncthreads();
    const u64 lo = s.word[0] * a.chunk, hi = min(a.n, lo + a.chunk);
    for (u64 i = lo + tid; i < hi; i += SPLIT_THREADS)
      if (mx_float(row[i]) == most) {
        atomicMin(&words[1], (unsigned long long)i);
        break;
      }
    __syncthreads();
    if (tid == 0) {
      a.ids[r] = (u32)s.word[1];
      if (a.logprobs) a.logprobs[r] = 0.0f;
    }
    return;
  }
  float lowest = key_float(SAMPLE_LEAST + 1);
  u64 tie_end = a.n;
  if (a.rules)
    lowest = state.lowest, tie_end = state.tie_end;
  else if (rules.min_p > 0.0f)
    lowest = key_float(rules.min_p_key(SAMPLE_LEAST + 1));
  double upto;
  const double others = block_scan<double, WAVES>(chunk ? other : 0.0, s.wave, &upto);
  const double bests = block_scan<double, WAVES>(chunk ? one : 0.0, s.wave, &upto);
  const double mass = chunk ? other + one : 0.0;
  block_scan<double, WAVES>(mass, s.wave, &upto);
  double aim = rules.u * (bests + others);
  // the first whose running mass is above the aim, or (none, by rounding) the last that holds anything
  auto first_above = [&](double mine, double run) {
    if (tid == 0) s.word[0] = ~0ull, s.count = 0;
    __syncthreads();
    if (mine > 0.0) {
      if (run > aim) atomicMin(&words[0], (unsigned long long)tid);
      atomicMax(&s.count, tid);
    }
    __syncthreads();
    const u32 at = s.word[0] != ~0ull ? (u32)s.word[0] : s.count;
    if (tid == at) s.word[1] = __builtin_bit_cast(u64, run - mine);
    __syncthreads();
    return at;
  };
  const u32 at = first_above(mass, upto);
  aim -= at ? __builtin_bit_cast(double, s.word[1]) : 0.0;
  u64 lo = (u64)at * a.chunk;
  const u64 hi = min(a.n, lo + a.chunk);

  // 4,096 entries at a time (longer chunks have several such blocks), sixteen neighbours a thread
  float v[EACH];
  double weight[EACH];
  auto weigh = [&](u64 from) {
    const u64 mine = from + tid * EACH;
    if (reinterpret_cast<uintptr_t>(row) % 16 == 0 && mine + EACH <= hi) {
      Pack<T, V> x[EACH / V];
#pragma unroll
      for (u32 i = 0; i < EACH / V; ++i) x[i] = reinterpret_cast<const Pack<T, V>*>(row + mine)[i];
#pragma unroll
      for (u32 e = 0; e < EACH; ++e) v[e] = mx_float(x[e / V].v[e % V]);
    } else {
#pragma unroll
      for (u32 e = 0; e < EACH; ++e) v[e] = mine + e < hi ? mx_float(row[mine + e]) : -__builtin_inff();
    }
    double sum = 0.0;
#pragma unroll
    for (u32 e = 0; e < EACH; ++e) {
      const bool keep = v[e] > lowest || (v[e] == lowest && mine + e < tie_end);
      weight[e] = w.of(keep ? v[e] : -__builtin_inff());
      sum += weight[e];
    }
    return sum;
  };
  double mine = weigh(lo), run;
  double block = block_scan<double, WAVES>(mine, s.wave, &run);
  if (hi - lo > SPLIT_CHUNK) {
    u64 last = lo;
    double before = 0.0, before_last = 0.0;
    while (true) {
      if (block > 0.0) last = lo, before_last = before;
      if (before + block > aim || lo + SPLIT_CHUNK >= hi) break;
      before += block;
      lo += SPLIT_CHUNK;
      mine = weigh(lo);
      block = block_scan<double, WAVES>(mine, s.wave, &run);
    }
    if (lo != last) {
      lo = last;
      mine = weigh(lo);
      block_scan<double, WAVES>(mine, s.wave, &run);
    }
    aim -= before_last;
  }
  if (tid == first_above(mine, run)) {
    double before = run - mine, x = 0.0;
    u32 which = 0;
#pragma unroll
    for (u32 e = 0; e < EACH; ++e) {  // (the running mass before this one: the last taken is the one that passes the aim)
      if (weight[e] > 0.0 && !(x > 0.0 && before > aim)) which = e, x = weight[e];
      before += weight[e];
    }
    a.ids[r] = (u32)(lo + tid * EACH + which);
    if (a.logprobs) {
      float score = v[0];
#pragma unroll
      for (u32 e = 1; e < EACH; ++e)
        if (which == e) score = v[e];
      a.logprobs[r] = static_cast<float>(-log1p((score == most ? bests - 1.0 + others : bests + others - x) / x));
    }
  }
}

// Short rows: a workgroup holds a row in its registers, EACH neighbours a thread.
constexpr u32 SMALL_THREADS = 256;
template <u32 EACH>
struct SmallLds {
  alignas(16) u64 list[SMALL_THREADS * EACH];
  u64 hist[SAMPLE_BINS];
  double table[TABLE];
  u64 wave[SMALL_THREADS / 64];
  u64 word[3];
  u32 count;
};

// list[0 .. count) upwards, all of them different
template <u32 THREADS>
__device__ void sort_list(u64* list, u32 count) {
  const u32 i = threadIdx.x;
  __syncthreads();
  if (count <= THREADS) {  // placed by counting the ones before each
    const u64 mine = i < count ? list[i] : 0;
    u32 rank = 0;
    if (i < count)
      for (u32 j = 0; j < count; ++j) rank += list[j] < mine;
    __syncthreads();
    if (i < count) list[rank] = mine;
    __syncthreads();
    return;
  }
  u32 size = 2;
  while (size < count) size *= 2;
  for (u32 j = count + i; j < size; j += THREADS) list[j] = ~0ull;
  for (u32 run = 2; run <= size; run *= 2)
    for (u32 gap = run / 2; gap > 0; gap /= 2) {
      __syncthreads();
      for (u32 j = i; j < size / 2; j += THREADS) {
        const u32 lo = j / gap * 2 * gap + j % gap, hi = lo + gap;
        const u64 x = list[lo], y = list[hi];
        if ((x > y) == ((lo & run) == 0)) list[lo] = y, list[hi] = x;
      }
    }
  __syncthreads();
}

template <typename T, u32 EACH>
__global__ __launch_bounds__(SMALL_THREADS) void sample_short_kernel(SampleArgs a) {
  __shared__ SmallLds<EACH> s;
  constexpr u32 WAVES = SMALL_THREADS / 64, BINS = SAMPLE_BINS / SMALL_THREADS;
  const u32 tid = threadIdx.x, n = (u32)a.n, first = tid * EACH;
  const double unit = ldexp(1.0, (int)a.unit);
  auto* words = reinterpret_cast<unsigned long long*>(s.word);
  for (u32 i = tid; i < TABLE; i += SMALL_THREADS) s.table[i] = table_entry(i);
  for (u64 r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* row = reinterpret_cast<const T*>(a.scores) + r * a.ld;
    float v[EACH], most = -__builtin_inff();
#pragma unroll
    for (u32 e = 0; e < EACH; ++e) v[e] = mx_float(row[min(first + e, n - 1)]);
    RowRules rules(a, r, s.table);
#pragma unroll
    for (u32 e = 0; e < EACH; ++e) {
      if (!(first + e < n && v[e] == v[e])) v[e] = -__builtin_inff();
      most = __builtin_fmaxf(most, v[e]);
    }
    most = split_max(most, s.wave);
    __syncthreads();
    if (tid == 0) s.word[0] = ~0ull;
    if (!rules.set_best(most)) {  // (the same in all threads)
      if (tid == 0) {
        a.ids[r] = ANN_NONE;
        if (a.logprobs) a.logprobs[r] = -__builtin_inff();
      }
      continue;
    }
    const Weights& w = rules.w;
    most = w.most;
    __syncthreads();
    if (rules.greedy()) {
#pragma unroll
      for (u32 e = EACH; e-- > 0;)
        if (v[e] == most) atomicMin(&words[0], (unsigned long long)(first + e));
      __syncthreads();
      if (tid == 0) {
        a.ids[r] = (u32)s.word[0];
        if (a.logprobs) a.logprobs[r] = 0.0f;
      }
      __syncthreads();
      continue;
    }
    // Kept: above `lowest`, or at it with an id below tie_end.
    float lowest = key_float(SAMPLE_LEAST + 1);
    u32 tie_end = n;
    auto kept = [&](u32 e) { return v[e] > lowest || (v[e] == lowest && first + e < tie_end); };
    // Moves the cut to where the count (or mass) of the kept ones, from the best down, reaches `aim(total)`.
    auto cut = [&](auto masses, auto aim) {
      __syncthreads();
#pragma unroll
      for (u32 i = 0; i < BINS; ++i) s.hist[tid + i * SMALL_THREADS] = 0;
      if (tid == 0) s.count = 0;
      __syncthreads();
#pragma unroll
      for (u32 e = 0; e < EACH; ++e)
        if (kept(e)) atomicAdd(reinterpret_cast<unsigned long long*>(&s.hist[rules.linear_bin(v[e])]), (unsigned long long)(masses ? w.units(v[e], unit) : 1ull));
      __syncthreads();
      u64 bin[BINS], mine = 0, upto;
#pragma unroll
      for (u32 i = 0; i < BINS; ++i) mine += bin[i] = s.hist[tid * BINS + i];
      const u64 total = block_scan<u64, WAVES>(mine, s.wave, &upto), want = aim(total);
      if (want == 0) return;
      u64 before = upto - mine;
#pragma unroll
      for (u32 i = 0; i < BINS; ++i) {
        if (before < want && before + bin[i] >= want) s.word[0] = tid * BINS + i, s.word[1] = before;
        before += bin[i];
      }
      __syncthreads();
      const u32 b = (u32)s.word[0];
      before = s.word[1];
#pragma unroll
      for (u32 e = 0; e < EACH; ++e)
        if (kept(e) && rules.linear_bin(v[e]) == b) s.list[atomicAdd(&s.count, 1u)] = (u64)~float_key(v[e]) << 32 | (first + e);
      __syncthreads();
      const u32 count = s.count;
      sort_list<SMALL_THREADS>(s.list, count);
      for (u32 at = 0; at < count; at += SMALL_THREADS) {
        const u64 entry = at + tid < count ? s.list[at + tid] : 0;
        const u64 amount = at + tid >= count ? 0 : masses ? w.units(key_float(~(u32)(entry >> 32)), unit) : 1;
        const u64 sum = block_scan<u64, WAVES>(amount, s.wave, &upto);
        if (amount && before + upto - amount < want && before + upto >= want) s.word[2] = entry;
        before += sum;
        if (before >= want) break;
      }
      __syncthreads();
      lowest = key_float(~(u32)(s.word[2] >> 32));
      tie_end = (u32)s.word[2] + 1;
    };
    if (rules.k_on) cut(False(), [&](u64 total) { return (u64)rules.top_k < total ? (u64)rules.top_k : 0; });
    if (rules.p_on) cut(True(), [&](u64 total) { return rules.wanted_mass(total); });
    if (rules.min_p > 0.0f) {
      const u32 from = float_key(lowest), key = rules.min_p_key(from);
      if (key > from) lowest = key_float(key), tie_end = n;
    }
    double weight[EACH], mine = 0.0, others = 0.0, bests = 0.0, run, upto;
#pragma unroll
    for (u32 e = 0; e < EACH; ++e) {
      weight[e] = kept(e) ? w.of(v[e]) : 0.0;
      mine += weight[e];
      if (v[e] == most && weight[e] > 0.0)
        bests += 1.0;
      else
        others += weight[e];
    }
    others = block_scan<double, WAVES>(others, s.wave, &upto);
    bests = block_scan<double, WAVES>(bests, s.wave, &upto);
    block_scan<double, WAVES>(mine, s.wave, &run);
    const double aim = rules.u * (bests + others);
    // the first whose running mass is above the aim, or (none, by rounding) the last that holds anything
    if (tid == 0) s.word[0] = ~0ull, s.count = 0;
    __syncthreads();
    if (mine > 0.0) {
      if (run > aim) atomicMin(&words[0], (unsigned long long)tid);
      atomicMax(&s.count, tid);
    }
    __syncthreads();
    if (tid == (s.word[0] != ~0ull ? (u32)s.word[0] : s.count)) {
      double before = run - mine, x = 0.0;
      float score = 0.0f;
      u32 which = 0;
#pragma unroll
      for (u32 e = 0; e < EACH; ++e) {  // (the running mass before this one: the last taken is the one that passes the aim)
        if (weight[e] > 0.0 && !(x > 0.0 && before > aim)) which = e, x = weight[e], score = v[e];
        before += weight[e];
      }
      a.ids[r] = first + which;
      if (a.logprobs) a.logprobs[r] = static_cast<float>(-log1p((score == most ? bests - 1.0 + others : bests + others - x) / x));
    }
    __syncthreads();
  }
}

// Rows above SHORT entries are divided, SPLIT_ROWS of them at a time.
constexpr u64 SHORT = SMALL_THREADS * 16, SPLIT_ROWS = 4096;

// fills in what a divided call needs and returns its scratch, or 0 where rows are short
u64 plan_split(SampleArgs& a, u64 rows, u64 n, char* scratch) {
  a.chunks = 0;
  if (n <= SHORT || rows == 0) return 0;
  if (rows > SPLIT_ROWS) rows = SPLIT_ROWS;
  u64 chunk = SPLIT_CHUNK;
  while ((n + chunk - 1) / chunk > SPLIT_CHUNKS) chunk *= 2;
  a.chunk = (u32)chunk;
  a.chunks = (u32)((n + chunk - 1) / chunk);
  // Some eight thousand workgroups: 500 rows of 128,000 with settings of each take 197 us; by half and a quarter of that 198 and
  // 219, by a workgroup for each chunk 227.  (Rows with the same settings are served better by fewer: 200 x 128,000 with top-p
  // 158 us against 134 and 136, 3,000 x 20,000 with top-k 157 against 155 and 136.)
  const u64 groups = (8192 + rows - 1) / rows;
  a.per = (u32)(groups >= a.chunks ? 1 : (a.chunks + groups - 1) / groups);
  a.groups = (a.chunks + a.per - 1) / a.per;
  // A bin of the histogram, 1/32 of max(temperature, 1) of score, has about n / 200 of scores near their middle that spread by
  // 2.5; sorted rows bring up to 256 entries and a bin from each of some 17 chunks.  Scores that spread by little fill a list
  // with one bin, and such rows are taken whole: 64 x 128,000 with top-p 0.9 at temperature 1 take 97 us where the standard
  // deviation is 0.2, 232 at 0.1, 496 at 0.02 (one row at 0.1 186 us, at 0.3 50).  Lists of 16,384 for all would take 103 us in
  // the place of 232, the same where 6,144 do, and 32 us more than these where they do not.
  a.capacity = n / 64 < SPLIT_LEAST_LIST ? SPLIT_LEAST_LIST : n / 64 < SPLIT_LIST ? (u32)(n / 64) : SPLIT_LIST;
  u64 at = 0;
  auto take = [&](u64 bytes) {
    const u64 from = at;
    at += (bytes + 15) / 16 * 16;
    return scratch + from;
  };
  a.hist = reinterpret_cast<u64*>(take(rows * SAMPLE_BINS * 8));
  a.list = reinterpret_cast<u64*>(take(rows * a.capacity * 8));
  a.state = reinterpret_cast<SampleState*>(take(rows * sizeof(SampleState)));
  a.others = reinterpret_cast<double*>(take(rows * a.chunks * 8));
  a.ones = reinterpret_cast<u32*>(take(rows * a.chunks * 4));
  a.most = reinterpret_cast<float*>(take(rows * a.chunks * 4));
  a.top_lanes = a.chunks <= 64 ? 16 : a.chunks <= 128 ? 32 : 64;
  a.tops_of_row = a.chunks * (SPLIT_THREADS / a.top_lanes);
  a.tops = reinterpret_cast<float*>(take(rows * a.tops_of_row * 4));
  a.listed = reinterpret_cast<u32*>(take(rows * 4));
  a.bound = reinterpret_cast<float*>(take(rows * 4));
  a.table = reinterpret_cast<double*>(take(TABLE * 8));
  return at;
}

template <typename T>
hipError_t launch_sample(SampleArgs a, hipStream_t s) {
  if (a.chunks == 0) {
    const dim3 grid(a.rows < (1u << 20) ? a.rows : (1u << 20));
    if (a.n <= SMALL_THREADS * 4)
      hipLaunchKernelGGL((sample_short_kernel<T, 4>), grid, dim3(SMALL_THREADS), 0, s, a);
    else
      hipLaunchKernelGGL((sample_short_kernel<T, 16>), grid, dim3(SMALL_THREADS), 0, s, a);
    return hipGetLastError();
  }
  const u64 all = a.rows;
  for (u64 row0 = 0; row0 < all; row0 += SPLIT_ROWS) {
    a.rows = (u32)(all - row0 < SPLIT_ROWS ? all - row0 : SPLIT_ROWS);
    const dim3 parts(a.rows * a.groups), threads(SPLIT_THREADS);
    hipLaunchKernelGGL(sample_best_kernel<T>, parts, threads, 0, s, a);
    if (a.rules) {
      if (a.no_hist || a.o.top_k_dev) hipLaunchKernelGGL(sample_bound_kernel, dim3(a.rows), dim3(64), 0, s, a);
      if (!a.no_hist) hipLaunchKernelGGL(sample_hist_kernel<T>, parts, threads, 0, s, a);
      hipLaunchKernelGGL(sample_list_kernel<T>, parts, threads, 0, s, a);
      hipLaunchKernelGGL(sample_cut_kernel<T>, dim3(a.rows), dim3(SAMPLE_THREADS), 0, s, a);
    }
    if (!a.no_mass) {
      hipLaunchKernelGGL(sample_mass_kernel<T>, parts, threads, 0, s, a);
      hipLaunchKernelGGL(sample_draw_kernel<T>, dim3(a.rows), threads, 0, s, a);
    }
    if (a.rules) hipLaunchKernelGGL(sample_kernel<T>, dim3(a.rows < 256 ? a.rows : 256), dim3(SAMPLE_THREADS), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // the next rows
    a.scores += SPLIT_ROWS * a.ld * sizeof(T);
    a.uniform += SPLIT_ROWS;
    a.ids += SPLIT_ROWS;
    if (a.logprobs) a.logprobs += SPLIT_ROWS;
    if (a.o.temperature_dev) a.o.temperature_dev += SPLIT_ROWS;
    if (a.o.top_k_dev) a.o.top_k_dev += SPLIT_ROWS;
    if (a.o.top_p_dev) a.o.top_p_dev += SPLIT_ROWS;
    if (a.o.min_p_dev) a.o.min_p_dev += SPLIT_ROWS;
  }
  return hipSuccess;
}

}  // namespace annmi

using namespace annmi;

extern "C" {

int ann_sample_scratch(uint64_t rows, uint64_t n, uint64_t* bytes) try {
  if (!bytes) return fail(ANN_EINVAL, "null argument");
  if (rows > MX_MOST_ROWS || n < 1 || n > MX_MOST_ROWS) return fail(ANN_EINVAL, "ann_sample: n must be at least 1, rows and n below 2^31");
  SampleArgs a{};
  *bytes = plan_split(a, rows, n, nullptr);
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

int ann_sample(const void* scores_dev, uint64_t rows, uint64_t n, ann_dtype dtype, uint64_t ld, const ann_sample_opts* opts,
               const float* uniform_dev, uint32_t* ids_dev, float* logprobs_dev, void* scratch_dev, uint64_t scratch_bytes,
               void* stream) try {
  const u64 esz = dtype_bytes(dtype);
  if (esz < 2) return fail(ANN_EINVAL, "scores must be ANN_F32, ANN_F16 or ANN_BF16");
  u64 need = 0;
  int rc = ann_sample_scratch(rows, n, &need);
  if (rc) return rc;
  if (ld < n) return fail(ANN_EINVAL, "ld must be at least n");
  if (rows == 0) return ANN_OK;
  if (!scores_dev || !uniform_dev || !ids_dev) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(scores_dev, esz) || !aligned_to(uniform_dev, 4) || !aligned_to(ids_dev, 4) || !aligned_to(logprobs_dev, 4))
    return fail(ANN_EINVAL, "arguments not aligned to their elements");
  if (need && (!scratch_dev || !aligned_to(scratch_dev, 16) || scratch_bytes < need))
    return fail(ANN_EINVAL, "scratch: %llu bytes are needed, 16-byte aligned (ann_sample_scratch)", (unsigned long long)need);
  SampleArgs a{};
  a.scores = static_cast<const char*>(scores_dev);
  a.ld = ld;
  a.n = n;
  a.rows = (u32)rows;
  a.unit = 62;
  while ((1ull << (62 - a.unit)) < n) --a.unit;
  if (a.unit > 50) a.unit = 50;
  a.o.temperature = 1.0f;
  if (opts) a.o = *opts;
  a.uniform = uniform_dev;
  a.ids = ids_dev;
  a.logprobs = logprobs_dev;
  if (!aligned_to(a.o.temperature_dev, 4) || !aligned_to(a.o.top_k_dev, 4) || !aligned_to(a.o.top_p_dev, 4) || !aligned_to(a.o.min_p_dev, 4))
    return fail(ANN_EINVAL, "settings not aligned to their elements");
  plan_split(a, rows, n, static_cast<char*>(scratch_dev));
  // top-k and top-p are off for all rows where single values say so
  a.rules = a.o.top_k_dev || a.o.top_p_dev || (a.o.top_k > 0 && a.o.top_k < n) || (a.o.top_p > 0.0f && a.o.top_p < 1.0f);
  hipStream_t st = static_cast<hipStream_t>(stream);
  // one top-k for all rows of which their lists hold enough, but where many scores are equal or masked
  a.no_mass = !a.o.top_k_dev && a.o.top_k > 0 && a.o.top_k <= SAMPLE_FEW / 2 && a.o.top_k < n;
  a.no_hist = a.no_mass && bound_serves(a.o.top_k, a.tops_of_row);
  if (dtype == ANN_F16)
    HIP_TRY(launch_sample<__half>(a, st));
  else if (dtype == ANN_BF16)
    HIP_TRY(launch_sample<__bf16>(a, st));
  else
    HIP_TRY(launch_sample<float>(a, st));
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

}  // extern "C"
