// One id drawn for each row of scores, by temperature, top-k, top-p and min-p.
//
// All three rules keep a prefix of the candidates sorted by (score downwards, id), so the kept ones are told by a
// cut: every key above it, and the first `ties` of those at it.  The cuts of top-k (by counts) and top-p (by
// masses) are found by histograms over ever shorter ranges of keys.  Masses are sums of weights rounded to multiples
// of a power of two: whole numbers, whose sums depend on no order.  The draw sums the kept weights in fp64 in a
// fixed order.
#include "mx.hpp"

namespace annmi {

constexpr u32 SAMPLE_THREADS = 1024;
constexpr u32 SAMPLE_WAVES = SAMPLE_THREADS / 64;
constexpr u32 SAMPLE_BINS = 1024;  // one for each thread
constexpr u32 SAMPLE_FEW = 1024;   // so many kept by top-k are sorted in LDS, and the row is not read again

struct SampleArgs {
  const char* scores;
  u64 ld, n;
  u32 rows;
  u32 unit;  // weights count in units of 2^-unit in the masses of top-p
  ann_sample_opts o;
  const float* uniform;
  u32* ids;
  float* logprobs;
};

constexpr u32 SAMPLE_LEAST = 0x007FFFFFu;  // float_key(-inf): candidates have larger keys

// low bits of a key that are the same in all values of one sign of a type
template <typename T>
constexpr u32 key_grain() {
  return sizeof(T) == 4 ? 0 : __is_same(T, __half) ? 13 : 16;
}

// exp((score - best) / temperature) to a few units of the last place: 2^(j / 256) from a table, the rest, below
// ln 2 / 512, by its series.
struct Weights {
  double best, scale;  // scale: 256 / (temperature ln 2)
  u32 best_key;
  const double* table;
  __device__ __forceinline__ double of(u32 key) const {
    if (key == best_key) return 1.0;
    double y = (static_cast<double>(key_float(key)) - best) * scale;
    y = y > -300000.0 ? y : -300000.0;  // (2^-1171: 0)
    const double whole = __builtin_rint(y), r = (y - whole) * 0.0027076061740622863;  // ln 2 / 256
    const int e = static_cast<int>(whole);
    const double p = __builtin_fma(__builtin_fma(__builtin_fma(__builtin_fma(r, 1.0 / 24, 1.0 / 6), r, 0.5), r, 1.0), r, 1.0);
    return ldexp(table[e & 255] * p, e >> 8);
  }
  // in units of 2^-unit, to the nearest; unit <= 50: adding 2^52 leaves the whole number in the low bits
  __device__ __forceinline__ u64 units(u32 key, double unit) const {
    return static_cast<u64>(__double_as_longlong(__builtin_fma(of(key), unit, 4503599627370496.0)) & 0xFFFFFFFFFFFFFll);
  }
};

// f(id, key) for the row's entries from..to, dealt to `ranks` threads: 16 bytes at a time, four loads on their way
// at once; before the first and after the last whole piece one by one.
template <typename T, typename F>
__device__ __forceinline__ void each(const T* row, u64 from, u64 to, u32 rank, u32 ranks, F f) {
  constexpr u32 V = 16 / sizeof(T), AHEAD = 4;
  const u64 skew = reinterpret_cast<uintptr_t>(row + from) % 16 / sizeof(T);
  const u64 head = min(to, from + (V - skew) % V);
  const u64 pieces = (to - head) / V, tail = head + pieces * V;
  for (u64 i = from + rank; i < head; i += ranks) f(i, float_key(mx_float(row[i])));
  for (u64 p = rank; p < pieces; p += (u64)ranks * AHEAD) {
    Pack<T, V> x[AHEAD];
#pragma unroll
    for (u32 u = 0; u < AHEAD; ++u) x[u] = *reinterpret_cast<const Pack<T, V>*>(row + head + min(p + (u64)u * ranks, pieces - 1) * V);
#pragma unroll
    for (u32 u = 0; u < AHEAD; ++u) {
      __builtin_amdgcn_sched_barrier(0);  // (or the weights of several pieces would be taken at once, in too many registers)
      if (p + (u64)u * ranks < pieces)
#pragma unroll
        for (u32 e = 0; e < V; ++e) f(head + (p + (u64)u * ranks) * V + e, float_key(mx_float(x[u].v[e])));
    }
  }
  for (u64 i = tail + rank; i < to; i += ranks) f(i, float_key(mx_float(row[i])));
}

struct SampleLds {
  u64 hist[SAMPLE_BINS];    // counts or masses; sorted candidates
  u64 weight[SAMPLE_BINS];  // of the candidates that are sorted (bits of doubles)
  double table[256];
  u64 wave[SAMPLE_WAVES];
  u64 word;
  u32 count, bin;
};

// sums over the workgroup in a fixed order, the same in every thread: of all, and of this thread's and those before
template <typename V>
__device__ V block_scan(V v, SampleLds& s, V* upto) {
  const u32 lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
  for (int w = 1; w < 64; w *= 2) {
    const V x = __shfl_up(v, w);
    if (lane >= (u32)w) v += x;
  }
  __syncthreads();
  if (lane == 63) s.wave[wave] = __builtin_bit_cast(u64, v);
  __syncthreads();
  V sum = V(0), before = V(0);
  for (u32 w = 0; w < SAMPLE_WAVES; ++w) {
    if (w == wave) before = sum;
    sum += __builtin_bit_cast(V, s.wave[w]);
  }
  *upto = before + v;
  return sum;
}

// s.hist[0 .. size) upwards; size: a power of two
__device__ void block_sort(SampleLds& s, u32 size) {
  for (u32 run = 2; run <= size; run *= 2)
    for (u32 gap = run / 2; gap > 0; gap /= 2) {
      __syncthreads();
      const u32 i = threadIdx.x;
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
  u64 at;    // how many there are (top-k only)
};

// A workgroup per row.  The row is read once for its best score, once to three times for each cut, once for the draw
// (and a sixteenth of it, and so on, to find the draw's place); all but the first time from the caches.
template <typename T>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(SampleArgs a) {
  __shared__ SampleLds s;
  const u32 tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  constexpr u32 GRAIN = key_grain<T>();
  if (tid < 256) s.table[tid] = exp2(tid / 256.0);
  for (u64 r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* row = reinterpret_cast<const T*>(a.scores) + r * a.ld;
    const float temperature = a.o.temperature_dev ? a.o.temperature_dev[r] : a.o.temperature;
    const u32 top_k = a.o.top_k_dev ? a.o.top_k_dev[r] : a.o.top_k;
    const float top_p = a.o.top_p_dev ? a.o.top_p_dev[r] : a.o.top_p;
    const float min_p = a.o.min_p_dev ? a.o.min_p_dev[r] : a.o.min_p;
    auto all = [&](auto f) { each(row, 0, a.n, tid, SAMPLE_THREADS, f); };

    u32 best = 0;
    all([&](u64, u32 key) { best = max(best, key); });
#pragma unroll
    for (int w = 1; w < 64; w *= 2) best = max(best, (u32)__shfl_xor((int)best, w));
    __syncthreads();
    if (lane == 0) s.wave[wave] = best;
    __syncthreads();
    for (u32 w = 0; w < SAMPLE_WAVES; ++w) best = max(best, (u32)s.wave[w]);
    if (best <= SAMPLE_LEAST) {  // (the same in all threads)
      if (tid == 0) {
        a.ids[r] = ANN_NONE;
        if (a.logprobs) a.logprobs[r] = -__builtin_inff();
      }
      continue;
    }
    if (!(temperature > 0.0f)) {
      if (tid == 0) s.word = ~0ull;
      __syncthreads();
      u64 first = ~0ull;
      all([&](u64 i, u32 key) {
        if (key == best) first = min(first, i);
      });
      if (first != ~0ull) atomicMin(reinterpret_cast<unsigned long long*>(&s.word), (unsigned long long)first);
      __syncthreads();
      if (tid == 0) {
        a.ids[r] = (u32)s.word;
        if (a.logprobs) a.logprobs[r] = 0.0f;
      }
      continue;
    }
    Weights w;
    w.best_key = best;
    w.best = static_cast<double>(key_float(best));
    // (an infinite temperature has scale 0; next to an infinite best score any other has weight 0 all the same)
    w.scale = w.best < __builtin_inf() ? 369.3299304675746 / static_cast<double>(temperature) : 1.0;
    w.table = s.table;
    const double unit = ldexp(1.0, (int)a.unit);
    Cut cut = {SAMPLE_LEAST + 1, ~0ull, ~0ull};

    // The first histogram is linear in the score, 32 bins for each unit of max(temperature, 1) below the best, the
    // last one open; equal scores share a bin, and the bins fall with the score.
    const float per_score = 32.0f / (temperature > 1.0f ? temperature : 1.0f), best_score = key_float(best);
    auto linear_bin = [&](u32 key) {
      const float z = (best_score - key_float(key)) * per_score;
      return key == best ? 0u : z < (float)(SAMPLE_BINS - 1) ? (u32)z : SAMPLE_BINS - 1;
    };
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
        all([&](u64, u32 key) {
          if (key < lo || key > hi || (some_ties && key == floor.key)) return;
          const u32 b = level ? (hi - key) >> shift : linear_bin(key);
          atomicAdd(reinterpret_cast<unsigned long long*>(&s.hist[b]), (unsigned long long)(mass ? w.units(key, unit) : 1ull));
        });
        __syncthreads();
        if (tid == 0 && some_ties && floor.key >= lo)
          s.hist[level ? (hi - floor.key) >> shift : linear_bin(floor.key)] += floor.ties * w.units(floor.key, unit);
        __syncthreads();
        const u64 mine = s.hist[tid];
        u64 upto;
        const u64 total = block_scan<u64>(mine, s, &upto);
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
            if (linear_bin(mid) >= b)
              x = mid;
            else
              y = mid - 1;
          }
          const u32 top = x;
          x = lo, y = top;
          while (x < y) {  // the smallest key whose bin is b
            const u32 mid = x + (y - x) / 2;
            if (linear_bin(mid) <= b)
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

    if (top_k > 0 && top_k < a.n) {
      Cut found;
      u64 ties;
      if (select(cut, false, [&](u64 total) { return (u64)top_k < total ? (u64)top_k : 0; }, &found, &ties)) {
        cut = found;
        cut.ties = ties;
      }
    }
    double u = static_cast<double>(a.uniform[r]);
    // (1 and above: no running mass exceeds it, so that the last kept one is taken; below 0 and NaN count as 0)
    u = !(u >= 0.0) ? 0.0 : u < 1.0 ? u : __builtin_inf();
    const double floor_w = min_p < 1.0f ? static_cast<double>(min_p) : 1.0;

    if (cut.ties != ~0ull && top_k - cut.ties + cut.at <= SAMPLE_FEW) {
      // Few: sorted by (key downwards, id), cut, then sorted by id and drawn from, a thread for each.
      __syncthreads();
      if (tid == 0) s.count = 0;
      __syncthreads();
      all([&](u64 i, u32 key) {
        if (key >= cut.key) s.hist[atomicAdd(&s.count, 1u)] = (u64)~key << 32 | i;
      });
      __syncthreads();
      u32 size = 2;
      while (size < s.count) size *= 2;
      if (tid >= s.count && tid < size) s.hist[tid] = ~0ull;
      block_sort(s, size);
      const bool mine = tid < top_k;
      const u64 entry = mine ? s.hist[tid] : 0;
      const u32 key = ~(u32)(entry >> 32);
      const double weight = mine ? w.of(key) : 0.0;
      u64 upto;
      const u64 units = mine ? w.units(key, unit) : 0;
      const u64 total = block_scan<u64>(units, s, &upto);
      bool keep = mine;
      if (top_p > 0.0f && top_p < 1.0f) keep = keep && (tid == 0 || (double)(upto - units) < static_cast<double>(top_p) * static_cast<double>(total));
      if (min_p > 0.0f) keep = keep && weight >= floor_w;
      __syncthreads();
      if (tid < size) s.hist[tid] = keep ? (entry & 0xFFFFFFFFull) << 32 | tid : ~0ull;
      s.weight[tid] = __builtin_bit_cast(u64, weight);
      block_sort(s, size);
      const bool there = tid < size && s.hist[tid] != ~0ull;
      const u32 from = there ? (u32)s.hist[tid] : 0;
      const double x = there ? __builtin_bit_cast(double, s.weight[from]) : 0.0;
      double run, others;
      const double sum = block_scan<double>(x, s, &run);
      // the mass without this one, not as a difference from the whole where it is the best: it may be all the mass
      double rest = block_scan<double>(from == 0 ? 0.0 : x, s, &others);
      const double aim = u * sum;
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
      continue;
    }

    if (top_p > 0.0f && top_p < 1.0f) {
      Cut found;
      u64 left;
      if (select(cut, true,
                 [&](u64 total) {
                   const u64 aim = (u64)ceil(static_cast<double>(top_p) * static_cast<double>(total));
                   return aim < 1 ? 1 : aim > total ? total : aim;
                 },
                 &found, &left)) {
        const u64 each_one = w.units(found.key, unit);
        const u64 need = each_one ? (left + each_one - 1) / each_one : ~0ull;
        cut.ties = found.key == cut.key ? min(cut.ties, need) : need;
        cut.key = found.key;
      }
    }
    if (min_p > 0.0f) {
      // weights fall with the key: the smallest key whose weight reaches the floor
      u32 lo = cut.key, hi = best;  // hi reaches it
      while (lo < hi) {
        const u32 mid = lo + (hi - lo) / 2;
        if (w.of(mid) >= floor_w)
          hi = mid;
        else
          lo = mid + 1;
      }
      if (hi > cut.key) cut.key = hi, cut.ties = ~0ull;
    }
    // Where only some of those at the cut are kept, they are the first ones by id: those below `tie_end`.
    u64 tie_end = a.n;
    if (cut.ties != ~0ull) {
      u64 seen = 0;
      for (u64 i0 = 0; i0 < a.n; i0 += SAMPLE_THREADS) {
        const u64 i = i0 + tid;
        const bool tie = i < a.n && float_key(mx_float(row[i])) == cut.key;
        const u64 votes = __ballot(tie);
        __syncthreads();
        if (lane == 0) s.wave[wave] = (u64)__popcll(votes);
        if (tid == 0) s.word = ~0ull;
        __syncthreads();
        u64 before = seen, here = 0;
        for (u32 v = 0; v < SAMPLE_WAVES; ++v) {
          if (v < wave) before += s.wave[v];
          here += s.wave[v];
        }
        before += __popcll(votes & ((1ull << lane) - 1));
        if (tie && before == cut.ties) s.word = i;
        __syncthreads();
        if (s.word != ~0ull) {
          tie_end = s.word;
          break;
        }
        seen += here;
      }
    }
    // The draw: the span that holds it is dealt to the waves in runs, whose masses tell which run it is.  The best
    // candidates' weights, 1 each, are kept apart, so that a mass that is nearly all the drawn one's loses nothing.
    u64 lo = 0, hi = a.n;
    double others = 0.0, bests = 0.0, aim = 0.0;
    while (true) {
      const bool whole = lo == 0 && hi == a.n;
      u64 run = (hi - lo + SAMPLE_WAVES - 1) / SAMPLE_WAVES;
      run = (run + 63) / 64 * 64;
      const u64 from = min(hi, lo + wave * run), to = min(hi, from + run);
      double mine = 0.0, ones = 0.0;
      each(row, from, to, lane, 64, [&](u64 i, u32 key) {
        if (key > cut.key || (key == cut.key && i < tie_end)) {
          if (key == best)
            ones += 1.0;
          else
            mine += w.of(key);
        }
      });
#pragma unroll
      for (int v = 1; v < 64; v *= 2) mine += __shfl_xor(mine, v), ones += __shfl_xor(ones, v);
      __syncthreads();
      if (lane == 0) s.wave[wave] = __builtin_bit_cast(u64, mine), s.hist[wave] = __builtin_bit_cast(u64, ones);
      __syncthreads();
      if (whole) {
        others = bests = 0.0;
        for (u32 v = 0; v < SAMPLE_WAVES; ++v) others += __builtin_bit_cast(double, s.wave[v]), bests += __builtin_bit_cast(double, s.hist[v]);
        aim = u * (bests + others);
      }
      u32 at = 0, last = 0;
      double before = 0.0, before_last = 0.0;
      bool found = false;
      for (at = 0; at < SAMPLE_WAVES; ++at) {
        const double mass = __builtin_bit_cast(double, s.wave[at]) + __builtin_bit_cast(double, s.hist[at]);
        if (mass > 0.0) {
          last = at;
          before_last = before;
          if (before + mass > aim) {
            found = true;
            break;
          }
        }
        before += mass;
      }
      if (!found) at = last, before = before_last;  // rounding: the last run that holds anything
      aim -= before;
      lo += at * run;
      hi = min(hi, lo + run);
      if (hi - lo <= SAMPLE_THREADS) break;
    }
    // the last span, a thread for each entry
    const u64 i = lo + tid;
    const u32 key = i < hi ? float_key(mx_float(row[i])) : 0;
    const double mine = i < hi && (key > cut.key || (key == cut.key && i < tie_end)) ? w.of(key) : 0.0;
    double run;
    block_scan<double>(mine, s, &run);
    if (tid == 0) s.word = ~0ull, s.count = 0;
    __syncthreads();
    if (mine > 0.0) {
      if (run > aim) atomicMin(reinterpret_cast<unsigned long long*>(&s.word), (unsigned long long)tid);
      atomicMax(&s.count, tid);
    }
    __syncthreads();
    if (tid == (s.word != ~0ull ? (u32)s.word : s.count)) {
      a.ids[r] = (u32)i;
      if (a.logprobs) a.logprobs[r] = static_cast<float>(-log1p((key == best ? bests - 1.0 + others : bests + others - mine) / mine));
    }
  }
}

}  // namespace annmi

using namespace annmi;

extern "C" {

int ann_sample_scratch(uint64_t rows, uint64_t n, uint64_t* bytes) try {
  if (!bytes) return fail(ANN_EINVAL, "null argument");
  if (rows > MX_MOST_ROWS || n < 1 || n > MX_MOST_ROWS) return fail(ANN_EINVAL, "ann_sample: n must be at least 1, rows and n below 2^31");
  *bytes = 0;
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
  hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid((u32)(rows < (1u << 20) ? rows : (1u << 20)));
  if (dtype == ANN_F16)
    hipLaunchKernelGGL(sample_kernel<__half>, grid, dim3(SAMPLE_THREADS), 0, st, a);
  else if (dtype == ANN_BF16)
    hipLaunchKernelGGL(sample_kernel<__bf16>, grid, dim3(SAMPLE_THREADS), 0, st, a);
  else
    hipLaunchKernelGGL(sample_kernel<float>, grid, dim3(SAMPLE_THREADS), 0, st, a);
  HIP_TRY(hipGetLastError());
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

}  // extern "C"
