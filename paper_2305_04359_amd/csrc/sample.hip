// One id drawn for each row of scores, by temperature, top-k, top-p and min-p.
//
// All three rules keep a prefix of the candidates sorted by (score downwards, id), so the kept ones are told by a
// cut: every key above it, and the first `ties` of those at it.  The cut of top-k comes from counts of keys, the
// cut of top-p from masses, both by a radix selection, eight bits of the key at a time.  Masses are sums of
// weights rounded to multiples of a power of two: whole numbers, whose sums depend on no order.  The draw then
// sums the kept weights in fp64 in a fixed order.
#include "mx.hpp"

namespace annmi {

constexpr u32 SAMPLE_THREADS = 1024;

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

template <typename T>
__device__ __forceinline__ u32 score_key(const T* row, u64 i) {
  return float_key(mx_float(row[i]));
}

struct RowRules {
  double best, inverse;  // of the temperature
  u32 best_key;
  __device__ double weight(u32 key) const {
    return key == best_key ? 1.0 : exp((static_cast<double>(key_float(key)) - best) * inverse);
  }
};

// the sum of `v` over the workgroup, the same in every thread; the order of the sum is fixed
__device__ double block_sum(double v, double* shared) {
#pragma unroll
  for (int w = 1; w < 64; w *= 2) v += __shfl_xor(v, w);
  __syncthreads();
  if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = v;
  __syncthreads();
  double sum = 0.0;
  for (u32 i = 0; i < SAMPLE_THREADS / 64; ++i) sum += shared[i];
  return sum;
}

struct Cut {
  u32 key;
  u64 ties;  // how many of the candidates at `key` are kept, the first ones by id
};

// A workgroup per row.
template <typename T>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(SampleArgs a) {
  __shared__ unsigned long long hist[256];
  __shared__ double sums[SAMPLE_THREADS / 64];
  __shared__ unsigned long long s_best, s_left, s_before, s_ties[SAMPLE_THREADS / 64];
  __shared__ u32 s_prefix;
  const u32 tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  for (u64 r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* row = reinterpret_cast<const T*>(a.scores) + r * a.ld;
    const float temperature = a.o.temperature_dev ? a.o.temperature_dev[r] : a.o.temperature;
    const u32 top_k = a.o.top_k_dev ? a.o.top_k_dev[r] : a.o.top_k;
    const float top_p = a.o.top_p_dev ? a.o.top_p_dev[r] : a.o.top_p;
    const float min_p = a.o.min_p_dev ? a.o.min_p_dev[r] : a.o.min_p;
    __syncthreads();
    if (tid == 0) s_best = 0;
    __syncthreads();
    // the best candidate: largest key, smallest id
    unsigned long long best = 0;
    for (u64 i = tid; i < a.n; i += SAMPLE_THREADS) {
      const u64 k = (u64)score_key(row, i) << 32 | (u32)~(u32)i;
      best = max(best, (unsigned long long)k);
    }
    atomicMax(&s_best, best);
    __syncthreads();
    best = s_best;
    RowRules rules;
    rules.best_key = (u32)(best >> 32);
    const u32 first = ~(u32)best;
    if (rules.best_key <= SAMPLE_LEAST || !(temperature > 0.0f)) {  // (the same in all threads)
      if (tid == 0) {
        const bool none = rules.best_key <= SAMPLE_LEAST;
        a.ids[r] = none ? ANN_NONE : first;
        if (a.logprobs) a.logprobs[r] = none ? -__builtin_inff() : 0.0f;
      }
      continue;
    }
    rules.best = static_cast<double>(key_float(rules.best_key));
    // (an infinite temperature has inverse 0; next to an infinite best score any other has weight 0 all the same)
    rules.inverse = rules.best < __builtin_inf() ? 1.0 / static_cast<double>(temperature) : 1.0;
    Cut cut = {SAMPLE_LEAST + 1, ~0ull};

    // Radix selection: the key at which the running count (mass), from the largest key down, reaches `aim`.
    auto select = [&](unsigned long long aim, bool mass, u32 limit_key, unsigned long long limit_ties) {
      // (limit: only the prefix up to it counts; its ties enter by number, since equal keys have equal weights)
      if (tid == 0) s_prefix = 0, s_left = aim;
      for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        const u32 prefix = s_prefix;
        for (u64 i = tid; i < a.n; i += SAMPLE_THREADS) {
          const u32 key = score_key(row, i);
          if (key <= SAMPLE_LEAST || key < limit_key || (shift < 24 && key >> (shift + 8) != prefix)) continue;
          if (!mass)
            atomicAdd(&hist[key >> shift & 255], 1ull);
          else if (key > limit_key)
            atomicAdd(&hist[key >> shift & 255], (unsigned long long)__builtin_rint(ldexp(rules.weight(key), (int)a.unit)));
        }
        __syncthreads();
        if (tid == 0) {
          if (mass && limit_ties && (shift == 24 || limit_key >> (shift + 8) == prefix))
            hist[limit_key >> shift & 255] += limit_ties * (unsigned long long)__builtin_rint(ldexp(rules.weight(limit_key), (int)a.unit));
          unsigned long long left = s_left;
          u32 b = 255;
          while (b > 0 && hist[b] < left) left -= hist[b--];
          s_left = left;
          s_prefix = prefix << 8 | b;
        }
        __syncthreads();
      }
    };

    auto count_at = [&](u32 key, bool above) {
      __syncthreads();
      if (tid == 0) s_before = 0;
      __syncthreads();
      unsigned long long mine = 0;
      for (u64 i = tid; i < a.n; i += SAMPLE_THREADS) {
        const u32 k = score_key(row, i);
        mine += above ? k > key : k == key;
      }
      atomicAdd(&s_before, mine);
      __syncthreads();
      const u64 c = s_before;
      __syncthreads();
      return c;
    };
    if (top_k > 0 && top_k < a.n) {
      const u64 candidates = count_at(SAMPLE_LEAST, true);
      if (top_k < candidates) {
        select(top_k, false, SAMPLE_LEAST + 1, 0);
        cut.key = s_prefix;
        cut.ties = s_left;
        __syncthreads();
      }
    }
    if (top_p > 0.0f && top_p < 1.0f) {
      // the mass of what is kept so far, in whole units
      const u64 at_cut = min(cut.ties, (u64)count_at(cut.key, false));
      __syncthreads();
      if (tid == 0) s_before = 0;
      __syncthreads();
      unsigned long long mine = 0;
      for (u64 i = tid; i < a.n; i += SAMPLE_THREADS) {
        const u32 key = score_key(row, i);
        if (key > cut.key) mine += (unsigned long long)__builtin_rint(ldexp(rules.weight(key), (int)a.unit));
      }
      atomicAdd(&s_before, mine);
      __syncthreads();
      const unsigned long long total = s_before + at_cut * (unsigned long long)__builtin_rint(ldexp(rules.weight(cut.key), (int)a.unit));
      __syncthreads();
      unsigned long long aim = (unsigned long long)ceil(static_cast<double>(top_p) * static_cast<double>(total));
      if (aim < 1) aim = 1;
      if (aim > total) aim = total;
      select(aim, true, cut.key, at_cut);
      const u32 key = s_prefix;
      const unsigned long long left = s_left;
      __syncthreads();
      const unsigned long long w = (unsigned long long)__builtin_rint(ldexp(rules.weight(key), (int)a.unit));
      const u64 need = w ? (left + w - 1) / w : ~0ull;
      cut.ties = key == cut.key ? min(cut.ties, need) : need;
      cut.key = key;
    }
    if (min_p > 0.0f) {
      const double floor_w = min_p < 1.0f ? static_cast<double>(min_p) : 1.0;
      // weights fall with the key: the smallest key whose weight reaches the floor
      u32 lo = cut.key, hi = rules.best_key;  // hi reaches it
      while (lo < hi) {
        const u32 mid = lo + (hi - lo) / 2;
        if (rules.weight(mid) >= floor_w)
          hi = mid;
        else
          lo = mid + 1;
      }
      if (hi > cut.key) cut.key = hi, cut.ties = ~0ull;
    }
    // The draw.  The mass other than the first candidate's is kept apart, so that a mass that is nearly all its own
    // loses nothing.
    const u64 at_cut = count_at(cut.key, false);
    const bool all_ties = cut.ties >= at_cut;
    // where only some of the ties are kept: they are the first ones by id, up to and without `tie_end`
    u64 tie_end = a.n;
    if (!all_ties) {
      // find the id of the tie number cut.ties, block by block
      u64 seen = 0;
      for (u64 i0 = 0; i0 < a.n; i0 += SAMPLE_THREADS) {
        const u64 i = i0 + tid;
        const bool tie = i < a.n && score_key(row, i) == cut.key;
        const u64 votes = __ballot(tie);
        __syncthreads();
        if (lane == 0) s_ties[wave] = (unsigned long long)__popcll(votes);
        if (tid == 0) s_left = ~0ull;
        __syncthreads();
        u64 before = seen, all = 0;
        for (u32 w = 0; w < SAMPLE_THREADS / 64; ++w) {
          if (w < wave) before += s_ties[w];
          all += s_ties[w];
        }
        before += __popcll(votes & ((1ull << lane) - 1));
        if (tie && before == cut.ties) s_left = i;
        __syncthreads();
        if (s_left != ~0ull) {
          tie_end = s_left;
          break;
        }
        seen += all;
      }
      __syncthreads();
    }
    auto kept_weight = [&](u64 i) {
      const u32 key = score_key(row, i);
      return key > cut.key || (key == cut.key && i < tie_end) ? rules.weight(key) : 0.0;
    };
    // Narrow the span that holds the draw: it is dealt to the waves in runs, whose sums tell which run it is.
    u64 lo = 0, hi = a.n;
    double rest = 0.0;  // mass other than the first candidate's
    {
      double mine = 0.0;
      for (u64 i = tid; i < a.n; i += SAMPLE_THREADS)
        if (i != first) mine += kept_weight(i);
      rest = block_sum(mine, sums);
    }
    double u = static_cast<double>(a.uniform[r]);
    // (1 and above: no running mass exceeds it, so that the last kept one is taken; below 0 and NaN count as 0)
    u = !(u >= 0.0) ? 0.0 : u < 1.0 ? u : __builtin_inf();
    double aim = u * (1.0 + rest);
    constexpr u32 WAVES = SAMPLE_THREADS / 64;
    while (hi - lo > SAMPLE_THREADS) {
      const u64 run = (hi - lo + WAVES - 1) / WAVES;
      const u64 from = lo + wave * run, to = min(hi, from + run);
      double mine = 0.0;
      for (u64 i = from + lane; i < to; i += 64) mine += kept_weight(i);
#pragma unroll
      for (int w = 1; w < 64; w *= 2) mine += __shfl_xor(mine, w);
      __syncthreads();
      if (lane == 0) sums[wave] = mine;
      __syncthreads();
      u32 w = 0, last = 0;
      double before = 0.0, before_last = 0.0;
      bool found = false;
      for (w = 0; w < WAVES; ++w) {
        if (sums[w] > 0.0) {
          last = w;
          before_last = before;
          if (before + sums[w] > aim) {
            found = true;
            break;
          }
        }
        before += sums[w];
      }
      if (!found) w = last, before = before_last;  // rounding: the last run that holds anything
      aim -= before;
      lo = lo + w * run;
      hi = min(hi, lo + run);
    }
    // the last span, a thread for each entry
    const u64 i = lo + tid;
    const double mine = i < hi ? kept_weight(i) : 0.0;
    double run = mine;
#pragma unroll
    for (int w = 1; w < 64; w *= 2) {
      const double x = __shfl_up(run, w);
      if (lane >= (u32)w) run += x;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = run;
    if (tid == 0) s_left = ~0ull, s_before = 0;
    __syncthreads();
    for (u32 w = 0; w < wave; ++w) run += sums[w];
    if (mine > 0.0) {
      if (run > aim) atomicMin(&s_left, (unsigned long long)i);
      atomicMax(&s_before, (unsigned long long)i);
    }
    __syncthreads();
    if (tid == 0) {
      const u64 id = s_left != ~0ull ? s_left : s_before;
      a.ids[r] = (u32)id;
      const double w = kept_weight(id);
      if (a.logprobs) a.logprobs[r] = static_cast<float>(-log1p((id == first ? rest : 1.0 + rest - w) / w));
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
