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
constexpr u64 SEARCH_SCRATCH_FLOATS = 1ull << 26;  // of group maxima held at a time, where 64 queries fit in them
constexpr u64 SEARCH_MOST_AT_ONCE = 1ull << 22;   // queries of a launch: its threads are counted in 32 bits

struct MxSearchArgs {
  MxRows w, q;
  const float* norms;   // null: inner products
  const float* qnorms;
  u32 q0, nq;           // the queries of this launch
  u32 groups, k;
  float* most;          // (nq, groups)
  u32* ids;
  float* dists;
};

__device__ __forceinline__ v4i load_codes(const MxRows& m, u64 row, u32 step) {
  return *reinterpret_cast<const v4i*>(m.codes + (row * m.steps + step) * MX_STEP_BYTES + threadIdx.x % 64 / 16 * 16);
}
__device__ __forceinline__ int load_scale(const MxRows& m, u64 row, u32 step) {
  return m.scales[(row * m.steps + step) * MX_STEP_SCALES + threadIdx.x % 64 / 16];
}

// what the sums of rows row0 .. row0 + 3 start from: 0, or - |x|^2 / 2
__device__ __forceinline__ v4f first_sum(const MxSearchArgs& a, u64 row0) {
  v4f c = {};
  if (a.norms)
#pragma unroll
    for (int r = 0; r < 4; ++r) c[r] = -0.5f * a.norms[min(row0 + r, (u64)a.w.n - 1)];
  return c;
}

// A wave: 64 rows (a group) x 64 queries.
__global__ __launch_bounds__(256) void mx_group_most_kernel(MxSearchArgs a, u64 tiles) {
  const u32 lane = threadIdx.x % 64;
  const u64 t = (u64)blockIdx.x * 4 + threadIdx.x / 64;
  if (t >= tiles) return;
  const u64 g = t % a.groups, w0 = g * SEARCH_GROUP;
  const u64 x0 = t / a.groups * 64;
  v4f acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const v4f c = first_sum(a, w0 + 16 * i + lane / 16 * 4);
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
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (w0 + 16 * i + lane / 16 * 4 + r < a.w.n) m = __builtin_fmaxf(m, acc[i][j][r]);
    m = __builtin_fmaxf(m, __shfl_xor(m, 16));
    m = __builtin_fmaxf(m, __shfl_xor(m, 32));
    const u64 x = x0 + 16 * j + lane;
    if (lane < 16 && x < a.nq) a.most[x * a.groups + g] = m;
  }
}

// A workgroup per query: the first k groups by a radix selection on the keys of their maxima, eight bits at a time;
// their rows' scores; the k best of those that reach the last group's maximum, sorted.
__global__ __launch_bounds__(256) void mx_pick_kernel(MxSearchArgs a) {
  extern __shared__ u64 found[];  // as many as the rows of k groups, up to a power of two for the sort
  __shared__ u32 hist[256];
  __shared__ u32 chosen[SEARCH_MOST_K];
  __shared__ u32 s_prefix, s_left, s_count, s_scan[4];
  const u32 tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const u32 q = blockIdx.x;
  const float* most = a.most + (u64)q * a.groups;
  const u32 least = float_key(-__builtin_inff());  // keys up to this one are of groups without a score

  // the k-th largest key
  if (tid == 0) s_prefix = 0, s_left = min(a.k, a.groups), s_count = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    hist[tid] = 0;
    __syncthreads();
    const u32 prefix = s_prefix;
    for (u32 i = tid; i < a.groups; i += 256) {
      const u32 key = float_key(most[i]);
      if (shift == 24 || key >> (shift + 8) == prefix) atomicAdd(&hist[key >> shift & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      u32 left = s_left, b = 255;
      while (b > 0 && hist[b] < left) left -= hist[b--];
      s_left = left;
      s_prefix = prefix << 8 | b;
    }
    __syncthreads();
  }
  const u32 cut = s_prefix, ties = s_left;  // groups above the cut, and the first `ties` of those at it
  __syncthreads();
  if (tid == 0) s_left = 0;
  __syncthreads();
  // in the order of groups, so that the ties taken are the first ones
  for (u32 i0 = 0; i0 < a.groups; i0 += 256) {
    const u32 i = i0 + tid;
    const u32 key = i < a.groups ? float_key(most[i]) : 0u;
    const bool tie = key == cut && key > least;
    const u64 votes = __ballot(tie);
    if (lane == 0) s_scan[wave] = (u32)__popcll(votes);
    __syncthreads();
    u32 before = s_left + (u32)__popcll(votes & ((1ull << lane) - 1));
    for (u32 w = 0; w < wave; ++w) before += s_scan[w];
    if (i < a.groups && ((key > cut && key > least) || (tie && before < ties))) chosen[atomicAdd(&s_count, 1u)] = i;
    __syncthreads();
    if (tid == 0) s_left += s_scan[0] + s_scan[1] + s_scan[2] + s_scan[3];
    __syncthreads();
  }
  const u32 nchosen = s_count;
  __syncthreads();
  if (tid == 0) s_count = 0;
  __syncthreads();
  // k groups: k points reach the smallest of their maxima, and no other point matters
  const u32 low = nchosen == a.k ? max(cut, least + 1) : least + 1;
  const u64 qrow = (u64)a.q0 + q;
  for (u32 c = wave; c < nchosen * 4; c += 4) {  // 16 rows at a time
    const u64 w0 = (u64)chosen[c / 4] * SEARCH_GROUP + c % 4 * 16;
    const u64 wr = min(w0 + lane % 16, (u64)a.w.n - 1);
    v4f acc = first_sum(a, w0 + lane / 16 * 4);
    for (u32 s = 0; s < a.w.steps; ++s)
      acc = mx_mfma(load_codes(a.w, wr, s), load_codes(a.q, qrow, s), acc, load_scale(a.w, wr, s), load_scale(a.q, qrow, s));
    // (all columns are this query's: one of them is used)
    if (lane % 16 == 0)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const u64 id = w0 + lane / 16 * 4 + r;
        const u32 key = float_key(acc[r]);
        if (id < a.w.n && key >= low) found[atomicAdd(&s_count, 1u)] = (u64)~key << 32 | id;
      }
  }
  __syncthreads();
  const u32 count = s_count;
  u32 size = 2;
  while (size < count) size *= 2;
  for (u32 i = count + tid; i < size; i += 256) found[i] = ~0ull;
  __syncthreads();
  for (u32 run = 2; run <= size; run *= 2)
    for (u32 gap = run / 2; gap > 0; gap /= 2) {
      for (u32 i = tid; i < size / 2; i += 256) {
        const u32 lo = i / gap * 2 * gap + i % gap, hi = lo + gap;
        const u64 x = found[lo], y = found[hi];
        if ((x > y) == ((lo & run) == 0)) found[lo] = y, found[hi] = x;
      }
      __syncthreads();
    }
  for (u32 i = tid; i < a.k; i += 256) {
    const u64 at = qrow * a.k + i;
    if (i < count) {
      const float s = key_float(~(u32)(found[i] >> 32));
      a.ids[at] = (u32)found[i];
      a.dists[at] = a.norms ? __builtin_fmaxf(0.0f, __builtin_fmaf(-2.0f, s, a.qnorms[qrow])) : 0.0f - s;
    } else {
      a.ids[at] = ANN_NONE;
      a.dists[at] = __builtin_inff();
    }
  }
}

u64 search_queries_at_once(u64 groups, u64 nq) {
  u64 most = SEARCH_SCRATCH_FLOATS / groups / 64 * 64;
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
  const u64 groups = (n + SEARCH_GROUP - 1) / SEARCH_GROUP;
  return groups == 0 ? 0 : (search_queries_at_once(groups, nq) * groups * 4 + 15) / 16 * 16;
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
  const u64 part = search_queries_at_once(a.groups, nq);
  size_t room = 2;
  while (room < (size_t)(k < a.groups ? k : a.groups) * SEARCH_GROUP) room *= 2;
  room *= 8;
  HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(mx_pick_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)room));
  for (u64 q0 = 0; q0 < nq; q0 += part) {
    a.q0 = (u32)q0;
    a.nq = (u32)(nq - q0 < part ? nq - q0 : part);
    const u64 tiles = a.groups * (((u64)a.nq + 63) / 64);
    hipLaunchKernelGGL(mx_group_most_kernel, dim3((u32)((tiles + 3) / 4)), dim3(256), 0, st, a, tiles);
    HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL(mx_pick_kernel, dim3(a.nq), dim3(256), room, st, a);
    HIP_TRY(hipGetLastError());
  }
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

}  // extern "C"
