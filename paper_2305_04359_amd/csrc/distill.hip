// The loss of scores against a teacher's best entries of each row, and its gradient.
//
// With T the temperature, of a row of scores z and its teacher's entries (id_j, t_j):
//   p_j  = exp((t_j - max t) / T) / P        over the entries that are there, P the sum
//   q_i  = exp((z_i - m) / T) / S            over the whole row, m = max z, S the sum
//   loss = T^2 sum_j p_j (log p_j - log q_id_j) = T^2 (sum_j p_j ((t_j - max t) - (z_id_j - m)) / T + log S - log P)
//   d loss / d z_i = T (q_i - sum over j with id_j = i of p_j)
// One pass over the scores makes m and S together: a thread keeps the maximum so far and the sum relative to it.  The loss
// is made of the teacher's few entries in 64 bits; m and S stay with the caller for the gradient, which takes one more
// pass and writes every score's once, rounded once.
#include <algorithm>

#include "mx.hpp"

namespace annmi {

constexpr u32 DISTILL_MOST_K = 1024;
constexpr u32 DISTILL_THREADS = 256;
constexpr u64 DISTILL_MOST_PLACE = 1ull << 60;  // elements from a matrix's beginning: 64 bits hold their bytes

struct DistillArgs {
  const char* scores;
  u64 rows;
  u32 n;
  u64 ld;
  const u32* ids;
  const char* teacher;
  int tdtype;
  u32 k;
  float t, c;  // temperature; log2(e) / temperature
  float* losses;
  float* stats;  // m and S of every row
  float* parts;  // the same of every part of a row, where rows are divided
  u32 chunks, chunk;
  // gradient
  const float* upstream;
  float scale;
  char* out;
  u64 ldo;
};

// a maximum and the sum of exp2((z - maximum) c) below it; nothing yet: -inf and 0
struct Soft {
  float m, s;
};
__device__ __forceinline__ float soft_exp(float z, float m, float c) { return __builtin_amdgcn_exp2f((z - m) * c); }
// (maxima of -inf leave sums of 0 or NaN as they are)
__device__ __forceinline__ Soft soft_join(Soft a, Soft b, float c) {
  const float m = __builtin_fmaxf(a.m, b.m);
  const float to = m == -INFINITY ? 0.0f : m;
  return {m, a.s * soft_exp(a.m, to, c) + b.s * soft_exp(b.m, to, c)};
}

// 16 bytes wherever they begin.  Gradients go past the caches, and scores that are more than these hold (PAST) come past
// them, so that they do not drive out what is needed.  Loss and gradient with scores read so, and not: 4,096 x 128,000 bf16
// (1 GB) 546 us and 627, 2,500 x 50,001 fp32 (500 MB) 269 and 285, 1,500 (300 MB) 166 and 146, 700 (140 MB) 82 and 70.  With gradients
// written the plain way 1,500 x 50,001 fp32 take 179 us, 147 so.
constexpr u64 DISTILL_PAST = 384ull << 20;
using Streamed = v4i __attribute__((aligned(2)));
template <bool PAST, int E, typename T>
__device__ __forceinline__ AnyPack<T, E> stream_in(const T* from) {
  static_assert(E * sizeof(T) == 16);
  if constexpr (PAST) return __builtin_bit_cast(AnyPack<T, E>, v4i(__builtin_nontemporal_load(reinterpret_cast<const Streamed*>(from))));
  return *reinterpret_cast<const AnyPack<T, E>*>(from);
}
template <int E, typename T>
__device__ __forceinline__ void stream_out(T* to, const AnyPack<T, E>& v) {
  __builtin_nontemporal_store(__builtin_bit_cast(v4i, v), reinterpret_cast<Streamed*>(to));
}

template <typename T>
__device__ __forceinline__ float distill_float(const char* at, u64 i) {
  return mx_float(reinterpret_cast<const T*>(at)[i]);
}
__device__ __forceinline__ float teacher_at(const DistillArgs& a, u64 i) {
  return a.tdtype == ANN_F32 ? distill_float<float>(a.teacher, i) : a.tdtype == ANN_F16 ? distill_float<__half>(a.teacher, i) : distill_float<__bf16>(a.teacher, i);
}

// What a thread sees of entries [from, to) of a row: every 256th pack of 16 bytes, four at a time.  What is lost when such a
// turn's sum is added to those before it is kept: one weight after another, thousands of equal ones (520 rows of 2^22 scores of 0 and
// -0.25) would leave the row's sum off by 2e-4 of itself, and more the longer the row.
template <bool PAST, typename T>
__device__ __forceinline__ Soft soft_scan(const T* z, u32 from, u32 to, float c) {
  constexpr u32 E = 16 / sizeof(T), AHEAD = 4;
  Soft mine = {-INFINITY, 0.0f};
  float more = 0.0f;  // that the sum has too much
  const u32 packs = (to - from) / E;
  auto take = [&](const float* v, u32 count) {
    float m = mine.m;
    for (u32 e = 0; e < count; ++e) m = __builtin_fmaxf(m, v[e]);
    const float base = m == -INFINITY ? 0.0f : m;
    float turn = 0.0f;
    for (u32 e = 0; e < count; ++e) turn += soft_exp(v[e], base, c);
    const float to_new = soft_exp(mine.m, base, c), before = mine.s * to_new, add = turn - more * to_new;
    const float s = before + add;
    more = (s - before) - add;
    mine = {m, s};
  };
  for (u32 p = threadIdx.x; p < packs; p += DISTILL_THREADS * AHEAD) {
    float v[E * AHEAD];
#pragma unroll
    for (u32 u = 0; u < AHEAD; ++u) {
      const u32 at = p + DISTILL_THREADS * u;
      const AnyPack<T, E> in = stream_in<PAST, E>(z + from + (u64)min(at, packs - 1) * E);
#pragma unroll
      for (u32 e = 0; e < E; ++e) v[u * E + e] = at < packs ? mx_float(static_cast<T>(in.v[e])) : -INFINITY;
    }
    take(v, E * AHEAD);
  }
  const u32 left = from + packs * E + threadIdx.x;
  if (left < to) {
    const float v = mx_float(z[left]);
    take(&v, 1);
  }
  return mine;
}

// the whole workgroup's, in every thread
__device__ __forceinline__ Soft soft_block(Soft v, float c, Soft* room) {
#pragma unroll
  for (int w = 1; w < 64; w *= 2) v = soft_join(v, {__shfl_xor(v.m, w), __shfl_xor(v.s, w)}, c);
  __syncthreads();  // (the room's last readers)
  if (threadIdx.x % 64 == 0) room[threadIdx.x / 64] = v;
  __syncthreads();
  v = room[0];
#pragma unroll
  for (u32 w = 1; w < DISTILL_THREADS / 64; ++w) v = soft_join(v, room[w], c);
  return v;
}

__device__ __forceinline__ double block_sum(double v, double* room) {
#pragma unroll
  for (int w = 1; w < 64; w *= 2) v += __shfl_xor(v, w);
  __syncthreads();
  if (threadIdx.x % 64 == 0) room[threadIdx.x / 64] = v;
  __syncthreads();
  v = room[0];
#pragma unroll
  for (u32 w = 1; w < DISTILL_THREADS / 64; ++w) v += room[w];
  return v;
}
__device__ __forceinline__ float block_max(float v, float* room) {
#pragma unroll
  for (int w = 1; w < 64; w *= 2) v = __builtin_fmaxf(v, __shfl_xor(v, w));
  __syncthreads();
  if (threadIdx.x % 64 == 0) room[threadIdx.x / 64] = v;
  __syncthreads();
  v = room[0];
#pragma unroll
  for (u32 w = 1; w < DISTILL_THREADS / 64; ++w) v = __builtin_fmaxf(v, room[w]);
  return v;
}

struct DistillRoom {
  Soft soft[4];
  double sums[4];
  float most[4];
};

// the teacher's j-th score of a row, -inf where its entry is not there; and the entry
__device__ __forceinline__ float teacher_entry(const DistillArgs& a, u64 row, u32 j, u32* id) {
  *id = a.ids[row * a.k + j];
  return *id < a.n ? teacher_at(a, row * a.k + j) : -INFINITY;
}

// A row's loss from its m and S, by a workgroup.
template <typename T>
__device__ __forceinline__ void distill_finish(const DistillArgs& a, u64 row, Soft all, DistillRoom& room) {
  const T* z = reinterpret_cast<const T*>(a.scores) + row * a.ld;
  u32 id;
  float most = -INFINITY;
#pragma unroll 1
  for (u32 j = threadIdx.x; j < a.k; j += DISTILL_THREADS) most = __builtin_fmaxf(most, teacher_entry(a, row, j, &id));
  most = block_max(most, room.most);
  double weights = 0.0, terms = 0.0;
#pragma unroll 1
  for (u32 j = threadIdx.x; j < a.k; j += DISTILL_THREADS) {
    const float t = teacher_entry(a, row, j, &id);
    if (t == -INFINITY) continue;
    const double off = ((double)t - most) / a.t, w = exp(off);
    weights += w;
    if (!(w == 0.0)) terms += w * (off - ((double)mx_float(z[id]) - all.m) / a.t);
  }
  weights = block_sum(weights, room.sums);
  terms = block_sum(terms, room.sums);
  if (threadIdx.x == 0) {
    double loss = (double)a.t * a.t * (terms / weights + log((double)all.s) - log(weights));
    if (weights == 0.0 || all.s == 0.0f) loss = 0.0;  // no teacher, or no score that is not masked
    a.losses[row] = (float)loss;
    a.stats[2 * row] = all.m;
    a.stats[2 * row + 1] = all.s;
  }
}

// Rows by a workgroup each, or by one for each of their chunks, which leaves its part's m and S.
template <typename T, bool WHOLE, bool PAST>
__global__ __launch_bounds__(DISTILL_THREADS) void distill_scan_kernel(DistillArgs a) {
  __shared__ DistillRoom room;
  for (u64 b = blockIdx.x; b < a.rows * a.chunks; b += gridDim.x) {
    const u64 row = WHOLE ? b : b / a.chunks;
    const u32 part = WHOLE ? 0 : (u32)(b % a.chunks);
    const u32 from = part * a.chunk, to = WHOLE ? a.n : min(from + a.chunk, a.n);
    const Soft all = soft_block(soft_scan<PAST>(reinterpret_cast<const T*>(a.scores) + row * a.ld, from, to, a.c), a.c, room.soft);
    if constexpr (WHOLE) {
      distill_finish<T>(a, row, all, room);
    } else if (threadIdx.x == 0) {
      a.parts[2 * b] = all.m;
      a.parts[2 * b + 1] = all.s;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(DISTILL_THREADS) void distill_finish_kernel(DistillArgs a) {
  __shared__ DistillRoom room;
  for (u64 row = blockIdx.x; row < a.rows; row += gridDim.x) {
    Soft all = {-INFINITY, 0.0f};
    for (u32 c = threadIdx.x; c < a.chunks; c += DISTILL_THREADS) {
      const float* part = a.parts + 2 * (row * a.chunks + c);
      all = soft_join(all, {part[0], part[1]}, a.c);
    }
    all = soft_block(all, a.c, room.soft);
    distill_finish<T>(a, row, all, room);
  }
}

// The gradient of a chunk of a row.  The teacher's shares are made anew by every workgroup (k is small); entries of the
// teacher inside the chunk are read before and written after all others, by the first thread that holds their id,
// which adds up the shares of the same id in their order.  So `out` may be the scores themselves.  Up to 64 entries lie one a lane
// in the first wave, which compares them while the gradients are on their way (37 rows of 10,000 fp32 with k = 64 8.0 us, from LDS
// 10.7).  Of more a table tells whether any id is there twice: without it 1,000 rows of 20,000 bf16 with k = 1,000 take 247 us,
// with it 33.  Of many rows a workgroup takes 32 KB: 4,096 x 128,000 bf16 374 us, 2,000 x 50,001 fp32 157; 16 KB 385 and 151,
// 64 KB 386 and 173, whole rows 410 and 189.
constexpr u32 DISTILL_FEW = 64, DISTILL_TABLE = 2 * DISTILL_MOST_K, GRAD_CHUNK = 32768;
template <typename T, bool PAST>
__global__ __launch_bounds__(DISTILL_THREADS) void distill_grad_kernel(DistillArgs a) {
  constexpr u32 E = 16 / sizeof(T), AHEAD = 4;
  __shared__ DistillRoom room;
  __shared__ u32 ids[DISTILL_MOST_K];  // ANN_NONE outside of the chunk
  __shared__ float shares[DISTILL_MOST_K], kept[DISTILL_MOST_K];
  __shared__ u32 table[DISTILL_TABLE], twice;
  for (u64 b = blockIdx.x; b < a.rows * a.chunks; b += gridDim.x) {
    const u64 row = b / a.chunks;
    const u32 from = (u32)(b % a.chunks) * a.chunk, to = min(from + a.chunk, a.n);
    const T* z = reinterpret_cast<const T*>(a.scores) + row * a.ld;
    T* out = reinterpret_cast<T*>(a.out) + row * a.ldo;
    const float m = a.stats[2 * row], s = a.stats[2 * row + 1];
    const bool few = a.k <= DISTILL_FEW;
    double weights = 0.0;
    u32 id;
    float own_kept = 0.0f, own_share = 0.0f;  // of the entry that a thread writes last, where there are few
    u32 own_id = ANN_NONE;
    if (few) {  // every wave makes them by itself, and holds an entry a lane
      const u32 j = threadIdx.x % 64;
      float t = -INFINITY;
      u32 mine = ANN_NONE;
      if (j < a.k) {
        t = teacher_entry(a, row, j, &id);
        if (id >= from && id < to) mine = id;
        if (mine != ANN_NONE) own_kept = mx_float(z[mine]);
      }
      float most = t;
#pragma unroll
      for (int w = 1; w < 64; w *= 2) most = __builtin_fmaxf(most, __shfl_xor(most, w));
      const float share = t == -INFINITY ? 0.0f : soft_exp(t, most, a.c);
      weights = share;
#pragma unroll
      for (int w = 1; w < 64; w *= 2) weights += __shfl_xor(weights, w);
      own_id = mine;
      own_share = share;
      asm volatile("" : "+v"(own_kept));  // the scores kept are there before any wave writes where they were
      __syncthreads();
    } else {
      for (u32 i = threadIdx.x; i < DISTILL_TABLE; i += DISTILL_THREADS) table[i] = ANN_NONE;
      if (threadIdx.x == 0) twice = 0;
      float most = -INFINITY;
#pragma unroll 1
      for (u32 j = threadIdx.x; j < a.k; j += DISTILL_THREADS) {
        const float t = teacher_entry(a, row, j, &id);
        most = __builtin_fmaxf(most, t);
        shares[j] = t;
        const bool here = id >= from && id < to;
        ids[j] = here ? id : ANN_NONE;
        if (here) kept[j] = mx_float(z[id]);
      }
      most = block_max(most, room.most);
#pragma unroll 1
      for (u32 j = threadIdx.x; j < a.k; j += DISTILL_THREADS) {  // (a thread's own ones)
        const float t = shares[j], w = t == -INFINITY ? 0.0f : soft_exp(t, most, a.c);
        shares[j] = w;
        weights += w;
        if (ids[j] != ANN_NONE)
          for (u32 at = ids[j] * 2654435761u;; ++at) {  // (the table has twice the room of all ids)
            const u32 there = atomicCAS(&table[at % DISTILL_TABLE], ANN_NONE, ids[j]);
            if (there == ids[j]) twice = 1;
            if (there == ids[j] || there == ANN_NONE) break;
          }
      }
      weights = block_sum(weights, room.sums);
    }
    const bool none = weights == 0.0 || s == 0.0f;
    const float over = (float)(1.0 / weights);
    const float up = a.t * a.scale * (a.upstream ? a.upstream[row] : 1.0f);
    const float base = m == -INFINITY ? 0.0f : m, share = 1.0f / s;
    auto grad = [&](float v, float p) { return mx_round<T>(none ? 0.0f : up * (soft_exp(v, base, a.c) * share - p)); };
    const u32 packs = (to - from) / E;
    for (u32 p = threadIdx.x; p < packs; p += DISTILL_THREADS * AHEAD) {
      AnyPack<T, E> in[AHEAD];
#pragma unroll
      for (u32 u = 0; u < AHEAD; ++u) in[u] = stream_in<PAST, E>(z + from + (u64)min(p + DISTILL_THREADS * u, packs - 1) * E);
#pragma unroll
      for (u32 u = 0; u < AHEAD; ++u) {
        if (p + DISTILL_THREADS * u >= packs) break;
        AnyPack<T, E> o;
#pragma unroll
        for (u32 e = 0; e < E; ++e) o.v[e] = grad(mx_float(static_cast<T>(in[u].v[e])), 0.0f);
        stream_out<E>(out + from + (u64)(p + DISTILL_THREADS * u) * E, o);
      }
    }
    const u32 left = from + packs * E + threadIdx.x;
    if (left < to) out[left] = grad(mx_float(z[left]), 0.0f);
    if (few) {
      bool first = threadIdx.x < 64 && own_id != ANN_NONE;
      float p = 0.0f;
      if (__any(first))  // shares of one id are added up in their order, and written by the first lane that holds it
        for (u32 i = 0; i < a.k; ++i) {
          const bool same = (u32)__builtin_amdgcn_readlane((int)own_id, (int)i) == own_id;
          const float other = __uint_as_float((u32)__builtin_amdgcn_readlane((int)__float_as_uint(own_share), (int)i));
          p += same ? other * over : 0.0f;
          first = first && !(same && i < threadIdx.x);
        }
      __syncthreads();  // the teacher's entries come last
      if (first) out[own_id] = grad(own_kept, p);
      continue;
    }
    __syncthreads();  // the teacher's entries come last
#pragma unroll 1
    for (u32 j = threadIdx.x; j < a.k; j += DISTILL_THREADS) {
      const u32 mine = ids[j];
      if (mine == ANN_NONE) continue;
      float p = shares[j] * over;
      bool first = true;
      if (twice) {
        p = 0.0f;
        for (u32 i = 0; i < a.k; ++i) {
          if (ids[i] != mine) continue;
          first = first && i >= j;
          p += shares[i] * over;
        }
      }
      if (first) out[mine] = grad(kept[j], p);
    }
    __syncthreads();  // (the next row's ids and shares)
  }
}

// Workgroups for a row: more than one where rows are long and too few for the chip, of at least 8,192 entries each.  Loss and
// gradient of 37 rows of 10,000 fp32 whole 10.7 us, in two 13.0; of one row of 30,000 bf16 in four 12.7 us, in two 13.9, whole 14.6.
u32 distill_chunks(u64 rows, u64 n) {
  const u64 want = rows >= 512 || n <= 16384 ? 1 : 1024 / rows, most = (n + 8191) / 8192;
  return (u32)std::max<u64>(1, std::min(want, most));
}
void set_chunks(DistillArgs& a) {
  a.chunks = distill_chunks(a.rows, a.n);
  a.chunk = (a.n + a.chunks - 1) / a.chunks;
  a.chunk = (a.chunk + 7) / 8 * 8;  // (whole packs; the last one is shorter, and none is empty: 8 chunks < 8,192)
  a.chunks = (a.n + a.chunk - 1) / a.chunk;
}

template <typename T, bool PAST>
hipError_t launch_distill(const DistillArgs& a, hipStream_t s) {
  const u64 blocks = a.rows * a.chunks;
  const dim3 grid((u32)std::min<u64>(blocks, 1u << 22)), threads(DISTILL_THREADS);
  if (a.chunks == 1) {
    hipLaunchKernelGGL((distill_scan_kernel<T, true, PAST>), grid, threads, 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((distill_scan_kernel<T, false, PAST>), grid, threads, 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(distill_finish_kernel<T>, dim3((u32)a.rows), threads, 0, s, a);  // (fewer than 512 rows)
  return hipGetLastError();
}
template <typename T, bool PAST>
hipError_t launch_distill_grad(const DistillArgs& a, hipStream_t s) {
  const u64 blocks = a.rows * a.chunks;
  hipLaunchKernelGGL((distill_grad_kernel<T, PAST>), dim3((u32)std::min<u64>(blocks, 1u << 22)), dim3(DISTILL_THREADS), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_distill(const DistillArgs& a, bool grad, hipStream_t s) {
  if (a.rows * a.n * sizeof(T) > DISTILL_PAST) return grad ? launch_distill_grad<T, true>(a, s) : launch_distill<T, true>(a, s);
  return grad ? launch_distill_grad<T, false>(a, s) : launch_distill<T, false>(a, s);
}
int launch_distill(const DistillArgs& a, int dtype, bool grad, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == ANN_F32)
    HIP_TRY(launch_distill<float>(a, grad, st));
  else if (dtype == ANN_F16)
    HIP_TRY(launch_distill<__half>(a, grad, st));
  else
    HIP_TRY(launch_distill<__bf16>(a, grad, st));
  return ANN_OK;
}

// what both calls check; false in *work where there is nothing to do
int check_distill(const char* what, const void* scores, u64 rows, u64 n, int dtype, u64 ld, const uint32_t* ids, const void* teacher, int tdtype, u32 k,
                  float temperature, const float* stats, bool* work) {
  *work = false;
  const u64 esz = dtype_bytes(dtype), tsz = dtype_bytes(tdtype);
  if (esz < 2 || tsz < 2) return fail(ANN_EINVAL, "%s: scores and teacher must be ANN_F32, ANN_F16 or ANN_BF16", what);
  if (rows >= 1ull << 31) return fail(ANN_EINVAL, "%s: rows must stay below 2^31", what);
  if (n < 1 || n >= 1ull << 31) return fail(ANN_EINVAL, "%s: n must be 1 to 2^31 - 1", what);
  if (k < 1 || k > DISTILL_MOST_K) return fail(ANN_EINVAL, "%s: k must be 1 to %u", what, DISTILL_MOST_K);
  if (ld < n) return fail(ANN_EINVAL, "%s: ld must be at least n", what);
  if (rows && ld > DISTILL_MOST_PLACE / rows) return fail(ANN_EINVAL, "%s: rows * ld must be at most 2^60", what);
  // (log2(e) / T and T^2 then are ordinary numbers)
  if (!(temperature >= 0x1p-60f && temperature <= 0x1p60f)) return fail(ANN_EINVAL, "%s: temperature must be 2^-60 to 2^60", what);
  if (rows == 0) return ANN_OK;
  if (!scores || !ids || !teacher || !stats) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(scores, esz) || !aligned_to(teacher, tsz) || !aligned_to(ids, 4) || !aligned_to(stats, 4))
    return fail(ANN_EINVAL, "%s: an array is not aligned to its elements", what);
  *work = true;
  return ANN_OK;
}

}  // namespace annmi

using namespace annmi;

extern "C" {

int ann_distill_scratch(uint64_t rows, uint64_t n, uint64_t* bytes) try {
  if (!bytes) return fail(ANN_EINVAL, "null argument");
  if (rows >= 1ull << 31) return fail(ANN_EINVAL, "rows must stay below 2^31");
  if (n < 1 || n >= 1ull << 31) return fail(ANN_EINVAL, "n must be 1 to 2^31 - 1");
  const u32 chunks = rows ? distill_chunks(rows, n) : 1;
  *bytes = chunks > 1 ? rows * chunks * 8 : 0;
  return ANN_OK;
} catch (...) {
  return annmi::on_exception();
}

int ann_distill(const void* scores_dev, uint64_t rows, uint64_t n, ann_dtype dtype, uint64_t ld, const uint32_t* ids_dev,
                const void* teacher_dev, ann_dtype teacher_dtype, uint32_t k, float temperature, float* losses_dev,
                float* stats_dev, void* scratch_dev, uint64_t scratch_bytes, void* stream) try {
  bool work;
  int rc = check_distill("ann_distill", scores_dev, rows, n, dtype, ld, ids_dev, teacher_dev, teacher_dtype, k, temperature, stats_dev, &work);
  if (rc || !work) return rc;
  if (!losses_dev) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(losses_dev, 4)) return fail(ANN_EINVAL, "losses not aligned to their elements");
  uint64_t need = 0;
  rc = ann_distill_scratch(rows, n, &need);
  if (rc) return rc;
  if (need && (!scratch_dev || scratch_bytes < need)) return fail(ANN_EINVAL, "scratch must hold %llu bytes", (unsigned long long)need);
  if (need && !aligned_to(scratch_dev, 16)) return fail(ANN_EINVAL, "scratch must be 16-byte aligned");
  DistillArgs a{};
  a.scores = static_cast<const char*>(scores_dev);
  a.rows = rows;
  a.n = (u32)n;
  a.ld = ld;
  a.ids = ids_dev;
  a.teacher = static_cast<const char*>(teacher_dev);
  a.tdtype = teacher_dtype;
  a.k = k;
  a.t = temperature;
  a.c = 1.44269504088896340736f / temperature;
  a.losses = losses_dev;
  a.stats = stats_dev;
  a.parts = static_cast<float*>(scratch_dev);
  set_chunks(a);
  return launch_distill(a, dtype, false, stream);
} catch (...) {
  return annmi::on_exception();
}

int ann_distill_grad(const void* scores_dev, uint64_t rows, uint64_t n, ann_dtype dtype, uint64_t ld, const uint32_t* ids_dev,
                     const void* teacher_dev, ann_dtype teacher_dtype, uint32_t k, float temperature, const float* stats_dev,
                     const float* grad_losses_dev, float scale, void* out_dev, uint64_t ldo, void* stream) try {
  bool work;
  int rc = check_distill("ann_distill_grad", scores_dev, rows, n, dtype, ld, ids_dev, teacher_dev, teacher_dtype, k, temperature, stats_dev, &work);
  if (rc) return rc;
  if (ldo < n) return fail(ANN_EINVAL, "ldo must be at least n");
  if (rows && ldo > DISTILL_MOST_PLACE / rows) return fail(ANN_EINVAL, "rows * ldo must be at most 2^60");
  if (!work) return ANN_OK;
  if (!out_dev) return fail(ANN_EINVAL, "null argument");
  if (!aligned_to(out_dev, dtype_bytes(dtype)) || !aligned_to(grad_losses_dev, 4)) return fail(ANN_EINVAL, "out or grad_losses not aligned to their elements");
  if (out_dev != scores_dev || (ldo != ld && rows > 1)) {
    // apart, or side by side in rows of the same stride
    const u64 esz = dtype_bytes(dtype);
    const uintptr_t from = reinterpret_cast<uintptr_t>(scores_dev), to = reinterpret_cast<uintptr_t>(out_dev);
    const u64 scores_end = from + ((rows - 1) * ld + n) * esz, out_end = to + ((rows - 1) * ldo + n) * esz;
    const u64 off = (from < to ? to - from : from - to) % (ld * esz);
    const bool beside = ld == ldo && off >= n * esz && off <= (ld - n) * esz;
    if (from < out_end && to < scores_end && !beside) return fail(ANN_EINVAL, "gradients must lie in the scores' place or apart from them");
  }
  DistillArgs a{};
  a.scores = static_cast<const char*>(scores_dev);
  a.rows = rows;
  a.n = (u32)n;
  a.ld = ld;
  a.ids = ids_dev;
  a.teacher = static_cast<const char*>(teacher_dev);
  a.tdtype = teacher_dtype;
  a.k = k;
  a.t = temperature;
  a.c = 1.44269504088896340736f / temperature;
  a.stats = const_cast<float*>(stats_dev);
  a.upstream = grad_losses_dev;
  a.scale = scale;
  a.out = static_cast<char*>(out_dev);
  a.ldo = ldo;
  set_chunks(a);
  if (rows >= 512) {  // in the rows' order: the fewer places memory is read and written at, the better
    a.chunk = std::min(a.chunk, (u32)(GRAD_CHUNK / dtype_bytes(dtype)));
    a.chunks = (a.n + a.chunk - 1) / a.chunk;
  }
  return launch_distill(a, dtype, true, stream);
} catch (...) {
  return annmi::on_exception();
}

}  // extern "C"
