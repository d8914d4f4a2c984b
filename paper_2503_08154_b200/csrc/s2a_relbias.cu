// Learned relative position bias by buckets, added to attention scores, and the gradient of its table.
//
//   y[b, h, q, k] = x[b, h, q, k] + table[bucket(q, k)][h]
//   grad_table[u][h] = sum over b and over the (q, k) of bucket u of grad_out[b, h, q, k]
//
// bucket(q, k) is buckets[q * tk + k] (a map: 2-D windows) or buckets[k - q + tq - 1] (a vector over the distance: 1-D
// sequences).  A bucket outside 0 .. n_buckets - 1 adds nothing and has no gradient.
//
// Both kernels walk the batch inside a thread: a thread owns eight positions (q, k) of one head, one 16-byte vector of
// bfloat16 (two of binary32), whose biases (whose sums) stay in registers while the samples pass.  The slab of one (sample, head), tq tk
// elements, need not start on a vector boundary: its first element sits s = (offset mod 8) into a vector, and s goes
// round as the sample advances.  So the samples are taken one class of equal s at a time (`period` classes, 1 to 8), and
// within a class a thread's vector covers the same positions in every sample.
#include <math.h>

#include "s2a_launch.h"
#include "s2a_oct.cuh"

namespace s2a {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kPrivateBuckets = 64; // up to here every thread has its own copy of the table
constexpr uint32_t kBwdCtas = 592;       // CTAs of the backward kernel: four per SM of a B200
constexpr uint32_t kTableBytes = 128 * 1024;  // shared memory for the tables of a CTA's warps

struct BiasArgs {
  const void* x;          // x or grad_out
  void* y;                // forward
  const void* table;      // forward
  const int32_t* buckets;
  float* partials;        // backward: [head][CTA of the head][n_buckets]
  uint64_t slab;          // tq * tk
  uint32_t batch, heads, tq, tk;
  uint32_t n_buckets;
  uint32_t period;        // classes of samples of equal alignment
  uint32_t lanes;         // threads of a CTA along the vectors of a slab (a power of two); the others along the batch
  uint32_t splits;        // parts of the batch
  uint32_t ctas_per_head; // backward
  uint32_t threads;       // of a CTA
  int by_distance, wdt;
};

// The bucket ids of positions p .. p + 7 of a slab; -1 outside the slab and for ids outside the table.
__device__ __forceinline__ void load_buckets(const BiasArgs& a, int64_t p, int* u) {
  int64_t q = 0, k = 0;
  if (a.by_distance) {
    const int64_t pc = p < 0 ? 0 : p;
    q = pc / a.tk;
    k = pc - q * a.tk;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t pi = p + i;
    u[i] = -1;
    if (pi < 0 || pi >= (int64_t)a.slab) continue;
    const int b = a.buckets[a.by_distance ? k - q + (int64_t)a.tq - 1 : pi];
    if (b >= 0 && (uint32_t)b < a.n_buckets) u[i] = b;
    if (++k == a.tk) {
      k = 0;
      ++q;
    }
  }
}

// The vector `vec` of a slab in class c: its first position (negative where the vector begins before the slab).
__device__ __forceinline__ int64_t first_position(const BiasArgs& a, uint64_t vec, uint32_t c, uint32_t h) {
  const uint32_t shift = (uint32_t)((((uint64_t)c * a.heads + h) * a.slab) & 7u);
  return (int64_t)(vec * 8) - shift;
}

template <int DT>
__global__ void __launch_bounds__(kThreads) bias_fwd_kernel(BiasArgs a) {
  using T = typename Io<DT>::T;
  enter_grid();
  const uint32_t lane = threadIdx.x % a.lanes, row = threadIdx.x / a.lanes, rows = kThreads / a.lanes;
  const uint64_t vec = (uint64_t)blockIdx.x * a.lanes + lane;
  const uint32_t classes = a.period < a.batch ? a.period : a.batch;
  for (uint32_t h = blockIdx.y; h < a.heads; h += gridDim.y) {
    for (uint32_t c = 0; c < classes; ++c) {
      const int64_t p = first_position(a, vec, c, h);
      if (p >= (int64_t)a.slab || p + 8 <= 0) continue;
      const bool whole = p >= 0 && p + 8 <= (int64_t)a.slab;
      int u[8];
      load_buckets(a, p, u);
      float bias[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) bias[i] = u[i] >= 0 ? load_param(a.table, (uint64_t)u[i] * a.heads + h, a.wdt) : 0.0f;
      F2 bias2[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) bias2[i] = f2_pack(bias[2 * i], bias[2 * i + 1]);
      const uint64_t step = (uint64_t)a.period * rows * gridDim.z;
      for (uint64_t b = c + (uint64_t)a.period * (blockIdx.z * rows + row); b < a.batch; b += step) {
        const int64_t e = (int64_t)((b * a.heads + h) * a.slab) + p;
        const T* x = (const T*)a.x + e;
        T* y = (T*)a.y + e;
        if (whole) {
          Eight<DT> v;
          v.load(x);
          F2 w[4];
          v.get(w);
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = f2_add(w[i], bias2[i]);
          v.set(w);
          v.store(y);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (p + i >= 0 && p + i < (int64_t)a.slab) y[i] = Io<DT>::narrow(Io<DT>::widen(x[i]) + bias[i]);
        }
      }
    }
  }
}

// ---- backward.  Each CTA works for one head: it sums its samples in registers, adds the sums into a table in shared
// memory, and writes that table to scratch; bias_table_kernel adds the CTAs' tables in order.  No atomics: with few
// buckets (PRIVATE) each thread adds into a column of its own; with more, each warp has a table, and lanes that meet in
// one bucket take turns in lane order.  Either way the same bits come out on every run.
template <int DT, bool PRIVATE>
__global__ void __launch_bounds__(kThreads) bias_bwd_kernel(BiasArgs a) {
  using T = typename Io<DT>::T;
  extern __shared__ float sums[];  // PRIVATE: [n_buckets][thread]; otherwise [warp][n_buckets]
  enter_grid();
  const uint32_t warps = blockDim.x / 32, warp = threadIdx.x / 32;
  const uint32_t cells = a.n_buckets * (PRIVATE ? blockDim.x : warps);
  for (uint32_t i = threadIdx.x; i < cells; i += blockDim.x) sums[i] = 0.0f;
  __syncthreads();
  const uint32_t h = blockIdx.x / a.ctas_per_head, j = blockIdx.x % a.ctas_per_head;
  const uint32_t lane = threadIdx.x % a.lanes, row = threadIdx.x / a.lanes, rows = blockDim.x / a.lanes;
  const uint64_t vecs = (a.slab + 7 + 7) / 8, chunks = (vecs + a.lanes - 1) / a.lanes;
  const uint32_t classes = a.period < a.batch ? a.period : a.batch;
  for (uint64_t item = j; item < chunks * a.splits; item += a.ctas_per_head) {
    const uint64_t vec = (item / a.splits) * a.lanes + lane;
    const uint32_t split = (uint32_t)(item % a.splits);
    for (uint32_t c = 0; c < classes; ++c) {
      const int64_t p = first_position(a, vec, c, h);
      const bool none = p >= (int64_t)a.slab || p + 8 <= 0, whole = p >= 0 && p + 8 <= (int64_t)a.slab;
      F2 acc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = f2_both(0.0f);
      const uint64_t step = (uint64_t)a.period * rows * a.splits;
      for (uint64_t b = c + (uint64_t)a.period * (split * rows + row); !none && b < a.batch; b += step) {
        const T* g = (const T*)a.x + ((int64_t)((b * a.heads + h) * a.slab) + p);
        F2 w[4];
        if (whole) {
          Eight<DT> v;
          v.load(g);
          v.get(w);
        } else {
          float f[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = p + i >= 0 && p + i < (int64_t)a.slab ? Io<DT>::widen(g[i]) : 0.0f;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = f2_pack(f[2 * i], f[2 * i + 1]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = f2_add(acc[i], w[i]);
      }
      int u[8];
      load_buckets(a, p, u);
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) f2_unpack(acc[i], v[2 * i], v[2 * i + 1]);
      if (PRIVATE) {
        int open = -1;  // neighbours of one bucket are added up before they go to memory
        float run = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (u[i] != open) {
            if (open >= 0) sums[(uint32_t)open * blockDim.x + threadIdx.x] += run;
            open = u[i];
            run = 0.0f;
          }
          run += v[i];
        }
        if (open >= 0) sums[(uint32_t)open * blockDim.x + threadIdx.x] += run;
      } else {
        float* mine = sums + (uint64_t)warp * a.n_buckets;
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
          int ui = u[0];
          float vi = v[0];
#pragma unroll
          for (int k = 1; k < 8; ++k) {
            ui = i == k ? u[k] : ui;
            vi = i == k ? v[k] : vi;
          }
          const unsigned peers = __match_any_sync(0xffffffffu, ui);
          const int turn = __popc(peers & ((1u << (threadIdx.x % 32)) - 1u));
          const int turns = __reduce_max_sync(0xffffffffu, ui >= 0 ? turn : 0);
          for (int t = 0; t <= turns; ++t) {
            if (turn == t && ui >= 0) mine[ui] += vi;
            __syncwarp();
          }
        }
      }
    }
  }
  __syncthreads();
  float* part = a.partials + (uint64_t)blockIdx.x * a.n_buckets;
  if (PRIVATE) {
    for (uint32_t u = warp; u < a.n_buckets; u += warps) {
      float t = 0.0f;
      for (uint32_t i = threadIdx.x % 32; i < blockDim.x; i += 32) t += sums[u * blockDim.x + i];
      t = warp_sum(t);
      if (threadIdx.x % 32 == 0) part[u] = t;
    }
  } else {
    for (uint32_t u = threadIdx.x; u < a.n_buckets; u += blockDim.x) {
      float t = 0.0f;
      for (uint32_t w = 0; w < warps; ++w) t += sums[(uint64_t)w * a.n_buckets + u];
      part[u] = t;
    }
  }
}

// [head][CTA of the head][n_buckets] -> grad_table[n_buckets][heads].  A CTA owns 32 buckets of one head; its eight
// warps take every eighth of the head's tables.
__global__ void __launch_bounds__(256) bias_table_kernel(const float* partials, uint32_t ctas_per_head, uint32_t n_buckets,
                                                         uint32_t heads, void* grad_table, int wdt) {
  __shared__ float sums[8][32];
  enter_grid();
  const uint32_t u = blockIdx.x * 32 + threadIdx.x % 32, w = threadIdx.x / 32;
  for (uint32_t h = blockIdx.y; h < heads; h += gridDim.y) {
    float t = 0.0f;
    if (u < n_buckets)
      for (uint32_t j = w; j < ctas_per_head; j += 8) t += partials[((uint64_t)h * ctas_per_head + j) * n_buckets + u];
    sums[w][threadIdx.x % 32] = t;
    __syncthreads();
    if (w == 0 && u < n_buckets) {
#pragma unroll
      for (int k = 1; k < 8; ++k) t += sums[k][threadIdx.x];
      store_param(grad_table, (uint64_t)u * heads + h, wdt, t);
    }
    __syncthreads();
  }
}

uint32_t gcd8(uint64_t v) {  // gcd(8, v mod 8), 8 for a multiple of 8
  v &= 7u;
  return v == 0 ? 8u : (v & 1u ? 1u : (v & 2u ? 2u : 4u));
}

// Threads of a backward CTA: eight warps, fewer where eight tables of n_buckets would not fit shared memory.
uint32_t bwd_threads(uint32_t n_buckets) {
  if (n_buckets <= kPrivateBuckets) return kThreads;
  uint32_t warps = kThreads / 32;
  while (warps > 1 && warps * n_buckets * sizeof(float) > kTableBytes) warps /= 2;
  return warps * 32;
}

// Fills the fields that follow from the shape.
BiasArgs shape_args(uint32_t batch, uint32_t heads, uint32_t tq, uint32_t tk, uint32_t n_buckets, uint32_t threads) {
  BiasArgs a = {};
  a.threads = threads;
  a.slab = (uint64_t)tq * tk;
  a.batch = batch;
  a.heads = heads;
  a.tq = tq;
  a.tk = tk;
  a.n_buckets = n_buckets;
  a.period = 8 / gcd8((uint64_t)heads * (a.slab & 7u));
  const uint64_t vecs = (a.slab + 14) / 8;
  a.lanes = 1;
  while (a.lanes < threads && a.lanes < vecs) a.lanes *= 2;
  return a;
}

uint32_t bwd_ctas_per_head(uint32_t heads, uint64_t items) {
  const uint64_t want = kBwdCtas / heads > 0 ? kBwdCtas / heads : 1;
  return (uint32_t)(want < items ? want : items);
}

// Parts of the batch: enough to give `ctas` CTAs work, no more than there are samples for.
uint32_t batch_splits(const BiasArgs& a, uint64_t chunks, uint64_t ctas) {
  const uint64_t rows = a.threads / a.lanes, most = (a.batch + a.period * rows - 1) / (a.period * rows);
  const uint64_t want = (ctas + chunks * a.heads - 1) / (chunks * a.heads);
  return (uint32_t)(want < 1 ? 1 : (want < most ? want : (most < 1 ? 1 : most)));
}

}  // namespace

uint32_t relbias_bwd_ctas(uint32_t batch, uint32_t heads, uint32_t tq, uint32_t tk, uint32_t n_buckets) {
  const BiasArgs a = shape_args(batch, heads, tq, tk, n_buckets, bwd_threads(n_buckets));
  const uint64_t chunks = ((a.slab + 14) / 8 + a.lanes - 1) / a.lanes;
  return heads * bwd_ctas_per_head(heads, chunks * batch_splits(a, chunks, kBwdCtas));
}

cudaError_t launch_relbias_fwd(int dt, int wdt, const void* x, const void* table, const int32_t* buckets, int by_distance,
                               void* y, uint32_t batch, uint32_t heads, uint32_t tq, uint32_t tk, uint32_t n_buckets,
                               cudaStream_t st) {
  BiasArgs a = shape_args(batch, heads, tq, tk, n_buckets, kThreads);
  a.x = x;
  a.y = y;
  a.table = table;
  a.buckets = buckets;
  a.by_distance = by_distance;
  a.wdt = wdt;
  const uint64_t chunks = ((a.slab + 14) / 8 + a.lanes - 1) / a.lanes;
  const uint32_t splits = batch_splits(a, chunks, (uint64_t)sm_count() * 8);
  const dim3 grid((unsigned)chunks, heads < 65535u ? heads : 65535u, splits < 65535u ? splits : 65535u);
  return dt == kF32 ? launch_overlapped(bias_fwd_kernel<kF32>, grid, kThreads, 0, st, a)
                    : launch_overlapped(bias_fwd_kernel<kBF16>, grid, kThreads, 0, st, a);
}

template <int DT, bool PRIVATE>
cudaError_t launch_bias_bwd(const BiasArgs& a, size_t smem, cudaStream_t st) {
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(bias_bwd_kernel<DT, PRIVATE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
  }
  return launch_overlapped(bias_bwd_kernel<DT, PRIVATE>, dim3(a.heads * a.ctas_per_head), a.threads, smem, st, a);
}

cudaError_t launch_relbias_bwd(int dt, int wdt, const void* g, const int32_t* buckets, int by_distance, void* grad_table,
                               float* scratch, uint32_t batch, uint32_t heads, uint32_t tq, uint32_t tk, uint32_t n_buckets,
                               cudaStream_t st) {
  if ((uint64_t)batch * tq * tk == 0)  // a sum over nothing
    return cudaMemsetAsync(grad_table, 0, (size_t)n_buckets * heads * (wdt == kF32 ? 4u : 2u), st);
  BiasArgs a = shape_args(batch, heads, tq, tk, n_buckets, bwd_threads(n_buckets));
  a.x = g;
  a.buckets = buckets;
  a.by_distance = by_distance;
  a.partials = scratch;
  const uint64_t chunks = ((a.slab + 14) / 8 + a.lanes - 1) / a.lanes;
  a.splits = batch_splits(a, chunks, kBwdCtas);
  a.ctas_per_head = bwd_ctas_per_head(heads, chunks * a.splits);
  cudaError_t e;
  if (n_buckets <= kPrivateBuckets) {
    const size_t smem = (size_t)n_buckets * kThreads * sizeof(float);
    e = dt == kF32 ? launch_bias_bwd<kF32, true>(a, smem, st) : launch_bias_bwd<kBF16, true>(a, smem, st);
  } else {
    const size_t smem = (size_t)n_buckets * (a.threads / 32) * sizeof(float);
    e = dt == kF32 ? launch_bias_bwd<kF32, false>(a, smem, st) : launch_bias_bwd<kBF16, false>(a, smem, st);
  }
  if (e != cudaSuccess) return e;
  return launch_overlapped(bias_table_kernel, dim3((n_buckets + 31) / 32, heads < 65535u ? heads : 65535u), 256, 0, st,
                           scratch, a.ctas_per_head, n_buckets, heads, grad_table, wdt);
}

// The bucket of a distance, on the host.  Buckets of short distances hold one distance each; past max_exact (half of a
// side's buckets) they widen geometrically up to max_distance: bucket max_exact + j starts at the smallest n with
// n >= max_exact (max_distance / max_exact)^(j / (side - max_exact)).  The power is taken in long double, and a value that
// lies within its rounding of a whole number counts as that number (8 * 16^(2/4) is 32, not the next double above it).
void log_buckets(int32_t* out, int64_t first, uint64_t count, uint32_t n_buckets, uint32_t max_distance, bool bidirectional) {
  const uint32_t side = bidirectional ? n_buckets / 2 : n_buckets, exact = side / 2, wide = side - exact;
  const auto start = [=](uint32_t u) -> int64_t {  // the smallest n of bucket u of a side; beyond the last, no end
    if (u <= exact) return u;
    if (u >= side) return INT64_MAX;
    const long double v = exact * powl((long double)max_distance / exact, (long double)(u - exact) / wide), near = roundl(v);
    return (int64_t)(fabsl(v - near) <= 1e-15L * v ? near : ceill(v));
  };
  const int64_t end = first + (int64_t)count;  // distances first .. end - 1, d = k - q
  for (uint32_t u = 0; u < side; ++u) {
    const int64_t low = start(u), high = start(u + 1);
    // keys behind the query: d = -n for n = low .. high - 1
    for (int64_t d = high == INT64_MAX || 1 - high < first ? first : 1 - high; d < end && d <= -low; ++d) out[d - first] = (int32_t)u;
    // keys ahead of it: d = n, with buckets of their own, or all in bucket 0 where only the past counts
    if (bidirectional)
      for (int64_t d = low > first ? low : first; d < end && d < high; ++d) out[d - first] = (int32_t)(d > 0 ? u + side : u);
  }
  if (!bidirectional)
    for (int64_t d = first > 1 ? first : 1; d < end; ++d) out[d - first] = 0;
}

}  // namespace s2a
